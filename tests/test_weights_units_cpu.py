"""CPU check of how the work of amk_attention_weights is divided between blocks (tests/native/weights_units_check.cpp replays it), with
sequences of impossible length among the others."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LOWEST = -(1 << 31)


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("native") / "weights_units_check")
    subprocess.run(["g++", "-O2", "-std=c++17", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2606_09682_b200", "csrc"), "-o", exe,
                    os.path.join(ROOT, "tests", "native", "weights_units_check.cpp")], check=True)

    def run(*args):
        r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True)
        assert r.returncode == 0 and r.stdout == "ok\n", (args, r.stdout, r.stderr)
    return run


@pytest.mark.parametrize("span,rows,tokens", [(128, 1, 1), (128, 32, 32), (160, 129, 128), (160, 200, 32), (160, 1000, 32), (160, 2500, 18), (160, 700, 8)])
@pytest.mark.parametrize("nkv", [1, 8])
@pytest.mark.parametrize("blocks", [1, 7, 148])
def test_every_step_is_one_blocks(check, span, rows, tokens, nkv, blocks):
    slots = rows + 1900
    for lens in ([0], [1900], [159], [160], [161], [0, 1, 1900, 320, 777], [1899, 3, 1900] * 15):
        check(span, nkv, rows, slots, tokens, blocks, *lens)


@pytest.mark.parametrize("span,rows,tokens", [(128, 32, 32), (160, 1000, 32), (160, 200, 8)])
@pytest.mark.parametrize("length", [-1, -159, -160, -161, -320, -321, -1000, -1000000, -20000000, LOWEST, LOWEST + 1, LOWEST + 159, 2001, 2147483647])
def test_a_sequence_of_impossible_length_has_no_steps(check, span, rows, tokens, length):
    for lens in ([length], [length, 1500, 30], [1500, length, 30], [1500, 30, length], [length] * 40 + [999]):
        check(span, 8, rows, rows + 2000, tokens, 148, *lens)
