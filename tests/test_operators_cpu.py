"""CPU checks of the operators around the decode step: the packed argument structs match the C layout, and every entry
point refuses what it documents as refused before it touches a device (the pointers here are never read)."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2606_09682_b200 import build as amk_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED = 0, 1, 2
P = 0x7F0000000000                                    # an aligned address that no call here reads


@pytest.fixture(scope="module")
def amk():
    amk_build.build()
    from paper_2606_09682_b200 import binding
    return binding


def test_argument_structs_match_the_header(amk, tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "amk.h"', "int main(void){"]
    want = []
    for name, fmt in (("amk_prompt_args", amk._PROMPT), ("amk_tree_args", amk._TREE)):
        cls = getattr(amk, name)
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(cls))
        assert fmt.size == C.sizeof(cls)
        for field, _ in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {field}));')
            want.append(getattr(cls, field).offset)
        # the format puts a distinct value into every field, in the same order
        values = [i + 1 for i in range(len(cls._fields_))]
        got = cls.from_buffer_copy(fmt.pack(*values))
        assert [getattr(got, f) for f, _ in cls._fields_] == values
    for macro in ("AMK_TREE_MAX_ROWS", "AMK_LOGPROBS_MAX_TOP"):
        lines.append(f'printf("%d\\n", {macro});')
        want.append(getattr(amk, macro))
    lines.append("return 0;}")
    src = tmp_path / "t.c"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "t"), str(src)], check=True)
    assert [int(x) for x in subprocess.run([str(tmp_path / "t")], check=True, capture_output=True, text=True).stdout.split()] == want


def prompt_args(amk, **kw):
    a = dict(struct_size=amk._PROMPT.size, head_dim=64, n_q_heads=4, n_kv_heads=2, n_seqs=1, scale=0.0, total=10, q=P, k=P,
             v=P, out=P, lse=0, cu_seqlens=P, q_row=256, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64,
             out_row=256, out_head=64)
    assert set(kw) <= set(a)
    a.update(kw)
    return amk._PROMPT.pack(*[a[f] for f, _ in amk.amk_prompt_args._fields_])


def tree_args(amk, **kw):
    a = dict(struct_size=amk._TREE.size, head_dim=64, n_q_heads=4, n_kv_heads=2, kv_dtype=0, n_seqs=2, n_rows=3,
             n_slots=100, max_len=0, scale=0.0, q=P, k=P, v=P, out=P, lse=0, cache_len=P, mask=0, workspace=P,
             workspace_bytes=1 << 40, q_seq=768, q_row=256, q_head=64, k_seq=12800, k_head=6400, k_row=64, v_seq=12800,
             v_head=6400, v_row=64, out_seq=768, out_row=256, out_head=64)
    assert set(kw) <= set(a)
    a.update(kw)
    return amk._TREE.pack(*[a[f] for f, _ in amk.amk_tree_args._fields_])


def refused(fn, args, code, *words):
    msg = C.create_string_buffer(256)
    assert fn(*args, msg, 256, None) == code, msg.value
    for w in words:
        assert w.encode() in msg.value, msg.value
    assert fn(*args, None, 0, None) == code            # the reason is optional


NAN = float("nan")


@pytest.mark.parametrize("kw,code,word", [
    (dict(struct_size=8), INVALID, "struct_size"), (dict(head_dim=96), UNSUPPORTED, "head_dim 96"),
    (dict(n_q_heads=5), UNSUPPORTED, "multiple"), (dict(n_q_heads=34, n_kv_heads=2), UNSUPPORTED, "16"),
    (dict(n_q_heads=4098), UNSUPPORTED, "4096"), (dict(n_kv_heads=0), UNSUPPORTED, "heads"), (dict(n_q_heads=0), UNSUPPORTED, "heads"),
    (dict(scale=-1.0), INVALID, "scale"), (dict(scale=NAN), INVALID, "scale"), (dict(scale=float("inf")), INVALID, "scale"),
    (dict(total=-1), INVALID, "rows"), (dict(total=1 << 31), INVALID, "rows"),
    (dict(q=0), INVALID, "NULL"), (dict(k=0), INVALID, "NULL"), (dict(v=0), INVALID, "NULL"),
    (dict(out=0), INVALID, "NULL"), (dict(cu_seqlens=0), INVALID, "NULL"),
    (dict(q=P + 8), INVALID, "aligned"), (dict(k=P + 2), INVALID, "aligned"), (dict(v=P + 4), INVALID, "aligned"),
    (dict(out=P + 8), INVALID, "aligned"), (dict(lse=P + 2), INVALID, "aligned"), (dict(cu_seqlens=P + 1), INVALID, "aligned"),
    (dict(q_row=260), INVALID, "q row"), (dict(k_row=0), INVALID, "k row"), (dict(v_row=-128), INVALID, "v row"),
    (dict(k_head=32), INVALID, "k head"), (dict(q_head=68), INVALID, "q head"), (dict(v_head=0), INVALID, "v head"),
    (dict(out_row=0), INVALID, "out row"), (dict(out_head=0), INVALID, "out head"),
])
def test_prompt_attention_refuses(amk, kw, code, word):
    refused(amk.lib.amk_prompt_attention, (prompt_args(amk, **kw),), code, "amk_prompt_attention: ", word)


@pytest.mark.parametrize("kw,code,word", [
    (dict(struct_size=8), INVALID, "struct_size"), (dict(head_dim=32), UNSUPPORTED, "head_dim"),
    (dict(n_q_heads=34), UNSUPPORTED, "16"), (dict(kv_dtype=2), UNSUPPORTED, "kv_dtype"),
    (dict(n_rows=0), UNSUPPORTED, "drafted"), (dict(n_rows=1025, n_slots=4000), UNSUPPORTED, "1024"),
    (dict(n_slots=2), INVALID, "slots"), (dict(n_slots=0x7FFFFFFF), INVALID, "slots"),
    (dict(n_seqs=65536), UNSUPPORTED, "sequences"), (dict(scale=-0.5), INVALID, "scale"),
    (dict(q=0), INVALID, "NULL"), (dict(k=0), INVALID, "NULL"), (dict(cache_len=0), INVALID, "NULL"),
    (dict(mask=P + 4), INVALID, "aligned"), (dict(workspace=P + 128), INVALID, "aligned"), (dict(v=P + 8), INVALID, "aligned"),
    (dict(k_row=8), INVALID, "k row"), (dict(k_row=0), INVALID, "k row"), (dict(v_seq=0), INVALID, "v sequence"),
    (dict(kv_dtype=1, k_row=72), INVALID, "k row"), (dict(q_seq=4), INVALID, "q sequence"),
    (dict(out_seq=0), INVALID, "out sequence"),
])
def test_tree_attention_refuses(amk, kw, code, word):
    refused(amk.lib.amk_tree_attention, (tree_args(amk, **kw),), code, "amk_tree_attention: ", word)


def test_tree_workspace_refuses(amk):
    n, msg = C.c_size_t(), C.create_string_buffer(256)
    assert amk.lib.amk_tree_workspace_bytes(None, C.byref(n), msg, 256) == INVALID
    assert amk.lib.amk_tree_workspace_bytes(tree_args(amk), None, msg, 256) == INVALID
    assert amk.lib.amk_tree_workspace_bytes(tree_args(amk, n_rows=0), C.byref(n), msg, 256) == UNSUPPORTED
    assert b"drafted" in msg.value


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_a_scale_whose_product_with_log2e_overflows_is_refused(amk, scale):
    refused(amk.lib.amk_prompt_attention, (prompt_args(amk, scale=scale),), INVALID, "scale")
    refused(amk.lib.amk_tree_attention, (tree_args(amk, scale=scale),), INVALID, "scale")


@pytest.mark.parametrize("scale", [1e-46, 1e-320, 1e39, 0.0, -1.0, NAN, float("inf")])
def test_python_scale_is_the_one_that_fp32_holds(amk, scale):
    """A positive number that rounds to zero would mean the default."""
    with pytest.raises(amk.AmkError) as e:
        amk._scale("call", scale)
    assert e.value.code == INVALID and "scale" in str(e.value)
    assert amk._scale("call", None) == 0.0 and amk._scale("call", 0.125) == 0.125 and 0 < amk._scale("call", 1e-45) < 2e-45


def logprob_args(**kw):
    a = dict(logits=P, dtype=0, rows=3, vocab=100, stride=100, tokens=P, top=2, lp=P, ent=P, ids=P, tlp=P)
    assert set(kw) <= set(a)
    a.update(kw)
    return tuple(a.values())


@pytest.mark.parametrize("kw,code,word", [
    (dict(dtype=2), UNSUPPORTED, "dtype"), (dict(top=33), UNSUPPORTED, "AMK_LOGPROBS_MAX_TOP"), (dict(rows=-1), INVALID, "rows"),
    (dict(vocab=0), INVALID, "rows of 0"), (dict(vocab=1 << 31), INVALID, "logits"), (dict(stride=99), INVALID, "row_stride"),
    (dict(logits=None), INVALID, "NULL"), (dict(tokens=None), INVALID, "NULL"), (dict(ids=None), INVALID, "NULL"),
    (dict(tlp=None), INVALID, "NULL"), (dict(logits=P + 2), INVALID, "aligned"), (dict(tokens=P + 2), INVALID, "aligned"),
    (dict(dtype=1, logits=P + 1), INVALID, "aligned"), (dict(ent=P + 3), INVALID, "aligned"),
])
def test_token_logprobs_refuses(amk, kw, code, word):
    refused(amk.lib.amk_token_logprobs, logprob_args(**kw), code, "amk_token_logprobs: ", word)


def compact_args(**kw):
    a = dict(kv=P, caches=2, stride=16 * 100 * 8, planes=8, seq=100, row=16, base=P, keep=P, most=10, count=P)
    assert set(kw) <= set(a)
    a.update(kw)
    return tuple(a.values())


@pytest.mark.parametrize("kw,word", [
    (dict(caches=-1), "caches"), (dict(planes=0), "planes"), (dict(seq=0), "rows"), (dict(most=101), "kept"),
    (dict(most=-1), "kept"), (dict(row=24), "row_bytes"), (dict(row=0), "row_bytes"), (dict(row=1040), "row_bytes"),
    (dict(kv=None), "NULL"), (dict(base=None), "NULL"), (dict(keep=None), "NULL"), (dict(count=None), "NULL"),
    (dict(kv=P + 8), "aligned"), (dict(keep=P + 2), "aligned"), (dict(stride=16 * 100 * 8 - 16), "cache_stride"),
    (dict(stride=16 * 100 * 8 + 8), "cache_stride"), (dict(stride=0), "cache_stride"),
    (dict(caches=1 << 20, planes=1 << 12, stride=16 * 100 * (1 << 12)), "planes"),
])
def test_kv_compact_refuses(amk, kw, word):
    refused(amk.lib.amk_kv_compact, compact_args(**kw), INVALID, "amk_kv_compact: ", word)


def test_empty_calls_do_nothing(amk):
    """Nothing to compute: the call succeeds without a device."""
    assert amk.lib.amk_prompt_attention(prompt_args(amk, total=0, q=0, k=0, v=0, out=0), None, 0, None) == OK
    assert amk.lib.amk_prompt_attention(prompt_args(amk, n_seqs=0), None, 0, None) == OK
    assert amk.lib.amk_tree_attention(tree_args(amk, n_seqs=0, q=0), None, 0, None) == OK
    assert amk.lib.amk_token_logprobs(*logprob_args(rows=0, logits=None), None, 0, None) == OK
    assert amk.lib.amk_kv_compact(*compact_args(caches=0, kv=None), None, 0, None) == OK
    assert amk.lib.amk_kv_compact(*compact_args(most=0), None, 0, None) == OK


def test_python_layer_refuses_host_tensors(amk):
    import torch
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    cu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(amk.AmkError) as e:
        amk.amk_prompt_attention(q, q, q, cu)
    assert e.value.code == INVALID and "cuda" in str(e.value)
    with pytest.raises(amk.AmkError):
        amk.amk_token_logprobs(torch.zeros(2, 10), cu)
    with pytest.raises(amk.AmkError):
        amk.amk_kv_compact(torch.zeros(1, 2, 4, 64), cu[:1], cu[None], cu[:1])
    with pytest.raises(amk.AmkError):
        amk.amk_tree_attention(q[None], torch.zeros(1, 4, 8, 64, dtype=torch.bfloat16),
                               torch.zeros(1, 4, 8, 64, dtype=torch.bfloat16), cu[:1])
