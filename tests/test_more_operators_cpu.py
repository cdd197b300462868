"""CPU checks of the operators between projection, attention and cache: the packed argument structs match the C layout, and
every entry point refuses what it documents as refused before it touches a device (the pointers here are never read)."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2606_09682_b200 import build as amk_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED = 0, 1, 2
P = 0x7F0000000000                                    # an aligned address that no call here reads
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def amk():
    amk_build.build()
    from paper_2606_09682_b200 import binding
    return binding


def structs(amk):
    return (("amk_rope_args", amk._ROPE), ("amk_attention_weights_args", amk._WEIGHTS), ("amk_verify_args", amk._VERIFY))


def test_argument_structs_match_the_header(amk, tmp_path):
    lines, want = ['#include <stdio.h>', '#include <stddef.h>', '#include "amk.h"', "int main(void){"], []
    for name, fmt in structs(amk):
        cls = getattr(amk, name)
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(cls))
        assert fmt.size == C.sizeof(cls)
        for field, _ in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {field}));')
            want.append(getattr(cls, field).offset)
        values = [i + 1 for i in range(len(cls._fields_))]
        got = cls.from_buffer_copy(fmt.pack(*values))
        assert [getattr(got, f) for f, _ in cls._fields_] == values
    src = tmp_path / "t.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "t"), str(src)], check=True)
    assert [int(x) for x in subprocess.run([str(tmp_path / "t")], check=True, capture_output=True, text=True).stdout.split()] == want


def packed(amk, name, fmt, given, kw):
    assert set(kw) <= set(given)
    given = {**given, **kw}
    return fmt.pack(*[given[f] for f, _ in getattr(amk, name)._fields_])


def rope_args(amk, **kw):
    return packed(amk, "amk_rope_args", amk._ROPE, dict(
        struct_size=amk._ROPE.size, head_dim=64, n_q_heads=4, n_kv_heads=2, kv_dtype=0, n_seqs=2, n_slots=100, eps=1e-5, theta=1e4,
        reserved=0, rows=10, q=P, k=P, v=P, q_weight=0, k_weight=0, positions=P, slots=P, q_out=P, k_out=0, k_cache=P, v_cache=P,
        q_row=512, q_head=64, k_row=512, k_head=64, v_row=512, v_head=64, qo_row=256, qo_head=64, ko_row=128, ko_head=64,
        kc_seq=12800, kc_head=6400, kc_row=64, vc_seq=12800, vc_head=6400, vc_row=64), kw)


def weights_args(amk, **kw):
    return packed(amk, "amk_attention_weights_args", amk._WEIGHTS, dict(
        struct_size=amk._WEIGHTS.size, head_dim=64, n_q_heads=4, n_kv_heads=2, kv_dtype=0, n_seqs=2, n_rows=3, n_slots=100,
        scale=0.0, decay=1.0, q=P, k=P, lse=P, cache_len=P, before=P, out=P, workspace=P, workspace_bytes=1 << 40, q_seq=768,
        q_row=256, q_head=64, k_seq=12800, k_head=6400, k_row=64, before_seq=200, before_head=100, out_seq=200, out_head=100), kw)


def verify_args(amk, **kw):
    return packed(amk, "amk_verify_args", amk._VERIFY, dict(
        struct_size=amk._VERIFY.size, dtype=0, n_seqs=2, n_rows=3, vocab=100, logits=P, draft=P, tokens=P, parents=0, uniforms=P,
        temperature=0, cache_len=0, count=P, keep=P, token=P, workspace=P, workspace_bytes=1 << 40, logits_seq=300,
        logits_row=100, draft_seq=300, draft_row=100), kw)


def evict_args(**kw):
    a = dict(scores=P, seqs=2, heads=3, slots=100, seq=300, head=100, lens=P, budget=20, first=4, recent=8, keep=P, count=P,
             moved=0, mseq=300, mhead=100)
    assert set(kw) <= set(a)
    a.update(kw)
    return tuple(a.values())


def refused(fn, args, code, *words):
    msg = C.create_string_buffer(256)
    assert fn(*args, msg, 256, None) == code, msg.value
    for w in words:
        assert w.encode() in msg.value, msg.value
    assert fn(*args, None, 0, None) == code            # the reason is optional


@pytest.mark.parametrize("kw,code,word", [
    (dict(struct_size=8), INVALID, "struct_size"), (dict(reserved=1), INVALID, "reserved"), (dict(head_dim=96), UNSUPPORTED, "head_dim"),
    (dict(n_q_heads=0), UNSUPPORTED, "heads"), (dict(n_kv_heads=4097), UNSUPPORTED, "4096"), (dict(kv_dtype=2), UNSUPPORTED, "kv_dtype"),
    (dict(eps=-1e-9), INVALID, "eps"), (dict(eps=NAN), INVALID, "eps"), (dict(eps=INF), INVALID, "eps"),
    (dict(theta=0.0), INVALID, "theta"), (dict(theta=NAN), INVALID, "theta"), (dict(theta=INF), INVALID, "theta"),
    (dict(rows=-1), INVALID, "rows"), (dict(rows=1 << 31), INVALID, "rows"), (dict(v_cache=0), INVALID, "both"), (dict(k_cache=0), INVALID, "both"),
    (dict(n_seqs=0), INVALID, "caches"), (dict(n_slots=0), INVALID, "caches"), (dict(n_slots=1 << 31), INVALID, "caches"),
    (dict(q=0), INVALID, "NULL"), (dict(k=0), INVALID, "NULL"), (dict(v=0), INVALID, "NULL"), (dict(positions=0), INVALID, "NULL"),
    (dict(slots=0), INVALID, "NULL"), (dict(q_out=0), INVALID, "NULL"), (dict(q=P + 8), INVALID, "aligned"), (dict(k_weight=P + 2), INVALID, "aligned"),
    (dict(k_cache=P + 8), INVALID, "aligned"), (dict(k_out=P + 4), INVALID, "aligned"), (dict(positions=P + 2), INVALID, "positions"),
    (dict(slots=P + 4), INVALID, "slots"), (dict(q_row=260), INVALID, "q row"), (dict(k_head=32), INVALID, "k head"), (dict(v_row=0), INVALID, "v row"),
    (dict(qo_head=-64), INVALID, "q_out head"), (dict(k_out=P, ko_row=8), INVALID, "k_out row"), (dict(kc_row=0), INVALID, "k_cache row"),
    (dict(vc_seq=4), INVALID, "v_cache sequence"), (dict(kv_dtype=1, kc_row=72), INVALID, "k_cache row"), (dict(q_row=1 << 40), INVALID, "q row"),
])
def test_norm_rope_append_refuses(amk, kw, code, word):
    refused(amk.lib.amk_norm_rope_append, (rope_args(amk, **kw),), code, "amk_norm_rope_append: ", word)


@pytest.mark.parametrize("kw", [dict(), dict(q_out=P + 4096, k_out=P), dict(qo_row=512, k_out=P, ko_row=520), dict(qo_row=512, qo_head=72)])
def test_norm_rope_append_refuses_outputs_over_inputs_at_other_strides(amk, kw):
    refused(amk.lib.amk_norm_rope_append, (rope_args(amk, **kw),), INVALID, "amk_norm_rope_append: ", "other strides")


@pytest.mark.parametrize("kw,code,word", [
    (dict(struct_size=8), INVALID, "struct_size"), (dict(head_dim=32), UNSUPPORTED, "head_dim"), (dict(n_q_heads=34), UNSUPPORTED, "16"),
    (dict(n_q_heads=3), UNSUPPORTED, "multiple"), (dict(kv_dtype=2), UNSUPPORTED, "kv_dtype"), (dict(decay=NAN), INVALID, "decay"),
    (dict(decay=-INF), INVALID, "decay"), (dict(scale=-1.0), INVALID, "scale"), (dict(scale=3e38), INVALID, "scale"),
    (dict(n_rows=0), INVALID, "tokens"), (dict(n_rows=101), INVALID, "slots"), (dict(n_slots=0x7FFFFFFF), INVALID, "slots"),
    (dict(n_seqs=65536), UNSUPPORTED, "sequences"), (dict(n_seqs=60000, n_slots=1 << 20, n_rows=1 << 19), UNSUPPORTED, "2^31"),
    (dict(q=0), INVALID, "NULL"), (dict(k=0), INVALID, "NULL"), (dict(lse=0), INVALID, "NULL"), (dict(cache_len=0), INVALID, "NULL"),
    (dict(out=0), INVALID, "NULL"), (dict(q=P + 8), INVALID, "aligned"), (dict(before=P + 2), INVALID, "aligned"), (dict(out=P + 1), INVALID, "aligned"),
    (dict(workspace=P + 128), INVALID, "aligned"), (dict(q_row=8), INVALID, "q row"), (dict(k_row=0), INVALID, "k row"),
    (dict(kv_dtype=1, k_row=72), INVALID, "k row"), (dict(out_head=99), INVALID, "sums"), (dict(out_seq=0), INVALID, "sums"),
    (dict(before_seq=-200), INVALID, "sums"), (dict(out=P, before=P, before_head=104, before_seq=208), INVALID, "other strides"),
])
def test_attention_weights_refuses(amk, kw, code, word):
    refused(amk.lib.amk_attention_weights, (weights_args(amk, **kw),), code, "amk_attention_weights: ", word)


@pytest.mark.parametrize("kw,word", [
    (dict(seqs=-1), "sequences"), (dict(heads=0), "heads"), (dict(slots=0), "slots"), (dict(seqs=1 << 30), "sequences"),
    (dict(budget=0), "budget"), (dict(budget=101), "budget"), (dict(first=-1), "first"), (dict(recent=-1), "recent"),
    (dict(first=10, recent=11), "together"), (dict(first=1 << 62, recent=1 << 62), "together"), (dict(scores=None), "NULL"), (dict(lens=None), "NULL"),
    (dict(keep=None), "NULL"), (dict(count=None), "NULL"), (dict(scores=P + 2), "aligned"), (dict(moved=P + 1), "aligned"),
    (dict(head=99), "strides"), (dict(seq=-300), "strides"), (dict(moved=P + 64, mhead=0), "strides"),
    (dict(moved=P, mhead=104, mseq=312), "other strides"),
])
def test_evict_select_refuses(amk, kw, word):
    refused(amk.lib.amk_evict_select, evict_args(**kw), INVALID, "amk_evict_select: ", word)


@pytest.mark.parametrize("kw,code,word", [
    (dict(struct_size=8), INVALID, "struct_size"), (dict(dtype=2), UNSUPPORTED, "dtype"), (dict(n_rows=0), UNSUPPORTED, "rows"),
    (dict(n_rows=1025), UNSUPPORTED, "1024"), (dict(vocab=0), INVALID, "logits"), (dict(vocab=1 << 31), INVALID, "logits"),
    (dict(n_seqs=1 << 30), INVALID, "sequences"), (dict(logits=0), INVALID, "NULL"), (dict(tokens=0), INVALID, "NULL"),
    (dict(uniforms=0), INVALID, "NULL"), (dict(count=0), INVALID, "NULL"), (dict(keep=0), INVALID, "NULL"), (dict(token=0), INVALID, "NULL"),
    (dict(logits=P + 2), INVALID, "aligned"), (dict(draft=P + 2), INVALID, "aligned"), (dict(parents=P + 1), INVALID, "aligned"),
    (dict(workspace=P + 128), INVALID, "aligned"), (dict(dtype=1, logits=P + 1), INVALID, "aligned"), (dict(logits_row=99), INVALID, "strides"),
    (dict(logits_seq=-1), INVALID, "strides"), (dict(draft_row=0), INVALID, "strides"),
    (dict(workspace_bytes=10), INVALID, "workspace"), (dict(workspace=0), INVALID, "workspace"),
])
def test_verify_draft_refuses(amk, kw, code, word):
    refused(amk.lib.amk_verify_draft, (verify_args(amk, **kw),), code, "amk_verify_draft: ", word)


def test_workspace_sizes(amk):
    n, msg = C.c_size_t(), C.create_string_buffer(256)
    for fn, args in ((amk.lib.amk_attention_weights_workspace_bytes, weights_args), (amk.lib.amk_verify_workspace_bytes, verify_args)):
        assert fn(None, C.byref(n), msg, 256) == INVALID
        assert fn(args(amk), None, msg, 256) == INVALID
        assert fn(args(amk, n_rows=0), C.byref(n), msg, 256) in (INVALID, UNSUPPORTED)
        assert fn(args(amk), C.byref(n), msg, 256) == OK


def test_empty_calls_do_nothing(amk):
    assert amk.lib.amk_norm_rope_append(rope_args(amk, rows=0, q=0, q_out=0), None, 0, None) == OK
    assert amk.lib.amk_attention_weights(weights_args(amk, n_seqs=0, q=0, out=0), None, 0, None) == OK
    assert amk.lib.amk_evict_select(*evict_args(seqs=0, scores=None), None, 0, None) == OK
    assert amk.lib.amk_verify_draft(verify_args(amk, n_seqs=0, logits=0, workspace=0), None, 0, None) == OK


def test_python_layer_refuses_host_tensors(amk):
    import torch
    x, n = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    f = torch.zeros(2, 4, 64)
    for call in (lambda: amk.amk_norm_rope_append(x, x, None, n), lambda: amk.amk_attention_weights(x[None], x[None], f[None, :, :, 0], n[:1]),
                 lambda: amk.amk_evict_select(f, n, 3), lambda: amk.amk_verify_draft(f, torch.zeros(2, 4, dtype=torch.int32), f[..., 0])):
        with pytest.raises(amk.AmkError) as e:
            call()
        assert e.value.code == INVALID and "cuda" in str(e.value)
