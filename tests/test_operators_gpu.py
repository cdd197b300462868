"""GPU tests of the operators around the decode step, each against a plain implementation in 64 bits.

Tolerance of the attentions, element by element.  With p the normalised softmax weights and A = sum p |v|:
  - the numerators enter the second product rounded to bf16, each off by at most 2^-8 of itself: 2^-8 A;
  - a score is a sum of head_dim exact products in fp32: off by at most E = head_dim 2^-23 sum |q||k| scale (2^-23: also
    for adders that truncate), which changes a weight by a factor within e^(+-2E), E far below 1: 2 E A (1 + small);
  - exponentials (2^-21 relative), the sums over n keys (n 2^-24 each for numerator and denominator: 2^-12 for 4096 keys,
    far less in practice), taken together as 2^-10 A;
  - one rounding of the result: 2^-8 |out|.
The log-sum-exp is off by E + n 2^-24 + 2^-20 (1 + |lse|).
"""
import math

import numpy as np
import pytest
import torch

from paper_2606_09682_b200 import inputs as inp

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def amk():
    from paper_2606_09682_b200 import binding
    return binding


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def attention64(q, k, v, sees, scale):
    """(out, lse, tolerance, tolerance of lse, rows that see a value that is not finite) for one sequence:
    q [t][nq][hd], k / v [n][nkv][hd], sees [t][n]; nothing that a row does not see is used for it."""
    hd, rep, n = q.shape[2], q.shape[1] // k.shape[1], k.shape[0]
    qd = q.double().permute(1, 0, 2)
    kd = k.double().permute(1, 0, 2).repeat_interleave(rep, 0)
    vd = v.double().permute(1, 0, 2).repeat_interleave(rep, 0)
    broken = ~(torch.isfinite(kd).all(2) & torch.isfinite(vd).all(2))              # [nq][n]
    touched = (sees[None] & broken[:, None]).any(2)                                # [nq][t]
    kd, vd = torch.nan_to_num(kd, 0, 0, 0), torch.nan_to_num(vd, 0, 0, 0)
    x = (qd @ kd.transpose(1, 2) * scale).masked_fill(~sees[None], -math.inf)
    lse = torch.logsumexp(x, 2)
    p = torch.where(sees[None], torch.exp(x - torch.where(torch.isinf(lse), 0.0, lse)[..., None]), 0.0)
    out, A = p @ vd, p @ vd.abs()
    mag = (qd.abs() @ kd.abs().transpose(1, 2)).masked_fill(~sees[None], 0.0)
    E = hd * 2.0 ** -23 * scale * (mag.amax(2) if n else torch.zeros_like(lse))
    tol = (2.0 ** -8 + 2.0 ** -10 + 2.2 * E[..., None]) * A + 2.0 ** -8 * out.abs() + 1e-30
    tol_lse = E + n * 2.0 ** -24 + 2.0 ** -20 * (1 + torch.nan_to_num(lse, 0, 0, 0).abs())
    return (out.permute(1, 0, 2), lse.permute(1, 0), tol.permute(1, 0, 2), tol_lse.permute(1, 0), touched.permute(1, 0))


def check(out, lse, ref, what=""):
    o, l, tol, tol_l, touched = ref
    fine = ~touched
    err = (out.double() - o).abs()[fine]
    assert bool((err <= tol[fine]).all()), (what, float((err / tol[fine]).max()), int((~(err <= tol[fine])).sum()))
    if lse is not None:
        a, b = lse.double()[fine], l[fine]
        empty = torch.isinf(b)
        assert torch.equal(a[empty], b[empty]), what
        d = (a - b).abs()[~empty]
        assert bool((d <= tol_l[fine][~empty]).all()), (what, float((d / tol_l[fine][~empty]).max()))


def causal(n):
    return torch.ones(n, n, dtype=torch.bool, device=DEV).tril()


# ---- prompt attention -------------------------------------------------------------------------------------------

def prompt_inputs(lens, nq, nkv, hd, seed, fused=True, std=1.0, slack=0):
    total = sum(lens) + slack
    g = gen(seed)
    if fused:
        rows = randn(g, total, nq + 2 * nkv, hd) * std
        q, k, v = rows[:, :nq], rows[:, nq:nq + nkv], rows[:, nq + nkv:]
    else:
        # head-major buffers with gaps between rows
        q = (randn(g, nq, total, hd + 8) * std)[:, :, :hd].permute(1, 0, 2)
        k = randn(g, nkv, total, 2 * hd)[:, :, hd:].permute(1, 0, 2)
        v = randn(g, total, nkv, hd)
    cu = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device=DEV)
    return q, k, v, cu


def check_prompt(q, k, v, lens, out, lse, scale, start=0, heads=None):
    at = start
    for n in lens:
        if n:
            s = slice(at, at + n)
            check(out[s], None if lse is None else lse[s], attention64(q[s], k[s], v[s], causal(n), scale), (at, n))
        at += n


@pytest.mark.parametrize("nq,nkv,hd", [(9, 3, 64), (32, 4, 64), (32, 8, 128), (4, 4, 64), (3, 3, 128), (2, 1, 128),
                                       (16, 1, 64), (10, 2, 128), (7, 1, 64), (13, 1, 128)])
@pytest.mark.parametrize("lens", [[1], [7], [128], [129], [0, 5, 0, 1, 64, 0], [300, 1, 2, 255, 257, 0]])
def test_prompt_attention_shapes(amk, nq, nkv, hd, lens):
    q, k, v, cu = prompt_inputs(lens, nq, nkv, hd, 11 * sum(lens) + nq + hd)
    lse = torch.full((sum(lens), nq), math.nan, device=DEV)
    out = amk.amk_prompt_attention(q, k, v, cu, lse=lse)
    check_prompt(q, k, v, lens, out, lse, hd ** -0.5)


@pytest.mark.parametrize("nq,nkv,hd,lens", [(8, 2, 64, [1500, 700]), (4, 1, 128, [2047, 1, 1030]), (6, 2, 128, [1111]),
                                            (2, 2, 64, [1300, 640]), (16, 2, 128, [520, 900])])
def test_prompt_attention_long(amk, nq, nkv, hd, lens):
    q, k, v, cu = prompt_inputs(lens, nq, nkv, hd, 5, fused=False, std=2.0)
    lse = torch.full((sum(lens), nq), math.nan, device=DEV)
    out = amk.amk_prompt_attention(q, k, v, cu, scale=0.11, lse=lse)
    check_prompt(q, k, v, lens, out, lse, float(np.float32(0.11)))


def test_prompt_attention_largest_context(amk):
    """A 20000-token prompt: some rows against 64 bits."""
    n, nq, nkv, hd = 20001, 4, 1, 128
    q, k, v, cu = prompt_inputs([n], nq, nkv, hd, 21)
    out = amk.amk_prompt_attention(q, k, v, cu)
    rows = torch.tensor([0, 1, 127, 128, 4095, 9999, 15000, 19999, 20000], device=DEV)
    sees = torch.arange(n, device=DEV)[None] <= rows[:, None]
    check(out[rows], None, attention64(q[rows], k, v, sees, hd ** -0.5))


def test_prompt_attention_large_scores_and_rising_maxima(amk):
    """Scores that grow along the keys by hundreds, so that every tile raises the running maximum, and fall again."""
    n, nq, nkv, hd = 700, 4, 2, 64
    q, k, v, cu = prompt_inputs([n], nq, nkv, hd, 3, fused=False)
    ramp = torch.linspace(0, 30, n, device=DEV)
    ramp[350:] = ramp[350:].flip(0) * 1.5
    q = torch.ones_like(q) + 0.01 * q
    k = (ramp[:, None, None] * torch.ones_like(k) + 0.1 * k).to(torch.bfloat16)
    lse = torch.empty(n, nq, device=DEV)
    out = amk.amk_prompt_attention(q, k, v, cu, lse=lse)
    check_prompt(q, k, v, [n], out, lse, hd ** -0.5)


def test_prompt_attention_leaves_other_rows_alone(amk):
    """Rows before the first prompt, behind the last one and of prompts with impossible bounds stay as they were; what
    the inputs hold there, NaN included, reaches nothing."""
    nq, nkv, hd, total = 4, 2, 64, 600
    g = gen(8)
    q, k, v = randn(g, total, nq, hd), randn(g, total, nkv, hd), randn(g, total, nkv, hd)
    for t in (q, k, v):
        t[:10] = math.nan
        t[300:] = math.inf
    cu = torch.tensor([10, 10, 150, 290, 300, 5, 900], dtype=torch.int32, device=DEV)   # 300..5 and 5..900: skipped
    out = torch.full((total, nq, hd), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((total, nq), 7.0, device=DEV)
    amk.amk_prompt_attention(q, k, v, cu, out=out, lse=lse)
    for a, b in ((10, 150), (150, 290), (290, 300)):
        check(out[a:b], lse[a:b], attention64(q[a:b], k[a:b], v[a:b], causal(b - a), hd ** -0.5), (a, b))
    assert bool((out[:10] == 7).all()) and bool((out[300:] == 7).all())
    assert bool((lse[:10] == 7).all()) and bool((lse[300:] == 7).all())


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["k", "v"])
def test_prompt_attention_hidden_values_reach_nothing(amk, value, where):
    """A token whose K or V row is not finite changes only the queries that attend to it."""
    n, nq, nkv, hd = 400, 4, 2, 128
    q, k, v, cu = prompt_inputs([n], nq, nkv, hd, 9, fused=False)
    q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    t = k if where == "k" else v
    t[200, 0, 3] = value
    t[333, 1, 77] = value
    out = amk.amk_prompt_attention(q, k, v, cu)
    ref = attention64(q, k, v, causal(n), hd ** -0.5)
    check(out, None, ref)
    assert int(ref[4].sum()) == 2 * (400 - 200) + 2 * (400 - 333)
    if where == "v":                                   # and those that do attend to it show it
        assert bool((~torch.isfinite(out[200:, :2, 3].float())).all()) and bool((~torch.isfinite(out[333:, 2:, 77].float())).all())
        assert bool(torch.isfinite(out[:, :2, 4].float()).all())
    elif value != value:
        assert bool(torch.isnan(out[200:, :2].float()).all()) and bool(torch.isnan(out[333:, 2:].float()).all())


def test_prompt_attention_many_short_prompts(amk):
    rng = np.random.default_rng(4)
    lens = [int(x) for x in rng.integers(0, 9, 700)]
    nq, nkv, hd = 6, 2, 64
    q, k, v, cu = prompt_inputs(lens, nq, nkv, hd, 14)
    out = amk.amk_prompt_attention(q, k, v, cu)
    at = np.repeat(np.arange(len(lens)), lens)
    seq = torch.from_numpy(at).to(DEV)
    sees = (seq[:, None] == seq[None]) & causal(sum(lens))
    check(out, None, attention64(q, k, v, sees, hd ** -0.5))


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_attention_thousands_of_prompts(amk, hd):
    """Prompts of 0 to 40 tokens and some of 300 to 600, several units for every block; some bounds are impossible and
    their prompts left out."""
    rng = np.random.default_rng(hd)
    lens = [int(x) for x in rng.integers(0, 41, 2500)]
    for at in rng.integers(0, 2500, 12):
        lens[at] = int(rng.integers(300, 601))
    q, k, v, cu = prompt_inputs(lens, 6, 2, hd, 77)
    total, ends = sum(lens), np.cumsum([0] + lens)
    out = torch.full((total, 6, hd), 3.0, dtype=torch.bfloat16, device=DEV)
    bad = sorted(int(x) for x in rng.choice(np.arange(1, 2499), 9, replace=False))
    for at in bad:
        cu[at] = total + 5 if at % 2 else -1            # the end of prompt at - 1, the beginning of prompt at
    amk.amk_prompt_attention(q, k, v, cu, out=out)
    skipped = {x for at in bad for x in (at - 1, at)}
    for s, n in enumerate(lens):
        a = int(ends[s])
        if s in skipped:
            assert bool((out[a:a + n] == 3).all()), s
        elif n and (n > 200 or s % 50 == 0):
            check_prompt(q, k, v, [n], out, None, hd ** -0.5, start=a)


@pytest.mark.parametrize("n_seqs", [31, 32, 33, 65])
def test_prompt_attention_around_32_prompts(amk, n_seqs):
    """Blocks are looked up in another way from 33 prompts on; with one head group of 16 a block is 16 tokens."""
    rng = np.random.default_rng(n_seqs)
    lens = [int(x) for x in rng.integers(0, 90, n_seqs)]
    lens[n_seqs // 2], lens[-1] = 700, 0
    q, k, v, cu = prompt_inputs(lens, 16, 1, 64, n_seqs)
    lse = torch.full((sum(lens), 16), math.nan, device=DEV)
    out = amk.amk_prompt_attention(q, k, v, cu, lse=lse)
    check_prompt(q, k, v, lens, out, lse, 0.125)


@pytest.mark.parametrize("nq,nkv,hd,n_seqs", [(8, 4, 64, 30), (16, 1, 128, 5000), (2, 2, 64, 20000)])
def test_prompt_attention_among_blocks_without_queries(amk, nq, nkv, hd, n_seqs):
    """The grid has a block for every prompt that could need one: here nearly all find none -- empty prompts, impossible
    bounds, far more prompts than tokens -- and only take over what is left."""
    rng = np.random.default_rng(n_seqs)
    lens = [0] * n_seqs
    for at, n in zip(rng.choice(n_seqs - 2, 6, replace=False), (1, 300, 2, 77, 1030, 20)):
        lens[int(at)] = n
    total = sum(lens)
    q, k, v, cu = prompt_inputs(lens, nq, nkv, hd, n_seqs, slack=400)
    cu[-1] = total + 900                               # impossible: the last prompt is left out
    out = torch.full((total + 400, nq, hd), 5.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((total + 400, nq), 5.0, device=DEV)
    for _ in range(3):
        amk.amk_prompt_attention(q, k, v, cu, out=out, lse=lse)
        check_prompt(q, k, v, lens, out, lse, hd ** -0.5)
        assert bool((out[total:] == 5).all()) and bool((lse[total:] == 5).all())
        out[:total], lse[:total] = 5.0, 5.0
    assert amk.amk_operator_status() == 0


def test_attention_a_broken_query_spoils_its_own_row_only(amk):
    nq, nkv, hd, n = 4, 2, 128, 300
    q, k, v, cu = prompt_inputs([n], nq, nkv, hd, 19, fused=False)
    q = q.contiguous()
    q[140, 1, 5], q[7, 3, 0] = math.nan, math.inf
    out = amk.amk_prompt_attention(q, k, v, cu).float()
    o, _, tol, _, _ = attention64(torch.nan_to_num(q, 0, 0, 0), k, v, causal(n), hd ** -0.5)
    fine = torch.ones(n, nq, dtype=torch.bool, device=DEV)
    fine[140, 1] = fine[7, 3] = False
    assert bool(((out.double() - o).abs() <= tol)[fine].all())
    assert bool(torch.isnan(out[140, 1]).all()) and not bool(torch.isfinite(out[7, 3]).any())


def test_attentions_on_two_streams_at_once(amk):
    """Calls that overlap, each with its own scratch, give what they give alone; what follows in a stream sees the result."""
    q, k, v, cu = prompt_inputs([900, 300], 8, 2, 64, 23)
    qt, kt, vt = tree_inputs(2, 9, 3000, 8, 2, 128, "bf16", 24)
    length = torch.tensor([2900, 1500], dtype=torch.int32, device=DEV)
    want_p, want_t = amk.amk_prompt_attention(q, k, v, cu), amk.amk_tree_attention(qt, kt, vt, length)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for i in range(30):
        with torch.cuda.stream(streams[i % 3]):
            if i % 2:
                got.append((want_p, amk.amk_prompt_attention(q, k, v, cu).clone()))
            else:
                got.append((want_t, amk.amk_tree_attention(qt, kt, vt, length).clone()))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in got)


@pytest.mark.parametrize("captured", [False, True])
def test_operators_wait_for_what_is_in_front_of_them(amk, captured):
    """The kernels may begin while the one before them ends: inputs that are written last thing before the call -- by a
    kernel, a memset, a copy, another stream, another operator -- and outputs that are overwritten right behind it."""
    n, nq, nkv, hd, slots, rows, vocab = 700, 8, 2, 128, 1500, 4, 50000
    q, k, v, cu = prompt_inputs([n - 200, 200], nq, nkv, hd, 5, fused=False)
    qt, kt, vt = tree_inputs(1, rows, slots, nq, nkv, hd, "bf16", 6)
    logits = torch.randn(rows, vocab, generator=gen(7), device=DEV)
    tokens = torch.tensor([1, 2, 3, 49999], dtype=torch.int32, device=DEV)
    one = lambda x: torch.tensor([x], dtype=torch.int32, device=DEV)
    base, keep, count = one(1400), torch.tensor([[1401, 1403, 1404]], dtype=torch.int32, device=DEV), one(3)
    src = [t.clone() for t in (q, k, v, qt, kt, vt, logits)]
    dst = [torch.zeros_like(t) for t in src]
    late = [torch.zeros_like(t) for t in (cu, tokens, count)]
    length = one(0)
    side = torch.cuda.Stream()
    big = torch.zeros(1 << 24, device=DEV)

    def steps():
        outs = []
        big.add_(1.0)                                          # a long kernel, and then the inputs at the last moment
        for d, s in zip(dst, src):
            d.copy_(s)
        late[0].copy_(cu)
        outs.append(amk.amk_prompt_attention(dst[0], dst[1], dst[2], late[0]))
        for d in dst[:3]:
            d.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            big.add_(1.0)
            length.fill_(1400)
        torch.cuda.current_stream().wait_stream(side)
        for _ in range(2):                                     # its own output is the next one's query
            outs.append(amk.amk_tree_attention(dst[3] if len(outs) == 1 else outs[-1], dst[4], dst[5], length))
        kv = torch.stack([dst[4][0], dst[5][0]])[None].contiguous()
        late[2].copy_(count)
        amk.amk_kv_compact(kv, base, keep, late[2])
        outs.append(amk.amk_tree_attention(dst[3], kv[:, 0], kv[:, 1], length))
        for d in dst[3:6]:
            d.zero_()
        length.zero_()
        late[1].copy_(tokens)
        outs += [x.clone() for x in amk.amk_token_logprobs(dst[6], late[1], 5)]
        dst[6].zero_()
        late[1].zero_()
        kv.zero_()
        return outs

    def alone():
        wait = torch.cuda.synchronize
        wait()
        outs = [amk.amk_prompt_attention(*src[:3], cu)]
        wait()
        at = one(1400)
        outs.append(amk.amk_tree_attention(src[3], src[4], src[5], at))
        wait()
        outs.append(amk.amk_tree_attention(outs[-1], src[4], src[5], at))
        kv = torch.stack([src[4][0], src[5][0]])[None].contiguous()
        wait()
        amk.amk_kv_compact(kv, base, keep, count)
        wait()
        outs.append(amk.amk_tree_attention(src[3], kv[:, 0], kv[:, 1], at))
        wait()
        outs += list(amk.amk_token_logprobs(src[6], tokens, 5))
        wait()
        return outs

    want = alone()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = steps()
    for _ in range(5):
        if captured:
            graph.replay()
        else:
            outs = steps()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("tiles", [0, 1, 2, 3])
@pytest.mark.parametrize("kind", ["prompt", "prompts", "tree run", "tree cluster", "tree block", "tree fp8", "tree rows"])
def test_attention_waits_run_out_and_the_next_call_is_fine(amk, kind, tiles):
    """A block that gets no more than some of its tiles: every wait for the next one ends, the status says so once, and what
    comes after is as ever."""
    hd = 64
    if kind.startswith("prompt"):
        q, k, v, cu = prompt_inputs([700] if kind == "prompt" else [300, 0, 5, 200, 129] * 20, 4, 2, hd, 3)
        call = lambda: amk.amk_prompt_attention(q, k, v, cu)
    else:
        rows, slots, nq, nkv, seqs = {"run": (9, 4000, 8, 2, 3), "cluster": (3, 2000, 4, 2, 1), "block": (20, 700, 8, 2, 50),
                                      "fp8": (5, 3000, 8, 2, 2), "rows": (100, 1500, 8, 2, 1)}[kind.split()[1]]
        q, k, v = tree_inputs(seqs, rows, slots, nq, nkv, hd, "fp8" if kind == "tree fp8" else "bf16", 4)
        length = torch.full((seqs,), slots - rows, dtype=torch.int32, device=DEV)
        call = lambda: amk.amk_tree_attention(q, k, v, length)
    want = call()
    assert amk.amk_operator_status() == amk.AMK_OK
    amk.amk_debug_operator_wait(2_000_000, tiles)      # about a millisecond
    try:
        call()
        assert amk.amk_operator_status() == amk.AMK_ERR_TIMEOUT
        assert amk.amk_operator_status() == amk.AMK_OK
    finally:
        amk.amk_debug_operator_wait()
    assert torch.equal(call(), want) and amk.amk_operator_status() == amk.AMK_OK
    with pytest.raises(amk.AmkError):
        amk.amk_debug_operator_wait(4_000_000_001)


def test_an_expired_wait_is_told_of_once_whichever_stream_asks(amk):
    """Two expiries on two streams, asked about in between: the second one is not lost."""
    q, k, v, cu = prompt_inputs([300], 4, 2, 64, 3)
    side = torch.cuda.Stream()
    amk.amk_operator_status()
    for stream in (torch.cuda.current_stream(), side, torch.cuda.current_stream()):
        amk.amk_debug_operator_wait(2_000_000, 0)
        try:
            with torch.cuda.stream(stream):
                amk.amk_prompt_attention(q, k, v, cu)
            torch.cuda.synchronize()
        finally:
            amk.amk_debug_operator_wait()
        amk.amk_prompt_attention(q, k, v, cu)
        assert amk.amk_operator_status() == amk.AMK_ERR_TIMEOUT
        with torch.cuda.stream(side):
            assert amk.amk_operator_status() == amk.AMK_OK


def test_first_call_of_a_process_may_be_captured():
    """Everything that a call sets up once happens in the call itself, and capture allows it."""
    code = """
import torch
from paper_2606_09682_b200 import binding as amk
q = torch.randn(1, 3, 4, 64, device="cuda").to(torch.bfloat16)
k = torch.randn(1, 2, 500, 64, device="cuda").to(torch.bfloat16)
x, tok = torch.randn(2, 5000, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
n, cu = torch.full((1,), 400, dtype=torch.int32, device="cuda"), torch.tensor([0, 3], dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    a = amk.amk_tree_attention(q, k, k, n)
    b = amk.amk_prompt_attention(q[0], q[0, :, :2], q[0, :, 2:], cu)
    c = amk.amk_token_logprobs(x, tok, 3)
    amk.amk_kv_compact(k, n, n[None], n)
graph.replay()
assert torch.equal(a, amk.amk_tree_attention(q, k, k, n)) and torch.equal(b, amk.amk_prompt_attention(q[0], q[0, :, :2], q[0, :, 2:], cu))
assert all(torch.equal(u, v) for u, v in zip(c, amk.amk_token_logprobs(x, tok, 3))) and amk.amk_operator_status() == 0
print("fine")
"""
    import os
    import subprocess
    import sys
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]


def test_prompt_attention_is_deterministic_and_replays(amk):
    """The same bits every time, on another stream, and from a captured graph whose inputs and bounds change."""
    lens, nq, nkv, hd = [333, 100, 267], 8, 2, 128
    q, k, v, cu = prompt_inputs(lens, nq, nkv, hd, 6)
    a = amk.amk_prompt_attention(q, k, v, cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = amk.amk_prompt_attention(q, k, v, cu)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, b)
    out = torch.empty_like(a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        amk.amk_prompt_attention(q, k, v, cu, out=out)
    graph.replay()
    assert torch.equal(a, out)
    q2, k2, v2, _ = prompt_inputs(lens, nq, nkv, hd, 7)
    q.copy_(q2), k.copy_(k2), v.copy_(v2)
    lens2 = [20, 600, 80]
    cu.copy_(torch.tensor([0, 20, 620, 700], dtype=torch.int32))
    graph.replay()
    check_prompt(q, k, v, lens2, out, None, hd ** -0.5)


# ---- tree attention ---------------------------------------------------------------------------------------------

def tree_bits(rng, rows):
    """[rows][rows] of a random tree: a token sees its ancestors and itself."""
    sees = np.zeros((rows, rows), dtype=bool)
    for i in range(rows):
        parent = int(rng.integers(-1, i)) if i else -1
        if parent >= 0:
            sees[i] = sees[parent]
        sees[i, i] = True
    return sees


def words(sees):
    """bool [seqs][rows][rows] -> int64 words."""
    seqs, rows, _ = sees.shape
    w = np.zeros((seqs, rows, (rows + 63) // 64), dtype=np.uint64)
    for j in range(rows):
        w[:, :, j // 64] |= sees[:, :, j].astype(np.uint64) << np.uint64(j % 64)
    return torch.from_numpy(w.view(np.int64)).to(DEV)


def tree_inputs(seqs, rows, slots, nq, nkv, hd, cache, seed):
    g = gen(seed)
    q = randn(g, seqs, rows, nq, hd)
    kv = randn(g, 2, seqs, nkv, slots, hd, dtype=torch.float32)
    kv = kv.to(torch.float8_e4m3fn).view(torch.uint8) if cache == "fp8" else kv.to(torch.bfloat16)
    return q, kv[0], kv[1]


def check_tree(q, k, v, lens, bits, out, lse, scale, what=""):
    rows = q.shape[1]
    for b, n in enumerate(lens):
        sees = torch.ones(rows, n + rows, dtype=torch.bool)
        sees[:, n:] = torch.from_numpy(bits[b])
        kk, vv = k[b, :, :n + rows], v[b, :, :n + rows]
        if kk.dtype == torch.uint8:
            kk, vv = kk.view(torch.float8_e4m3fn).float(), vv.view(torch.float8_e4m3fn).float()
        check(out[b], None if lse is None else lse[b],
              attention64(q[b], kk.permute(1, 0, 2), vv.permute(1, 0, 2), sees.to(DEV), scale), (what, b, n))


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("nq,nkv,hd", [(9, 3, 64), (32, 4, 64), (32, 8, 128), (3, 3, 128), (16, 1, 64), (7, 1, 128)])
@pytest.mark.parametrize("rows,slots,lens", [(1, 1, [0]), (1, 300, [0, 299, 128, 5]), (5, 200, [195, 0, 60]),
                                             (26, 700, [600, 102]), (64, 400, [0, 64, 333]), (65, 900, [800, 1])])
def test_tree_attention_shapes(amk, cache, nq, nkv, hd, rows, slots, lens):
    rng = np.random.default_rng(rows * 1000 + slots)
    q, k, v = tree_inputs(len(lens), rows, slots, nq, nkv, hd, cache, rows + nq)
    bits = np.stack([tree_bits(rng, rows) for _ in lens])
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)
    lse = torch.empty(len(lens), rows, nq, device=DEV)
    out = amk.amk_tree_attention(q, k, v, length, words(bits), lse=lse)
    check_tree(q, k, v, lens, bits, out, lse, hd ** -0.5)
    chain = np.stack([np.tril(np.ones((rows, rows), dtype=bool))] * len(lens))
    out = amk.amk_tree_attention(q, k, v, length, lse=lse)
    check_tree(q, k, v, lens, chain, out, lse, hd ** -0.5, "chain")


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("seqs,rows,slots,nq,nkv,hd", [(1, 1, 8192, 32, 8, 128), (1, 1, 20000, 32, 4, 64),
                                                       (3, 16, 5000, 8, 2, 128), (2, 200, 3000, 8, 2, 64),
                                                       (1, 1000, 2500, 4, 1, 128), (40, 2, 900, 4, 4, 64)])
def test_tree_attention_long_caches(amk, cache, seqs, rows, slots, nq, nkv, hd):
    rng = np.random.default_rng(slots)
    q, k, v = tree_inputs(seqs, rows, slots, nq, nkv, hd, cache, slots)
    lens = [int(x) for x in rng.integers(0, slots - rows + 1, seqs)]
    lens[0] = slots - rows
    bits = np.stack([tree_bits(rng, rows) for _ in lens])
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for hint in (None, 17):                            # the bound is a hint: a wrong one changes no result's meaning
        lse = torch.empty(seqs, rows, nq, device=DEV)
        out = amk.amk_tree_attention(q, k, v, length, words(bits), max_len=hint, scale=0.2, lse=lse)
        check_tree(q, k, v, lens, bits, out, lse, float(np.float32(0.2)), hint)


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("len_", [0, 70, 1000])
def test_tree_attention_rows_that_see_nothing(amk, cache, len_):
    """A mask row of zeros: with no context the output is zero and the log-sum-exp -inf, with one it is the context's."""
    rows, nq, nkv, hd = 9, 4, 2, 64
    q, k, v = tree_inputs(1, rows, 1100, nq, nkv, hd, cache, 2)
    bits = np.stack([tree_bits(np.random.default_rng(1), rows)])
    bits[0, 4] = bits[0, 8] = bits[0, 0] = False
    lse = torch.empty(1, rows, nq, device=DEV)
    out = amk.amk_tree_attention(q, k, v, torch.tensor([len_], dtype=torch.int32, device=DEV), words(bits), lse=lse)
    check_tree(q, k, v, [len_], bits, out, lse, hd ** -0.5)
    if not len_:
        assert bool((out[0, [0, 4, 8]] == 0).all()) and bool((lse[0, [0, 4, 8]] == -math.inf).all())


@pytest.mark.parametrize("rows", [1, 5, 31, 33, 64, 70, 127])
def test_tree_attention_ignores_bits_behind_the_last_token(amk, rows):
    nq, nkv, hd, slots = 8, 2, 64, 700
    q, k, v = tree_inputs(1, rows, slots, nq, nkv, hd, "bf16", rows)
    bits = np.stack([tree_bits(np.random.default_rng(rows), rows)])
    mask = words(bits)
    if rows % 64:
        mask[:, :, -1] |= -1 << (rows % 64)
    for n in (0, 100, slots - rows):
        out = amk.amk_tree_attention(q, k, v, torch.tensor([n], dtype=torch.int32, device=DEV), mask)
        check_tree(q, k, v, [n], bits, out, None, hd ** -0.5)


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_tree_attention_largest_draft(amk, cache):
    """1024 drafted tokens of 16 heads to one: 64 blocks of rows."""
    rows, nq, nkv, hd, slots = 1024, 16, 1, 64, 1500
    q, k, v = tree_inputs(1, rows, slots, nq, nkv, hd, cache, 61)
    bits = np.stack([tree_bits(np.random.default_rng(8), rows)])
    lse = torch.empty(1, rows, nq, device=DEV)
    out = amk.amk_tree_attention(q, k, v, torch.tensor([476], dtype=torch.int32, device=DEV), words(bits), lse=lse)
    check_tree(q, k, v, [476], bits, out, lse, hd ** -0.5)


def test_tree_attention_many_sequences(amk):
    """300 sequences, empty ones and bad lengths among them."""
    seqs, rows, nq, nkv, hd, slots = 300, 3, 6, 3, 64, 260
    q, k, v = tree_inputs(seqs, rows, slots, nq, nkv, hd, "bf16", 62)
    rng = np.random.default_rng(2)
    lens = [int(x) for x in rng.integers(0, slots - rows + 1, seqs)]
    lens[7] = lens[299] = -3
    lens[100], lens[0] = slots, 0
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out = amk.amk_tree_attention(q, k, v, length)
    chain = np.tril(np.ones((rows, rows), dtype=bool))
    for b in range(seqs):
        if 0 <= lens[b] <= slots - rows:
            check_tree(q[b:b + 1], k[b:b + 1], v[b:b + 1], [lens[b]], chain[None], out[b:b + 1], None, hd ** -0.5, b)
        else:
            assert bool(torch.isnan(out[b].float()).all())


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("nq,nkv,hd,rows,slots", [(4, 2, 64, 3, 2048), (2, 1, 128, 7, 2000), (8, 4, 128, 8, 1000), (9, 3, 64, 5, 500),
                                                  (16, 8, 64, 16, 260), (32, 2, 64, 8, 256), (3, 1, 128, 1, 128)])
def test_tree_attention_short_calls(amk, cache, nq, nkv, hd, rows, slots):
    """Calls whose blocks join their parts in one launch: lengths that leave some or most of an item's blocks without a
    tile, a length that breaks max_len, one that is impossible."""
    q, k, v = tree_inputs(1, rows, slots, nq, nkv, hd, cache, slots + rows)
    bits = tree_bits(np.random.default_rng(rows), rows)[None]
    bits[0, rows // 2] = rows == 1
    most = slots - rows
    for n in sorted({0, 1, 127 - rows, 128 - rows, 129 - rows, 200, 3 * 128, most // 2, most - 1, most}):
        if not 0 <= n <= most:
            continue
        length = torch.tensor([n], dtype=torch.int32, device=DEV)
        for hint in (None, 100):
            lse = torch.full((1, rows, nq), math.nan, device=DEV)
            out = amk.amk_tree_attention(q, k, v, length, words(bits), max_len=hint and min(hint, slots), lse=lse)
            check_tree(q, k, v, [n], bits, out, lse, hd ** -0.5, n)
    lse = torch.zeros(1, rows, nq, device=DEV)
    out = amk.amk_tree_attention(q, k, v, torch.tensor([most + 1], dtype=torch.int32, device=DEV), words(bits), lse=lse)
    assert bool(torch.isnan(out.float()).all()) and bool(torch.isnan(lse).all())


@pytest.mark.parametrize("nq,nkv,hd", [(4096, 4096, 128), (4096, 256, 64)])
def test_attentions_of_the_most_heads(amk, nq, nkv, hd):
    rows, slots, lens = 2, 150, [131]
    q, k, v = tree_inputs(1, rows, slots, nq, nkv, hd, "bf16", 17)
    lse = torch.full((1, rows, nq), math.nan, device=DEV)
    out = amk.amk_tree_attention(q, k, v, torch.tensor(lens, dtype=torch.int32, device=DEV), lse=lse)
    check_tree(q, k, v, lens, np.tril(np.ones((1, rows, rows), bool)), out, lse, hd ** -0.5)
    q, k, v, cu = prompt_inputs([3, 131], nq, nkv, hd, 18)
    out = amk.amk_prompt_attention(q, k, v, cu)
    check_prompt(q, k, v, [3, 131], out, None, hd ** -0.5)


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_tree_attention_hidden_values_reach_nothing(amk, cache):
    """NaN in slots behind the drafted tokens reaches nothing; in a drafted token's K or V it reaches that token's
    descendants only."""
    rows, nq, nkv, hd, slots, lens = 20, 8, 2, 128, 600, [300, 250]
    q, k, v = tree_inputs(2, rows, slots, nq, nkv, hd, cache, 12)
    bits = np.stack([tree_bits(np.random.default_rng(s), rows) for s in (5, 6)])
    nan = 0x7F if cache == "fp8" else math.nan
    for b, n in enumerate(lens):
        k[b, :, n + rows:] = nan
        v[b, :, n + rows:] = nan
    k[0, 0, 300 + 7, 5] = nan
    v[0, 1, 300 + 3, 9] = nan
    v[1, 0, 250 + 11, :] = nan
    out = amk.amk_tree_attention(q, k, v, torch.tensor(lens, dtype=torch.int32, device=DEV), words(bits))
    check_tree(q, k, v, lens, bits, out, None, hd ** -0.5)
    o = out.float()
    for b, g, j in ((0, 0, 7), (0, 1, 3), (1, 0, 11)):
        sees = torch.from_numpy(bits[b][:, j]).to(DEV)
        heads = o[b][:, g * 4:(g + 1) * 4]
        assert bool(torch.isnan(heads[sees]).flatten(1).any(1).all()) and bool(torch.isfinite(heads[~sees]).all()), (b, g, j)


@pytest.mark.parametrize("hd", [64, 128])
def test_tree_attention_every_8bit_code(amk, hd):
    """Uniformly drawn codes, all 254 numbers among them (subnormals, both zeros, +-448); and one key alone, whose V row
    has to come out as it is."""
    g = gen(hd)
    codes = torch.randint(0, 256, (2, 1, 2, 700, hd), generator=g, device=DEV).to(torch.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x7E
    assert len(codes.unique()) == 254
    q = randn(g, 1, 5, 4, hd)
    bits = np.stack([tree_bits(np.random.default_rng(3), 5)])
    lse = torch.empty(1, 5, 4, device=DEV)
    out = amk.amk_tree_attention(q, codes[0], codes[1], torch.tensor([690], dtype=torch.int32, device=DEV), words(bits),
                                 scale=2.0 ** -12, lse=lse)
    check_tree(q, codes[0], codes[1], [690], bits, out, lse, 2.0 ** -12)
    for start in range(0, 700, 71):
        k, v = codes[0][:, :, start:start + 1], codes[1][:, :, start:start + 1]
        out = amk.amk_tree_attention(q[:, :1], k.contiguous(), v.contiguous(), torch.zeros(1, dtype=torch.int32, device=DEV))
        want = v.view(torch.float8_e4m3fn).to(torch.bfloat16)[0, :, 0].repeat_interleave(2, 0)
        assert torch.equal(out[0, 0], want)


@pytest.mark.parametrize("slots,rows,nq,nkv,hd", [(300, 9, 4, 2, 64), (8192, 9, 8, 2, 128), (8192, 9, 16, 1, 64), (3000, 36, 16, 2, 128)])
@pytest.mark.parametrize("place", ["first", "middle", "last"])
def test_tree_attention_small_numerators_over_the_8bit_cache(amk, slots, rows, nq, nkv, hd, place):
    """One dominating key whose V is zero, and all others 2^-10 to 2^-30 below it: the output is theirs alone.  Each numerator
    is off by 2^-11 of itself or 2^-34 of the row's largest one, whichever is more (half of f16's last place, 2^-25, where the
    largest is at least 2^9), beside the other terms of every case."""
    g = gen(slots + rows)
    n = slots - rows
    at = {"first": 0, "middle": n // 2, "last": n - 1}[place]
    k = torch.zeros(1, nkv, slots, hd, device=DEV)
    k[:, :, at, 0] = 1.0
    v = torch.randn(1, nkv, slots, hd, generator=g, device=DEV).abs()
    v[:, :, at] = 0.0
    k, v = (t.to(torch.float8_e4m3fn).view(torch.uint8) for t in (k, v))
    gaps = torch.tensor([10.0, 13.0, 16.0, 18.0, 20.0, 22.0, 24.0, 27.0, 30.0], device=DEV)[torch.arange(rows, device=DEV) % 9]
    q = torch.zeros(1, rows, nq, hd, device=DEV)
    q[..., 0] = (gaps * math.log(2) * hd ** 0.5)[:, None]
    q = q.to(torch.bfloat16)
    lse = torch.empty(1, rows, nq, device=DEV)
    out = amk.amk_tree_attention(q, k, v, torch.tensor([n], dtype=torch.int32, device=DEV), lse=lse)
    sees = torch.ones(rows, slots, dtype=torch.bool, device=DEV)
    sees[:, n:] = causal(rows)
    vv = v[0].view(torch.float8_e4m3fn).float()
    o, l, tol, tol_l, touched = attention64(q[0], k[0].view(torch.float8_e4m3fn).float().permute(1, 0, 2), vv.permute(1, 0, 2), sees, hd ** -0.5)
    tol = tol + 2.0 ** -34 * vv.double().sum(1).repeat_interleave(nq // nkv, 0)[None]
    check(out[0], lse[0], (o, l, tol, tol_l, touched), place)


def check_exact_scores(q, k, v, sees, out, lse, scale, what=""):
    """As check(attention64(..)) where fp32 holds every score without rounding (E = 0): q [t][nq][hd], k / v [n][nkv][hd]."""
    rep, n = q.shape[1] // k.shape[1], k.shape[0]
    qd, kd, vd = (t.double().permute(1, 0, 2) for t in (q, k, v))
    x = (qd @ kd.repeat_interleave(rep, 0).transpose(1, 2) * scale).masked_fill(~sees[None], -math.inf)
    l, p = torch.logsumexp(x, 2), torch.softmax(x, 2)  # (softmax: exp(x - l) would lose the log 2 of two equal scores of 1e17)
    o, A = p @ vd.repeat_interleave(rep, 0), p @ vd.abs().repeat_interleave(rep, 0)
    tol = ((2.0 ** -8 + 2.0 ** -10) * A + 2.0 ** -8 * o.abs() + 1e-30).permute(1, 0, 2)
    tol_l = (n * 2.0 ** -24 + 2.0 ** -20 * (1 + l.abs())).permute(1, 0)
    err, err_l = (out.double() - o.permute(1, 0, 2)).abs(), (lse.double() - l.permute(1, 0)).abs()
    assert bool((err <= tol).all()), (what, float((err / tol).max()))
    assert bool((err_l <= tol_l).all()), (what, float((err_l / tol_l).max()))


def distinct_bf16(n, seed):
    """n distinct positive bf16 values from 1 up, in an order drawn from the seed: neighbours are 2^-7 of themselves apart."""
    order = torch.randperm(n, generator=gen(seed), device=DEV)
    return (order.to(torch.int32) + 0x3F80).to(torch.int16).view(torch.bfloat16)


@pytest.mark.parametrize("power", [8, 20, 40, 90])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("sign", [1, -1])
def test_prompt_attention_scores_beyond_the_integers(amk, power, hd, sign):
    """Scores so large that the product of the maximum with scale log2 e is off by more than an exponential can take: one key
    has all the weight (of equal ones each the same).  All scores are exact in fp32 here: powers of two times bf16 values."""
    n, nq, nkv = 900, 4, 2
    _, _, v, cu = prompt_inputs([n - 1, 1], nq, nkv, hd, power, fused=False)
    q = torch.full((n, nq, hd), 2.0 ** power * sign, device=DEV).to(torch.bfloat16)
    k = distinct_bf16(300, power).repeat(3)[:, None, None].expand(n, nkv, hd).contiguous()
    k[450:460] *= 16                                    # a key far above the others in the middle
    scale = 2.0 ** 12 if power < 90 else 1.0
    lse = torch.empty(n, nq, device=DEV)
    out = amk.amk_prompt_attention(q, k, v, cu, scale=scale, lse=lse)
    for s in (slice(0, n - 1), slice(n - 1, n)):
        check_exact_scores(q[s], k[s], v[s], causal(s.stop - s.start), out[s], lse[s], scale)
    assert torch.equal(out[0], v[0].repeat_interleave(2, 0))


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("power", [8, 20, 40, 90])
@pytest.mark.parametrize("rows,slots,nq,nkv,hd", [(3, 700, 4, 2, 64), (5, 1900, 8, 1, 128), (40, 700, 8, 1, 64), (1, 120, 2, 2, 128)])
def test_tree_attention_scores_beyond_the_integers(amk, cache, power, rows, slots, nq, nkv, hd):
    """As for prompts; every key has another value, so that one key has all the weight whichever parts the keys come in."""
    q, _, v = tree_inputs(1, rows, slots, nq, nkv, hd, cache, power)
    n = slots - rows
    q = torch.full_like(q, 2.0 ** power)
    if cache == "fp8":                                  # 126 positive codes (or as many as fit); below them the same negative one
        k = torch.full((slots,), 0xB8, device=DEV, dtype=torch.uint8)
        at = torch.randperm(slots, generator=gen(9), device=DEV)[:126]
        k[at] = torch.arange(127 - len(at), 127, device=DEV).to(torch.uint8)
        k[0] = k[n // 2]
        k[n // 2] = 0x7E
    else:
        k = distinct_bf16(slots, power)
    k = k[None, None, :, None].expand(1, nkv, slots, hd).contiguous()
    scale = 2.0 ** 14 if power < 90 else 1.0
    lse = torch.empty(1, rows, nq, device=DEV)
    out = amk.amk_tree_attention(q, k, v, torch.tensor([n], dtype=torch.int32, device=DEV), scale=scale, lse=lse)
    value = (lambda t: t[0].view(torch.float8_e4m3fn).float().permute(1, 0, 2)) if cache == "fp8" else (lambda t: t[0].permute(1, 0, 2))
    sees = torch.ones(rows, slots, dtype=torch.bool, device=DEV)
    sees[:, n:] = causal(rows)
    check_exact_scores(q[0], value(k), value(v), sees, out[0], lse[0], scale)


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("power", [6, 10, 16, 24, 60])
@pytest.mark.parametrize("seqs,rows,slots,nq,nkv,hd", [(1, 3, 1500, 4, 2, 64), (1, 2, 9001, 8, 1, 128), (3, 40, 5000, 8, 1, 64),
                                                       (1, 1, 6000, 32, 8, 128)])
def test_tree_attention_equal_scores_in_parts(amk, cache, power, seqs, rows, slots, nq, nkv, hd):
    """One large score for all keys: each weighs the same, in whichever part it comes and however many keys the part has."""
    q, _, v = tree_inputs(seqs, rows, slots, nq, nkv, hd, cache, power)
    v = v & 0x7F if cache == "fp8" else v.abs()
    lens = [slots - rows, 777, 130][:seqs]
    q = torch.full_like(q, 1.375 * 2.0 ** power)
    k = torch.full((seqs, nkv, slots, hd), 1.5, device=DEV)
    k = k.to(torch.float8_e4m3fn).view(torch.uint8) if cache == "fp8" else k.to(torch.bfloat16)
    lse = torch.empty(seqs, rows, nq, device=DEV)
    out = amk.amk_tree_attention(q, k, v, torch.tensor(lens, dtype=torch.int32, device=DEV), scale=0.125, lse=lse)
    value = (lambda t: t.view(torch.float8_e4m3fn).float().permute(1, 0, 2)) if cache == "fp8" else (lambda t: t.permute(1, 0, 2))
    for b, n in enumerate(lens):
        sees = torch.ones(rows, n + rows, dtype=torch.bool, device=DEV)
        sees[:, n:] = causal(rows)
        check_exact_scores(q[b], value(k[b, :, :n + rows]), value(v[b, :, :n + rows]), sees, out[b], lse[b], 0.125, b)


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("scale", [1e-12, 1e-30, 1e-44])
@pytest.mark.parametrize("rows,slots,nq,nkv,hd", [(5, 300, 4, 2, 64), (70, 900, 8, 2, 128)])
def test_tree_attention_vanishing_scores(amk, cache, scale, rows, slots, nq, nkv, hd):
    """Queries near the smallest numbers and a scale that all but vanishes: every key that is seen weighs the same."""
    q, k, v = tree_inputs(1, rows, slots, nq, nkv, hd, cache, 5)
    q = q * 1e-37
    bits = np.stack([tree_bits(np.random.default_rng(3), rows)])
    n = slots - rows
    lse = torch.empty(1, rows, nq, device=DEV)
    out = amk.amk_tree_attention(q, k, v, torch.tensor([n], dtype=torch.int32, device=DEV), words(bits), scale=scale, lse=lse)
    check_tree(q, k, v, [n], bits, out, lse, scale)


def test_tree_attention_bad_lengths(amk):
    rows, nq, nkv, hd, slots = 4, 4, 2, 64, 100
    q, k, v = tree_inputs(4, rows, slots, nq, nkv, hd, "bf16", 3)
    lens = [50, -1, 97, 96]
    lse = torch.empty(4, rows, nq, device=DEV)
    out = amk.amk_tree_attention(q, k, v, torch.tensor(lens, dtype=torch.int32, device=DEV), lse=lse)
    chain = np.tril(np.ones((rows, rows), dtype=bool))
    for b in (0, 3):
        check_tree(q[b:b + 1], k[b:b + 1], v[b:b + 1], [lens[b]], chain[None], out[b:b + 1], lse[b:b + 1], hd ** -0.5)
    assert bool(torch.isnan(out[1:3].float()).all()) and bool(torch.isnan(lse[1:3]).all())


def test_tree_attention_strides_out_and_workspace(amk):
    """Caches as slices of decoders' buffers, q and out with gaps, a workspace of the caller's with guard bytes, rows of
    a larger out left alone."""
    seqs, rows, nq, nkv, hd, slots, layers = 2, 6, 6, 3, 64, 1300, 3
    g = gen(31)
    caches = randn(g, seqs, 2, layers, nkv, slots, hd)
    k, v = caches[:, 0, 1], caches[:, 1, 1]
    q = randn(g, rows, seqs, nq, hd + 16)[..., :hd].permute(1, 0, 2, 3)
    lens = [1201, 700]
    bits = np.stack([tree_bits(np.random.default_rng(2), rows)] * seqs)
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)
    whole = torch.full((seqs, rows + 2, nq, hd + 8), 5.0, dtype=torch.bfloat16, device=DEV)
    out = whole[:, 1:-1, :, :hd]
    buf = torch.full((1 << 24,), 0x5A, dtype=torch.uint8, device=DEV)
    ws = buf[256:-256]
    amk.amk_tree_attention(q, k, v, length, words(bits), out=out, workspace=ws)
    check_tree(q, k, v, lens, bits, out, None, hd ** -0.5)
    assert bool((buf[:256] == 0x5A).all()) and bool((buf[-256:] == 0x5A).all())
    assert bool((whole[:, 0] == 5).all()) and bool((whole[:, -1] == 5).all()) and bool((whole[..., hd:] == 5).all())


def test_tree_attention_replays_with_new_lengths(amk):
    """Captured once, the call follows cache_len, the mask and the inputs; two graphs and an eager call in a row, each with
    its own scratch, give what they give alone."""
    seqs, rows, nq, nkv, hd, slots = 2, 8, 8, 2, 128, 4000
    q, k, v = tree_inputs(seqs, rows, slots, nq, nkv, hd, "bf16", 41)
    rng = np.random.default_rng(9)
    bits = np.stack([tree_bits(rng, rows) for _ in range(seqs)])
    mask, length = words(bits), torch.tensor([100, 3500], dtype=torch.int32, device=DEV)
    amk.amk_tree_attention(q, k, v, length, mask)
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(amk.amk_tree_attention(q, k, v, length, mask))
        graphs.append(graph)
    for lens in ([100, 3500], [3992, 0], [1, 2]):
        bits = np.stack([tree_bits(rng, rows) for _ in range(seqs)])
        mask.copy_(words(bits))
        length.copy_(torch.tensor(lens, dtype=torch.int32))
        graphs[0].replay()
        eager = amk.amk_tree_attention(q, k, v, length, mask)
        graphs[1].replay()
        check_tree(q, k, v, lens, bits, outs[0], None, hd ** -0.5)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], eager)


def test_tree_attention_row_offsets_beyond_32_bits(amk):
    """The last kv heads of a cache of more than 2^32 bytes."""
    seqs, rows, nq, nkv, hd, slots = 1, 3, 36, 36, 128, 500000
    kv = torch.zeros(seqs, nkv, slots, hd, dtype=torch.bfloat16, device=DEV)
    assert kv.numel() * 2 > 1 << 32
    g = gen(77)
    n = slots - rows
    kv[0, 0, -600:] = randn(g, 600, hd)
    kv[0, -1, -600:] = randn(g, 600, hd)
    q = randn(g, seqs, rows, nq, hd)
    out = amk.amk_tree_attention(q, kv, kv, torch.tensor([n], dtype=torch.int32, device=DEV))
    chain = torch.ones(rows, slots, dtype=torch.bool, device=DEV)
    chain[:, n:] = causal(rows)
    for h in (0, nkv - 1):
        kk = kv[0, h:h + 1].permute(1, 0, 2)
        check(out[0, :, h:h + 1], None, attention64(q[0, :, h:h + 1], kk, kk, chain, hd ** -0.5), h)


# ---- log probabilities ------------------------------------------------------------------------------------------

def logprobs64(x, tokens, top):
    lp = torch.log_softmax(x.double(), 1)
    ok = (tokens >= 0) & (tokens < x.shape[1])
    got = torch.where(ok, lp.gather(1, tokens.clamp(0, x.shape[1] - 1).long()[:, None])[:, 0], math.nan)
    p = lp.exp()
    ent = -torch.where(p > 0, p * lp, torch.where(torch.isnan(lp), lp, 0.0)).sum(1)
    ids = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :top]
    return got, ent, ids, lp.gather(1, ids)


def close(a, b, magnitude, n):
    """fp32 results off by at most: a few roundings of numbers as large as `magnitude` (2^-22 of it), exponentials good to
    2^-21 and sums of n positive terms in at least 64 partial sums (n 2^-30) inside a logarithm."""
    tol = 2.0 ** -22 * magnitude + 2.0 ** -21 + n * 2.0 ** -30
    same = (a.double() == b) | (torch.isnan(a) & torch.isnan(b)) | ((a.double() - b).abs() <= tol)
    assert bool(same.all()), float((a.double() - b).abs().nan_to_num(0).max() / tol)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (2, 31), (1, 1000), (5, 1003), (1, 32000), (7, 49152), (64, 128256),
                                        (400, 5000), (1, 300001), (1000, 33)])
@pytest.mark.parametrize("top", [0, 1, 20, 32])
def test_logprobs_shapes(amk, dtype, rows, vocab, top):
    g = gen(rows + vocab)
    x = (randn(g, rows, vocab, dtype=torch.float32) * 3).to(dtype)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device=DEV).to(torch.int32)
    lp, ent, ids, tlp = amk.amk_token_logprobs(x, tokens, top)
    want = logprobs64(x, tokens, top)
    n = min(top, vocab)
    mag = float(x.float().abs().max()) * 2 + 13
    close(lp, want[0], mag, vocab)
    close(ent, want[1], mag, vocab)
    assert torch.equal(ids[:, :n].long(), want[2])
    close(tlp[:, :n], want[3], mag, vocab)
    assert bool((ids[:, n:] == -1).all()) and bool(torch.isnan(tlp[:, n:]).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["rising", "falling", "equal", "two values", "one peak", "far apart", "spread", "edges"])
@pytest.mark.parametrize("vocab", [5003, 131072])
def test_logprobs_orders_and_ties(amk, dtype, kind, vocab):
    """Orders that renew the maximum or the alternatives at every element, ties, peaks and a wide range."""
    i = torch.arange(vocab, device=DEV, dtype=torch.float32)
    x = {"rising": i / 64, "falling": -i / 64, "equal": torch.full_like(i, 2.5), "two values": (i % 7 == 3).float(),
         "one peak": torch.where(i == vocab - 2, 50.0, 0.0), "far apart": torch.where(i % 97 == 0, 30000.0, -30000.0),
         "spread": (i * 7919 % vocab) / vocab * 200 - 100, "edges": torch.where((i == 0) | (i == vocab - 1), 9.0, -i / vocab)}[kind]
    x = torch.stack([x, x.flip(0)]).to(dtype)
    tokens = torch.tensor([vocab - 2, 0], dtype=torch.int32, device=DEV)
    lp, ent, ids, tlp = amk.amk_token_logprobs(x, tokens, 32)
    want = logprobs64(x, tokens, 32)
    mag = float(x.float().abs().max()) * 2 + 13
    close(lp, want[0], mag, vocab)
    close(ent, want[1], mag, vocab)
    assert torch.equal(ids.long(), want[2])
    close(tlp, want[3], mag, vocab)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [40, 9000, 128256])
def test_logprobs_special_values(amk, dtype, vocab):
    """Masked logits (-inf), nothing but masked ones, a +inf, NaN, tokens out of range; a strided, misaligned matrix."""
    g = gen(vocab)
    whole = randn(g, 8, vocab + 5, dtype=dtype)
    x = whole[:, 3:3 + vocab]
    x[1, 4:] = -math.inf
    x[2] = -math.inf
    x[3, vocab // 2] = math.inf
    x[4, vocab - 1] = math.nan
    x[7] = torch.finfo(dtype).min
    x[7, 5] = 0
    tokens = torch.tensor([2, 3, 0, 1, 0, -1, vocab, 6], dtype=torch.int32, device=DEV)
    lp, ent, ids, tlp = amk.amk_token_logprobs(x, tokens, 8)
    want = logprobs64(x, tokens, 8)
    close(lp[:2], want[0][:2], 40.0, vocab)
    close(ent[:2], want[1][:2], 40.0, vocab)
    close(tlp[:2], want[3][:2], 40.0, vocab)
    assert torch.equal(ids[:2].long(), want[2][:2])
    assert ids[2].tolist() == list(range(8))
    assert int(ids[3, 0]) == vocab // 2
    y = x[4].float().nan_to_num(-math.inf)
    assert torch.equal(ids[4].long(), torch.sort(y, descending=True, stable=True).indices[:8]) and vocab - 1 not in ids[4].tolist()
    for r in (2, 3, 4):
        assert math.isnan(lp[r]) and math.isnan(ent[r]) and bool(torch.isnan(tlp[r]).all())
    for r in (5, 6):
        assert math.isnan(lp[r]) and math.isfinite(ent[r]) and bool(torch.isfinite(tlp[r]).all())
    assert float(ent[7]) == 0.0 and float(tlp[7, 0]) == 0.0 and ids[7].tolist() == [5, 0, 1, 2, 3, 4, 6, 7]
    x = torch.full((1, vocab), math.nan, dtype=dtype, device=DEV)
    lp, ent, ids, tlp = amk.amk_token_logprobs(x, tokens[:1], 3)
    assert ids.tolist() == [[-1, -1, -1]] and bool(torch.isnan(tlp).all()) and math.isnan(lp[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(1, 40), (12, 9000), (7, 128256), (400, 5003), (3, 300001)])
def test_logprobs_large_finite_logits(amk, dtype, rows, vocab):
    """Rows masked with large finite values, rows whose maximum is far from zero, and rows of nothing but such values: NaN is for
    NaN and infinities alone.  A difference of two logits is rounded once (2^-24 of it) and is no larger than the log
    probability and log(vocab) <= 13 together; exponentials are good to 2^-21, the sums of n terms to n 2^-30."""
    g = gen(rows + vocab)
    far = [5e9, 1e10, 1e20, 3e6, 1e6, 1e30, 3e37, 4.5e9]
    kinds = [lambda i, c: ((torch.full((vocab,), -c, device=DEV)).scatter_(0, torch.randperm(vocab, generator=g, device=DEV)[:4],
                                                                          3 * torch.randn(4, generator=g, device=DEV))),
             lambda i, c: torch.randn(vocab, generator=g, device=DEV).scatter_(0, torch.tensor([vocab // 3], device=DEV), c),
             lambda i, c: torch.full((vocab,), -c if i % 2 else c, device=DEV),
             lambda i, c: c * torch.randn(vocab, generator=g, device=DEV),
             lambda i, c: torch.cat([torch.full((vocab // 2,), -c, device=DEV), torch.randn(vocab - vocab // 2, generator=g, device=DEV)]),
             lambda i, c: torch.randn(vocab, generator=g, device=DEV) * 4 - c]
    for at in range(0, len(far) * len(kinds), rows):
        pick = [(kinds[(at + i) % len(kinds)], far[(at + i) // len(kinds) % len(far)], i) for i in range(rows)]
        x = torch.stack([k(i, c) for k, c, i in pick]).to(dtype)
        assert bool(torch.isfinite(x).all())
        tokens = x.argmax(1).to(torch.int32)
        tokens[1::2] = torch.randint(0, vocab, (len(tokens[1::2]),), generator=g, device=DEV).to(torch.int32)
        got = amk.amk_token_logprobs(x, tokens, 8)
        want = logprobs64(x, tokens, 8)
        assert torch.equal(got[2].long(), want[2])
        for a, b in ((got[0], want[0]), (got[1], want[1]), (got[3], want[3])):
            tol = 2.0 ** -22 * (b.abs() + 13) + 2.0 ** -21 + vocab * 2.0 ** -30
            bad = ~((a.double() - b).abs() <= tol)
            assert not bool(bad.any()), (at, a[bad][:4].tolist(), b[bad][:4].tolist())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(1, 70), (70, 4980), (7, 128256), (600, 3001)])
@pytest.mark.parametrize("low", [-1.5e6, -1e7, -5e9, -1e30, -3e38])
def test_logprobs_low_logits_beside_minus_infinity(amk, dtype, rows, vocab, low):
    """Rows of -infinity but for a few logits far below zero, which lie in one part of the row or in several: one, two equal
    ones, and one with others far below it."""
    g = gen(vocab)
    x = torch.full((rows, vocab), -math.inf, device=DEV)
    place = torch.stack([torch.randperm(vocab, generator=g, device=DEV)[:5] for _ in range(rows)])
    for r in range(rows):
        x[r, place[r, 0]] = low
        if r % 3 == 1:
            x[r, place[r, 1]] = low
        if r % 3 == 2:
            x[r, place[r, 2:]] = low * 1.06
    x = x.to(dtype)
    tokens = place[:, 0].to(torch.int32)
    got, want = amk.amk_token_logprobs(x, tokens, 5), logprobs64(x, tokens, 5)
    assert torch.equal(got[2].long(), want[2])
    for a, b in ((got[0], want[0]), (got[1], want[1]), (got[3], want[3])):
        tol = 2.0 ** -22 * (b.abs().nan_to_num(0, 0, 0) + 13) + 2.0 ** -21 + vocab * 2.0 ** -30
        assert bool(((a.double() == b) | ((a.double() - b).abs() <= tol)).all())


def test_logprobs_token_agrees_with_argmax_static_and_replays(amk):
    g = gen(2)
    x = randn(g, 4, 32000, dtype=torch.float32)
    x[2, 100] = x[2, 31000] = 20.0
    tok = torch.zeros(1, dtype=torch.int32, device=DEV)
    tokens = torch.zeros(4, dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lp, ent, ids, tlp = amk.amk_token_logprobs(x, tokens, 1)
    graph.replay()
    for r in range(4):
        amk.amk_argmax_static(x[r], tok)
        assert int(tok) == int(ids[r, 0])
    x.copy_(randn(g, 4, 32000, dtype=torch.float32))
    graph.replay()
    eager = amk.amk_token_logprobs(x, tokens, 1)
    for a, b in zip((lp, ent, ids, tlp), eager):
        assert torch.equal(a, b)


def test_logprobs_rows_beyond_32_bit_offsets(amk):
    rows, vocab = 70000, 32768
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device=DEV)
    assert x.numel() > 1 << 31
    x[-1, 77] = 10.0
    x[35000, 5] = 3.0
    tokens = torch.full((rows,), 77, dtype=torch.int32, device=DEV)
    lp, ent, ids, tlp = amk.amk_token_logprobs(x, tokens, 1)
    pick = torch.tensor([0, 35000, rows - 1], device=DEV)
    want = logprobs64(x[pick], tokens[pick], 1)
    close(lp[pick], want[0], 30.0, vocab)
    close(ent[pick], want[1], 30.0, vocab)
    assert ids[pick].flatten().tolist() == [0, 5, 77]


# ---- compacting a cache -----------------------------------------------------------------------------------------

def compact_ref(kv, base, keep, count):
    out = kv.clone()
    for c in range(kv.shape[0]):
        if count[c]:
            idx = torch.tensor(keep[c][:count[c]], device=kv.device)
            out[c, ..., base[c]:base[c] + count[c], :] = kv[c].index_select(-2, idx)
    return out


def run_compact(amk, kv, base, keep, count):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    amk.amk_kv_compact(kv, i32(base), i32(keep), i32(count))


@pytest.mark.parametrize("dtype,hd", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.uint8, 64), (torch.uint8, 16),
                                      (torch.float32, 256), (torch.uint8, 48)])
@pytest.mark.parametrize("caches,planes,slots,most", [(1, 3, 1, 1), (2, 8, 100, 100), (3, 512, 300, 40), (1, 5, 3001, 2900),
                                                      (2, 2, 1025, 1000), (1, 300, 700, 690)])
def test_compact(amk, dtype, hd, caches, planes, slots, most):
    g = gen(slots + hd)
    rng = np.random.default_rng(slots + hd)
    kv = (torch.rand(caches, planes, slots, hd, generator=g, device=DEV) * 250).to(dtype)
    base, keep, count = [], [], []
    for c in range(caches):
        b = int(rng.integers(0, slots - most + 1))
        n = [most, int(rng.integers(0, most + 1)), 0][c % 3]
        rows = b + np.sort(rng.choice(slots - b, n, replace=False))
        base.append(b), count.append(n)
        keep.append([int(x) for x in rows] + [-5] * (most - n))
    want = compact_ref(kv, base, keep, count)
    run_compact(amk, kv, base, keep, count)
    assert torch.equal(kv, want)


@pytest.mark.parametrize("shift", [0, 1, 7, 500])
def test_compact_moves_down_over_itself(amk, shift):
    """Long runs that overlap their destination, and rows that stay where they are."""
    kv = torch.randn(2, 4, 4000, 64, device=DEV).to(torch.bfloat16)
    n = 3500 - shift
    rows = list(range(10 + shift, 10 + shift + n))
    want = compact_ref(kv, [10, 10], [rows, rows], [n, n - 1])
    run_compact(amk, kv, [10, 10], [rows, rows], [n, n - 1])
    assert torch.equal(kv, want)


@pytest.mark.parametrize("base,keep,count", [(-1, [5, 6, 7], 3), (0, [5, 5, 7], 3), (0, [7, 6, 8], 3), (6, [5, 6, 7], 3),
                                             (0, [5, 6, 100], 3), (0, [-1, 6, 7], 3), (0, [5, 6, 7], 4), (0, [5, 6, 7], -1)])
def test_compact_leaves_a_cache_with_a_bad_list_alone(amk, base, keep, count):
    kv = torch.randn(3, 4, 100, 64, device=DEV).to(torch.bfloat16)
    good = [8, 20, 99]
    want = compact_ref(kv, [3, 0, 0], [good, good, good], [3, 0, 2])
    run_compact(amk, kv, [3, base, 0], [good, keep, good], [3, count, 2])
    assert torch.equal(kv, want)


def test_compact_a_slice_of_a_larger_buffer(amk):
    """Caches with other memory between them, guard rows on both sides, replayed with new lists."""
    buf = torch.randn(3, 1000, 64, device=DEV).to(torch.bfloat16)
    kv = buf[:, 200:800].view(3, 6, 100, 64)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    base, keep, count = i32([0, 0, 0]), i32([[1, 2], [3, 9], [0, 1]]), i32([0, 0, 0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        amk.amk_kv_compact(kv, base, keep, count)
    before = buf.clone()
    graph.replay()
    assert torch.equal(buf, before)
    count.copy_(i32([2, 1, 2]))
    want = compact_ref(kv, [0, 0, 0], [[1, 2], [3, 9], [0, 1]], [2, 1, 2])
    graph.replay()
    assert torch.equal(kv, want) and torch.equal(buf[:, :200], before[:, :200]) and torch.equal(buf[:, 800:], before[:, 800:])


def test_compact_offsets_beyond_32_bits(amk):
    kv = torch.zeros(1, 17, 1 << 20, 128, dtype=torch.bfloat16, device=DEV)
    assert kv.numel() * 2 > 1 << 32
    kv[0, -1, -3:] = torch.arange(3, device=DEV)[:, None].to(torch.bfloat16) + 1
    run_compact(amk, kv, [4], [[9, (1 << 20) - 3, (1 << 20) - 1]], [3])
    assert kv[0, -1, 4:8, 0].tolist() == [0.0, 1.0, 3.0, 0.0] and float(kv[0, :-1].abs().max()) == 0.0


# ---- refusals of the Python layer ---------------------------------------------------------------------------------

def test_python_layer_refuses_what_does_not_fit(amk):
    q, k, v, cu = prompt_inputs([20], 4, 2, 64, 1)
    bad = [lambda: amk.amk_prompt_attention(q.float(), k, v, cu), lambda: amk.amk_prompt_attention(q, k[:, :1], v, cu),
           lambda: amk.amk_prompt_attention(q, k, v, cu.long()), lambda: amk.amk_prompt_attention(q, k, v, cu.cpu()),
           lambda: amk.amk_prompt_attention(q.transpose(1, 2).contiguous().transpose(1, 2), k, v, cu),
           lambda: amk.amk_prompt_attention(q, k, v, cu, out=torch.empty(20, 4, 64, device=DEV)),
           lambda: amk.amk_prompt_attention(q, k, v, cu, lse=torch.empty(4, 20, device=DEV)),
           lambda: amk.amk_token_logprobs(torch.zeros(2, 9, device=DEV), cu[:1], 1),
           lambda: amk.amk_token_logprobs(torch.zeros(2, 9, device=DEV, dtype=torch.float16), cu),
           lambda: amk.amk_token_logprobs(torch.zeros(9, 2, device=DEV).t(), cu),
           lambda: amk.amk_kv_compact(torch.zeros(1, 4, 8, 64, device=DEV).transpose(1, 2), cu[:1], cu[None], cu[:1]),
           lambda: amk.amk_kv_compact(torch.zeros(2, 4, 8, 64, device=DEV), cu[:1], cu[None], cu[:1])]
    qt, kt, vt = tree_inputs(2, 3, 50, 4, 2, 64, "bf16", 1)
    length = torch.zeros(2, dtype=torch.int32, device=DEV)
    bad += [lambda: amk.amk_tree_attention(qt, kt, vt.view(torch.uint8)[..., :64], length),
            lambda: amk.amk_tree_attention(qt, kt, vt, length[:1]),
            lambda: amk.amk_tree_attention(qt, kt, vt, length, torch.zeros(2, 3, 2, dtype=torch.int64, device=DEV)),
            lambda: amk.amk_tree_attention(qt, kt, vt, length, max_len=-1),
            lambda: amk.amk_tree_attention(qt, kt[:, :, :2], vt[:, :, :2], length)]
    for i, call in enumerate(bad):
        with pytest.raises(amk.AmkError) as e:
            call()
        assert e.value.code == amk.AMK_ERR_INVALID_ARG, i
    with pytest.raises(amk.AmkError) as e:
        amk.amk_token_logprobs(torch.zeros(2, 90, device=DEV), cu, 33)
    assert e.value.code == amk.AMK_ERR_UNSUPPORTED


@pytest.mark.parametrize("scale", [0.0, -1.0, math.nan, math.inf])
def test_python_layer_refuses_a_scale_that_is_none(amk, scale):
    """Zero would mean the default in the C struct."""
    q, k, v, cu = prompt_inputs([20], 4, 2, 64, 1)
    qt, kt, vt = tree_inputs(2, 3, 50, 4, 2, 64, "bf16", 1)
    for call in (lambda: amk.amk_prompt_attention(q, k, v, cu, scale=scale),
                 lambda: amk.amk_tree_attention(qt, kt, vt, torch.zeros(2, dtype=torch.int32, device=DEV), scale=scale)):
        with pytest.raises(amk.AmkError) as e:
            call()
        assert e.value.code == amk.AMK_ERR_INVALID_ARG


@pytest.mark.parametrize("scale", [1e-46, 1e-320, 1e39, 2.4e38])
def test_python_layer_refuses_a_scale_that_fp32_cannot_hold(amk, scale):
    """What rounds to zero would mean the default; scale and scale log2 e have to be finite."""
    q, k, v, cu = prompt_inputs([20], 4, 2, 64, 1)
    qt, kt, vt = tree_inputs(2, 3, 50, 4, 2, 64, "bf16", 1)
    for call in (lambda: amk.amk_prompt_attention(q, k, v, cu, scale=scale),
                 lambda: amk.amk_tree_attention(qt, kt, vt, torch.zeros(2, dtype=torch.int32, device=DEV), scale=scale)):
        with pytest.raises(amk.AmkError) as e:
            call()
        assert e.value.code == amk.AMK_ERR_INVALID_ARG and "scale" in str(e.value)


def test_a_bound_of_no_context_is_a_bound(amk, monkeypatch):
    """max_len = 0 states that every context is empty; in the C struct 0 means that nothing is known."""
    q, k, v = tree_inputs(2, 3, 9000, 4, 2, 64, "bf16", 1)
    length = torch.zeros(2, dtype=torch.int32, device=DEV)
    seen, run = [], amk._run
    monkeypatch.setattr(amk, "_run", lambda fn, name, index, args: (seen.append(amk.amk_tree_args.from_buffer_copy(args).max_len),
                                                                    run(fn, name, index, args)))
    for bound in (None, 0, 1, 500):
        out = amk.amk_tree_attention(q, k, v, length, max_len=bound)
        check_tree(q, k, v, [0, 0], np.tril(np.ones((2, 3, 3), bool)), out, None, 0.125, bound)
    assert seen == [0, 1, 1, 500]


def test_python_layer_refuses_inputs_that_want_gradients(amk):
    """The operators have no backward pass: where autograd would record the call, it is refused; elsewhere it runs."""
    q, k, v, cu = prompt_inputs([20], 4, 2, 64, 1)
    qt, kt, vt = tree_inputs(2, 3, 50, 4, 2, 64, "bf16", 1)
    length = torch.zeros(2, dtype=torch.int32, device=DEV)
    x, kv = torch.zeros(2, 90, device=DEV), torch.zeros(1, 4, 8, 64, device=DEV)
    grad = lambda t: t.detach().clone().requires_grad_()
    one, keep = cu[:1], cu[None, 1:]
    calls = [lambda: amk.amk_prompt_attention(grad(q), k, v, cu), lambda: amk.amk_prompt_attention(q, grad(k), v, cu),
             lambda: amk.amk_prompt_attention(q, k, grad(v), cu), lambda: amk.amk_prompt_attention(q, k, v, cu, out=grad(q)),
             lambda: amk.amk_prompt_attention(q, k, v, cu, lse=grad(torch.zeros(20, 4, device=DEV))),
             lambda: amk.amk_tree_attention(grad(qt), kt, vt, length), lambda: amk.amk_tree_attention(qt, grad(kt), vt, length),
             lambda: amk.amk_tree_attention(qt, kt, grad(vt), length), lambda: amk.amk_tree_attention(qt, kt, vt, length, out=grad(qt)),
             lambda: amk.amk_token_logprobs(grad(x), cu), lambda: amk.amk_kv_compact(grad(kv), one, keep, one)]
    for i, call in enumerate(calls):
        with pytest.raises(amk.AmkError) as e:
            call()
        assert e.value.code == amk.AMK_ERR_UNSUPPORTED and "gradient" in str(e.value), i
        with torch.no_grad():
            call()


# ---- together ---------------------------------------------------------------------------------------------------

def forward(shape, w, tokens, positions, attend):
    """The layers of the model in plain fp32 torch around an attention given by ``attend(layer, q, k, v)`` (k rotated)."""
    f = lambda t: t.float()
    hd, nq, nkv = shape.head_dim, shape.n_q_heads, shape.n_kv_heads

    def norm(x, g):
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + shape.rms_eps) * f(g)

    freq = shape.rope_theta ** (-torch.arange(0, hd, 2, device=DEV, dtype=torch.float64) / hd)
    ang = positions.double()[:, None] * freq
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]

    def rope(x):
        a, b = x[..., :hd // 2], x[..., hd // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    x = f(w["embed"])[tokens.long()]
    for l in range(shape.n_layers):
        h = norm(x, w["attn_norm"][l])
        n = len(tokens)
        q, k, v = ((h @ f(w[m][l]).t()).view(n, -1, hd) for m in ("wq", "wk", "wv"))
        o = attend(l, rope(q).to(torch.bfloat16), rope(k).to(torch.bfloat16), v.to(torch.bfloat16))
        x = x + o.float().reshape(n, nq * hd) @ f(w["wo"][l]).t()
        h = norm(x, w["mlp_norm"][l])
        x = x + (torch.nn.functional.silu(h @ f(w["wgate"][l]).t()) * (h @ f(w["wup"][l]).t())) @ f(w["wdown"][l]).t()
    head = w["embed"] if shape.tied else w["lm_head"]
    return norm(x, w["final_norm"]) @ f(head).t()


@pytest.mark.parametrize("name,kv_dtype", [("mini", "bf16"), ("mini_hd128", "bf16"), ("mini_ragged", "bf16"), ("mini", "fp8")])
def test_prompt_draft_verify_compact_and_decode(amk, name, kv_dtype):
    """A prompt through the prompt attention into a decoder's cache, a draft tree verified over it, the accepted tokens'
    rows compacted, and the decode step going on from there -- against the same decoder fed token by token."""
    shape = inp.SHAPES[name]
    w = inp.make_weights(shape, 99, device=DEV, std=0.05, norm_jitter=0.1)
    dec = amk.Decoder(shape, w, "bf16", kv_dtype=kv_dtype)
    n_prompt, n_new = 37, 9
    prompt = torch.randint(0, shape.vocab, (n_prompt,), generator=gen(3), device=DEV)

    # the reference: one step per token, then greedy
    kv_ref, toks, logits_ref = dec.new_cache(), prompt.tolist(), []
    for pos in range(n_prompt + n_new):
        dec.amk_decode_step(toks[pos], pos, kv_ref)
        assert dec.amk_last_status()[0] == 0
        logits_ref.append(dec.logits.clone())
        if pos + 1 >= len(toks):
            toks.append(int(dec.next_token))

    # the prompt in one go, its K/V rows into the cache
    kv = dec.new_cache()
    K, V = dec.cache_views(kv)
    code = (lambda t: t.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)) if kv_dtype == "fp8" else (lambda t: t)
    value = (lambda t: t.view(torch.float8_e4m3fn).to(torch.bfloat16)) if kv_dtype == "fp8" else (lambda t: t)
    cu = torch.tensor([0, n_prompt], dtype=torch.int32, device=DEV)

    def attend_prompt(l, q, k, v):
        K[l, :, :n_prompt], V[l, :, :n_prompt] = code(k).permute(1, 0, 2), code(v).permute(1, 0, 2)
        return amk.amk_prompt_attention(q, value(code(k)), value(code(v)), cu)   # what the cache holds is attended to

    logits = forward(shape, w, prompt, torch.arange(n_prompt, device=DEV), attend_prompt)
    near = lambda a, b: float((a - b).norm() / b.norm())
    # 3e-2: the roundings of q, k, v and the attention's output to bf16, through the layers.  With the 8-bit cache the two
    # sides round values that differ by up to 2^-8 (here to bf16 first) to e4m3, whose borders lie at least 2^-4 of the
    # value apart: at most 2 * 2^-8 / 2^-4 = 2^-3 of the entries fall on different sides, each then a step of at most 2^-3
    # apart: sqrt(2^-3) 2^-3 = 4.4e-2 of the norm of K and of V, which is what the layers' outputs can inherit
    tol_logits = 3e-2 + (4.4e-2 if kv_dtype == "fp8" else 0.0)
    assert near(logits[-1], logits_ref[n_prompt - 1]) < tol_logits
    lp, ent, ids, tlp = amk.amk_token_logprobs(logits[:-1], prompt[1:].to(torch.int32), 1)   # the prompt's own score
    want = torch.log_softmax(torch.stack(logits_ref[:n_prompt - 1]), 1).gather(1, prompt[1:, None])[:, 0]
    assert bool(torch.isfinite(lp).all()) and float((lp - want).abs().max()) < 0.25

    # a draft whose tree holds the greedy continuation among wrong tokens
    true = toks[n_prompt:n_prompt + n_new]
    nodes, parent, path, at = [], [], [], -1
    for t in true[:6]:
        nodes += [(t + 1) % shape.vocab, t, (t + 3) % shape.vocab]
        parent += [at] * 3
        at = len(nodes) - 2
        path.append(at)
    rows = len(nodes)
    sees, depth = np.zeros((1, rows, rows), dtype=bool), []
    for i in range(rows):
        if parent[i] >= 0:
            sees[0, i] = sees[0, parent[i]]
        sees[0, i, i] = True
        depth.append(int(sees[0, i].sum()) - 1)
    mask, length = words(sees), torch.tensor([n_prompt], dtype=torch.int32, device=DEV)

    def attend_tree(l, q, k, v):
        s = slice(n_prompt, n_prompt + rows)
        K[l, :, s], V[l, :, s] = code(k).permute(1, 0, 2), code(v).permute(1, 0, 2)
        return amk.amk_tree_attention(q[None], K[l][None], V[l][None], length, mask)[0]

    draft = torch.tensor(nodes, device=DEV)
    logits_t = forward(shape, w, draft, n_prompt + torch.tensor(depth, device=DEV), attend_tree)
    for i, node in enumerate(path):
        assert near(logits_t[node], logits_ref[n_prompt + i]) < tol_logits, i

    # verification: along the accepted path the true next token is (within the noise of 16 bits) the most likely one
    nxt = torch.tensor([toks[n_prompt + d + 1] for d in depth], dtype=torch.int32, device=DEV)
    lp, _, ids, tlp = amk.amk_token_logprobs(logits_t, nxt, 3)
    assert bool((lp[path] >= tlp[path, 0] - 0.1).all())

    # the accepted rows move together; the step goes on as if they had been decoded one by one
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    dec.amk_kv_compact(kv, length, i32([[n_prompt + j for j in path]]), i32([len(path)]))
    K_ref, V_ref = dec.cache_views(kv_ref)
    n = n_prompt + len(path)
    tol = 2e-1 if kv_dtype == "fp8" else 2e-2
    for a, b in ((K, K_ref), (V, V_ref)):
        assert near(value(a[:, :, :n].contiguous()).float(), value(b[:, :, :n].contiguous()).float()) < tol
    for pos in range(n, n_prompt + n_new):
        dec.amk_decode_step(toks[pos], pos, kv)
        assert dec.amk_last_status()[0] == 0
        assert near(dec.logits, logits_ref[pos]) < tol_logits, pos
    dec.close()


@pytest.mark.parametrize("name,kv_dtype", [("mini", "bf16"), ("mini_hd128", "bf16"), ("mini", "fp8")])
def test_a_cache_without_its_middle_goes_on_with_the_tree_attention(amk, name, kv_dtype):
    """The first tokens and a recent window of a decoder's cache, moved together: queries rotated for their true positions
    attend to the kept rows and to the new ones behind them, as a plain attention over those rows does.
    2e-2: one rounding of each attention's output to bf16 on either side (2^-8), and twice that of its numerators, through the
    layers; the kept 8-bit rows are the same on both sides, and the three new ones differ by a step where a value lies next to
    a border."""
    shape = inp.SHAPES[name]
    w = inp.make_weights(shape, 7, device=DEV, std=0.05, norm_jitter=0.1)
    dec = amk.Decoder(shape, w, "bf16", kv_dtype=kv_dtype)
    n, first, window, new = 60, 4, 21, 3
    tokens = torch.randint(0, shape.vocab, (n + new,), generator=gen(4), device=DEV)
    kv = dec.new_cache()
    for pos in range(n):
        dec.amk_decode_step(int(tokens[pos]), pos, kv)
        assert dec.amk_last_status()[0] == 0
    keep = list(range(first)) + list(range(n - window, n))
    code = (lambda t: t.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)) if kv_dtype == "fp8" else (lambda t: t)
    value = (lambda t: t.contiguous().view(torch.float8_e4m3fn).float()) if kv_dtype == "fp8" else (lambda t: t.float())
    before = kv.clone()
    Kb, Vb = (value(t)[:, :, keep] for t in dec.cache_views(before))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    dec.amk_kv_compact(kv, i32([0]), i32([keep]), i32([len(keep)]))
    K, V = dec.cache_views(kv)
    at, length = len(keep), i32([len(keep)])

    def tree(l, q, k, v):
        K[l, :, at:at + new], V[l, :, at:at + new] = code(k).permute(1, 0, 2), code(v).permute(1, 0, 2)
        return amk.amk_tree_attention(q[None], K[l][None], V[l][None], length)[0]

    def plain(l, q, k, v):
        rep = shape.n_q_heads // shape.n_kv_heads
        keys, values = (torch.cat([old[l], value(code(t)).permute(1, 0, 2)], 1).double().repeat_interleave(rep, 0)
                        for old, t in ((Kb, k), (Vb, v)))
        x = q.double().permute(1, 0, 2) @ keys.transpose(1, 2) * shape.head_dim ** -0.5
        hidden = torch.ones(new, at + new, dtype=torch.bool, device=DEV).triu(at + 1)
        return (torch.softmax(x.masked_fill(hidden, -math.inf), 2) @ values).permute(1, 0, 2).to(torch.bfloat16)

    where = n + torch.arange(new, device=DEV)
    got, want = forward(shape, w, tokens[n:], where, tree), forward(shape, w, tokens[n:], where, plain)
    assert float((got - want).norm() / want.norm()) < 2e-2
    dec.close()
