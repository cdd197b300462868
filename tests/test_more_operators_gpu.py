"""GPU tests of the operators between projection, attention and cache, each against a plain implementation in 64 bits.

Tolerances, element by element; eps is half a step of the result's type (bf16 2^-8, e4m3 2^-4 and 2^-10 near zero):
  - norm and rotation: with A, B the normed elements of a pair, fp32 operations (2^-24 each, under ten of them), an angle off by
    2^-25 of a turn (2^-22.3) and its sine by 2^-23: less than 2^-19 (|A| + |B|); then one rounding, eps |out|;
  - attention weights: a score is off by at most E = head_dim 2^-23 sum |q||k| scale (2^-23: also for adders that truncate), the
    log-sum-exp in base 2 by 2^-23 |lse|, the exponent by 2^-23 of itself, the power by 2^-21, all factors of a term;
    a sum of n terms is off by n 2^-24 of itself;
  - choices (positions, tokens) are equal.
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


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def value(t):
    return t.view(torch.float8_e4m3fn).double() if t.dtype == torch.uint8 else t.double()


def code(t):
    return t.float().to(torch.float8_e4m3fn).view(torch.uint8)


# ---- norm, rotation, storing ------------------------------------------------------------------------------------

def rotated64(x, weight, positions, theta, eps):
    """(the rotated heads in 64 bits, |A| + |B| of each element's pair)"""
    x = x.double()
    hd = x.shape[2]
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(2, keepdim=True) + eps) * weight.double()
    i = torch.arange(hd // 2, device=DEV, dtype=torch.float64)
    a = positions.double()[:, None] * torch.pow(torch.tensor(float(np.float32(theta)), dtype=torch.float64, device=DEV), -2 * i / hd)
    c, s = a.cos()[:, None], a.sin()[:, None]
    lo, hi = x[..., :hd // 2], x[..., hd // 2:]
    both = (lo.abs() + hi.abs()).repeat(1, 1, 2)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], 2), both


def near16(got, want, both):
    assert not bool(torch.isnan(got).any())
    assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * both).all())


def near8(got, want, both):
    want = want.clamp(-448, 448)
    assert bool(((value(got) - want).abs() <= (2.0 ** -4 * want.abs()).clamp(min=2.0 ** -10) + 2.0 ** -19 * both).all())


@pytest.mark.parametrize("nq,nkv,hd", [(9, 3, 64), (32, 8, 128), (1, 1, 64), (5, 2, 128), (40, 1, 64), (33, 17, 128)])
@pytest.mark.parametrize("rows", [1, 2, 37, 1300])
@pytest.mark.parametrize("cache", ["bf16", "fp8", None])
def test_norm_rope_append(amk, nq, nkv, hd, rows, cache):
    g = gen(rows * 31 + nq)
    x = randn(g, rows, nq + 2 * nkv, hd) * 1.5
    q, k, v = x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:]
    pos = torch.randint(0, 9000, (rows,), generator=g, device=DEV).to(torch.int32)
    pos[::3] = 0
    weights = [(None, None), (1, 1), (1, None), (None, 1)][(rows + nq) % 4]
    wq, wk = [None if w is None else (1 + 0.3 * randn(g, hd, dtype=torch.float32)).to(torch.bfloat16) for w in weights]
    seqs, slots = 3, rows + 5
    where = torch.randperm(seqs * slots, generator=g, device=DEV)[:rows]
    if rows > 2:
        where[1], where[2] = -1, seqs * slots           # not stored
    caches = (None, None, None)
    if cache:
        kc, vc = (randn(g, seqs, nkv, slots, hd) for _ in range(2))
        if cache == "fp8":
            kc, vc = code(kc), code(vc)
        caches = (kc, vc, where)
        k0, v0 = kc.clone(), vc.clone()
    k_out = torch.empty(rows, nkv, hd, dtype=torch.bfloat16, device=DEV)
    before = x.clone()
    q_out = amk.amk_norm_rope_append(q, k, v if cache else None, pos, *caches, q_weight=wq, k_weight=wk, eps=1e-5, theta=5e5, k_out=k_out)
    assert torch.equal(x, before)
    wantq, bothq = rotated64(q, wq, pos, 5e5, 1e-5)
    wantk, bothk = rotated64(k, wk, pos, 5e5, 1e-5)
    near16(q_out, wantq, bothq)
    near16(k_out, wantk, bothk)
    if not cache:
        return
    stored = (where >= 0) & (where < seqs * slots)
    at = where[stored]
    s, r = at // slots, at % slots
    if cache == "fp8":
        near8(kc[s, :, r], wantk[stored], bothk[stored])
        assert torch.equal(vc[s, :, r], v[stored].float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    else:
        near16(kc[s, :, r], wantk[stored], bothk[stored])
        assert torch.equal(vc[s, :, r], v[stored])
    kc[s, :, r], vc[s, :, r] = k0[s, :, r], v0[s, :, r]
    assert torch.equal(kc, k0) and torch.equal(vc, v0)  # nothing else was written


def test_norm_rope_append_far_positions(amk):
    """Angles of positions that 32 bits cannot hold times a frequency, negative ones among them."""
    pos = i32([0, 1, -1, 65537, 1 << 20, (1 << 24) + 1, -(1 << 24) - 3, (1 << 31) - 1, -(1 << 31)])
    for hd in (64, 128):
        q, k = randn(gen(5), 9, 3, hd), randn(gen(6), 9, 2, hd)
        k_out = torch.empty_like(k)
        got = amk.amk_norm_rope_append(q, k, None, pos, theta=10000.0, k_out=k_out)
        for out, x in ((got, q), (k_out, k)):
            want, both = rotated64(x, None, pos, 10000.0, 0)
            near16(out, want, both)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_norm_rope_append_norms_beyond_32_bits(amk, hd, eps):
    """Heads whose squares are more than fp32's largest number or less than its smallest, next to ordinary ones."""
    g = gen(hd)
    powers = torch.tensor([0, 120, -120, 70, -70, 64, -64, 63, -50, -49, 60, 100, -100, 0, 1], device=DEV)
    q, k = randn(g, 40, 15, hd, dtype=torch.float32), randn(g, 40, 3, hd, dtype=torch.float32)
    q, k = (q * torch.pow(2.0, powers[:, None].float())).to(torch.bfloat16), (k * 2.0 ** 100).to(torch.bfloat16)
    w = (1 + 0.3 * randn(g, hd, dtype=torch.float32)).to(torch.bfloat16)
    pos = torch.arange(40, device=DEV, dtype=torch.int32) * 7
    k_out = torch.empty_like(k)
    got = amk.amk_norm_rope_append(q, k, None, pos, q_weight=w, k_weight=w, eps=eps, k_out=k_out)
    for out, x in ((got, q), (k_out, k)):
        want, both = rotated64(x, w, pos, 10000.0, float(np.float32(eps)))
        near16(out, want, both)


@pytest.mark.parametrize("hd", [64, 128])
def test_norm_rope_append_in_place_and_strides(amk, hd):
    g = gen(hd)
    rows, nq, nkv = 21, 6, 2
    w = (1 + 0.2 * randn(g, hd, dtype=torch.float32)).to(torch.bfloat16)
    pos = torch.arange(rows, device=DEV, dtype=torch.int32) * 7
    x = randn(g, rows, nq + 2 * nkv, hd)
    q, k, v = x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:]
    want = amk.amk_norm_rope_append(q.clone(), k.clone(), None, pos, q_weight=w, k_weight=w, k_out=(k_out := torch.empty_like(k)))
    v0 = v.clone()
    assert amk.amk_norm_rope_append(q, k, None, pos, q_weight=w, k_weight=w, q_out=q, k_out=k) is q
    assert torch.equal(q, want) and torch.equal(k, k_out) and torch.equal(v, v0)
    # heads in front of rows, rows with a gap, a cache with rows in front of heads
    q2 = randn(g, nq, rows, hd).transpose(0, 1)
    k2, v2 = (randn(g, rows, 3 * nkv, hd)[:, ::3] for _ in range(2))
    kc = torch.zeros(2, 40, nkv, hd, dtype=torch.bfloat16, device=DEV).transpose(1, 2)
    vc = torch.zeros(2, nkv, 40, 2 * hd, dtype=torch.bfloat16, device=DEV)[..., :hd]
    out = torch.zeros(nq, rows, hd, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    where = 40 + torch.arange(rows, device=DEV)
    amk.amk_norm_rope_append(q2, k2, v2, pos, kc, vc, where, q_out=out)
    plain_k = torch.empty(rows, nkv, hd, dtype=torch.bfloat16, device=DEV)
    assert torch.equal(out, amk.amk_norm_rope_append(q2.contiguous(), k2.contiguous(), None, pos, k_out=plain_k))
    assert torch.equal(kc[1, :, :rows], plain_k.transpose(0, 1)) and torch.equal(vc[1, :, :rows], v2.transpose(0, 1))
    assert not bool(kc[0].any()) and not bool(vc[0].any()) and not bool(kc[1, :, rows:].any())


def test_norm_rope_append_broken_values_stay_in_their_head(amk):
    x = randn(gen(8), 5, 8, 64)
    x[2, 3, 7], x[3, 5, 40], x[4, 6, 0] = math.nan, math.inf, 3e38
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    w = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    pos = torch.arange(5, device=DEV, dtype=torch.int32)
    for cache_type in (torch.bfloat16, torch.uint8):
        kc, vc = (torch.zeros(1, 2, 8, 64, device=DEV, dtype=cache_type) for _ in range(2))
        out = amk.amk_norm_rope_append(q, k, v, pos, kc, vc, torch.arange(5, device=DEV), q_weight=w, k_weight=w)
        bad = torch.isnan(out.float()).any(2)
        assert bad.sum() == 1 and bool(bad[2, 3])
        badk = torch.isnan(value(kc)).any(3)[0]
        assert badk.sum() == 1 and bool(badk[1, 3])
        assert float(value(vc)[0, 0, 4, 0]) == (448.0 if cache_type == torch.uint8 else float(x[4, 6, 0]))
    amk.amk_norm_rope_append(x[:0, :4], x[:0, 4:6], None, pos[:0])


# ---- attention weights ------------------------------------------------------------------------------------------

def weights64(q, k, lse, length, before, decay, scale):
    """(out, tolerance), both fp64 [n_seqs][n_kv][slots]"""
    seqs, rows, nq, hd = q.shape
    nkv, slots = k.shape[1:3]
    rep = nq // nkv
    out = torch.zeros(seqs, nkv, slots, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(out)
    for s, n in enumerate(length):
        if n < 0 or n > slots - rows:
            out[s] = math.nan
            continue
        keys = n + rows
        sees = torch.arange(keys, device=DEV)[None] <= n + torch.arange(rows, device=DEV)[:, None]
        for h in range(nq):
            kd, qd, l = value(k[s, h // rep, :keys]), q[s, :, h].double(), lse[s, :, h].double()
            x, size = scale * (qd @ kd.T), scale * (qd.abs() @ kd.abs().T)
            y = x - l[:, None]
            p = torch.where(sees & ~torch.isinf(l)[:, None], torch.exp(y), 0.0)
            off = hd * 2.0 ** -23 * size + 2.0 ** -23 * l.abs()[:, None] + 2.0 ** -23 * y.abs() + 2.0 ** -21
            out[s, h // rep, :keys] += p.sum(0)
            tol[s, h // rep, :keys] += torch.where(p > 0, p * (off + rows * rep * 2.0 ** -24), 0.0).sum(0)
        if before is not None:
            old = decay * before[s, :, :n].double()
            out[s, :, :n] += old
            tol[s, :, :n] += 2.0 ** -23 * (old.abs() + out[s, :, :n].abs())
    return out, tol + 1e-37


def true_lse(q, k, length, scale):
    seqs, rows, nq, hd = q.shape
    nkv, slots = k.shape[1:3]
    lse = torch.full((seqs, rows, nq), -math.inf, device=DEV)
    for s, n in enumerate(length):
        if n < 0 or n > slots - rows:
            continue
        sees = torch.arange(n + rows, device=DEV)[None] <= n + torch.arange(rows, device=DEV)[:, None]
        for h in range(nq):
            x = scale * (q[s, :, h].double() @ value(k[s, h // (nq // nkv), :n + rows]).T)
            lse[s, :, h] = torch.logsumexp(x.masked_fill(~sees, -math.inf), 1).float()
    return lse


def weights_agree(got, want, tol):
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    bad = ~((got.double() - want).abs() <= tol) & ~torch.isnan(want)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), float(((got.double() - want).abs() / tol)[bad].max()))


@pytest.mark.parametrize("nq,nkv,hd", [(9, 3, 64), (32, 8, 128), (4, 4, 64), (16, 1, 128), (10, 2, 64), (7, 1, 128)])
@pytest.mark.parametrize("rows,slots,lens", [(1, 1, [0]), (1, 300, [0, 299, 127, 128]), (5, 700, [0, 600, 123, 695]),
                                             (64, 513, [449, 64, 63]), (200, 1000, [0, 1, 800]), (700, 700, [0])])
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_attention_weights(amk, nq, nkv, hd, rows, slots, lens, cache):
    g = gen(rows * 7 + nq)
    q = randn(g, len(lens), rows, nq, hd)
    k = randn(g, len(lens), nkv, slots, hd)
    k = code(k) if cache == "fp8" else k
    scale = hd ** -0.5
    lse = true_lse(q, k, lens, scale)
    before = torch.rand(len(lens), nkv, slots, generator=g, device=DEV)
    for b, decay in ((None, 1.0), (before, 0.75)):
        want, tol = weights64(q, k, lse, lens, b, decay, scale)
        got = amk.amk_attention_weights(q, k, lse, i32(lens), b, decay)
        weights_agree(got, want, tol)
    assert torch.equal(got, amk.amk_attention_weights(q, k, lse, i32(lens), before, 0.75))     # the same bits
    # the attention's own numbers: a row's weights add up to 1
    if b is None:
        assert float((got.sum() / (len(lens) * rows * nq) - 1).abs()) < 1e-4
    again = before.clone()
    assert amk.amk_attention_weights(q, k, lse, i32(lens), again, 0.75, out=again) is again and torch.equal(again, got)


def test_attention_weights_with_the_attentions_lse(amk):
    """A whole prompt, and a draft's worth of tokens over a cache: every row's weights add up to one."""
    g = gen(3)
    q, k, v = randn(g, 300, 8, 64), randn(g, 300, 2, 64), randn(g, 300, 2, 64)
    lse = torch.empty(300, 8, device=DEV)
    amk.amk_prompt_attention(q, k, v, i32([0, 300]), lse=lse)
    w = amk.amk_attention_weights(q[None], k.transpose(0, 1)[None], lse[None], i32([0]))
    # 300 * 4 rows for each kv head; each row's sum is off by its lse (2^-20 (1 + |lse|) and n 2^-24) and the scores (hd 2^-23 |q||k|)
    assert bool(((w.sum(2) / 1200 - 1).abs() < 1e-3).all())
    kc, vc = randn(g, 2, 2, 500, 64), randn(g, 2, 2, 500, 64)
    q, n = randn(g, 2, 7, 8, 64), i32([400, 20])
    lse = torch.empty(2, 7, 8, device=DEV)
    amk.amk_tree_attention(q, kc, vc, n, lse=lse)
    w = amk.amk_attention_weights(q, kc, lse, n)
    assert bool(((w.sum(2) / 28 - 1).abs() < 1e-3).all())
    assert not bool(w[0, :, 407:].any()) and not bool(w[1, :, 27:].any())


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("rows", [3, 150])
def test_attention_weights_broken_and_left_out(amk, rows, cache):
    """Impossible lengths, left-out tokens with broken queries, NaN in what nobody attends to, strides, other streams."""
    g = gen(rows)
    nq, nkv, hd, slots, lens = 4, 2, 64, 400, [100, -1, 250 - 0, 400, 0]
    q = randn(g, len(lens), nq, rows, hd).transpose(1, 2)
    kb = randn(g, len(lens), slots, nkv, hd)
    lse = true_lse(q, kb.transpose(1, 2), lens, 0.2)
    lse[0, 1], lse[2, 0, 2], lse[4, rows - 1] = -math.inf, math.inf, -math.inf
    q[0, 1, :, 3], q[4, rows - 1] = math.nan, math.inf
    kb[0, 100 + rows:], kb[2, 250 + rows:] = math.nan, math.inf          # behind the last row
    kb[2, 5, 1, 9] = math.nan                                              # one position of one head
    k = code(kb) if cache == "fp8" else kb
    k = k.transpose(1, 2)
    want, tol = weights64(q, k, lse, lens, None, 1, float(np.float32(0.2)))
    out = torch.full((len(lens), nkv, slots + 9), 7.0, device=DEV)
    got = amk.amk_attention_weights(q, k, lse, i32(lens), scale=0.2, out=out[:, :, :slots])
    assert bool(torch.isnan(want[2, 1, 5])) and int(torch.isnan(want[2]).sum()) == 1
    weights_agree(got, want, tol)
    assert bool((out[:, :, slots:] == 7).all())
    lse[4, 0, 0] = math.nan                                                # NaN reaches what the row attends to: slot 0
    got = amk.amk_attention_weights(q, k, lse, i32(lens), scale=0.2)
    assert bool(torch.isnan(got[4, 0, 0])) and int(torch.isnan(got[4]).sum()) == 1


def test_attention_weights_large_scores(amk):
    """Scores and log-sum-exps far from zero: the difference is what counts."""
    g = gen(4)
    q, k = randn(g, 1, 9, 2, 64) * 30, randn(g, 1, 1, 200, 64) * 30
    lse = true_lse(q, k, [191], 0.125)
    assert float(lse.abs().max()) > 1000
    want, tol = weights64(q, k, lse, [191], None, 1, 0.125)
    weights_agree(amk.amk_attention_weights(q, k, lse, i32([191])), want, tol)


# ---- choice of what stays ---------------------------------------------------------------------------------------

def evict_plain(scores, lens, budget, first, recent):
    seqs, heads, slots = scores.shape
    keep = np.full((seqs, heads, budget), -1, np.int32)
    count = np.zeros((seqs, heads), np.int32)
    moved = np.zeros(scores.shape, np.float32)
    for s, n in enumerate(lens):
        for h in range(heads):
            if n < 0 or n > slots:
                count[s, h], moved[s, h] = -1, scores[s, h]
                continue
            x = scores[s, h, :n]
            rank = sorted(range(n), key=lambda i: (not (i < first or i >= n - recent), bool(np.isnan(x[i])),
                                                   0.0 if np.isnan(x[i]) else -float(x[i]), i))
            rows = sorted(rank[:budget])
            count[s, h] = len(rows)
            keep[s, h, :len(rows)], moved[s, h, :len(rows)] = rows, x[rows]
    return keep, count, moved


def same_bits(a, b):
    return np.array_equal(np.ascontiguousarray(a).view(np.int32), np.ascontiguousarray(b).view(np.int32))


@pytest.mark.parametrize("slots,budget,first,recent", [(1, 1, 0, 0), (1, 1, 1, 0), (33, 32, 3, 5), (300, 1, 0, 1), (300, 7, 0, 0),
                                                       (300, 100, 100, 0), (300, 100, 40, 60), (2048, 512, 4, 64), (5000, 5000, 9, 9),
                                                       (5000, 4999, 0, 0), (49153, 1000, 4, 100), (100001, 60000, 4, 256)])
@pytest.mark.parametrize("kind", ["normal", "few", "odd"])
def test_evict_select(amk, slots, budget, first, recent, kind):
    rng = np.random.default_rng(slots + budget)
    lens = [slots, max(0, slots - 1), slots // 2, budget, min(budget + 1, slots), 0]
    lens = lens[:2] if slots > 40000 else lens
    shape = (len(lens), 2, slots)
    x = rng.standard_normal(shape).astype(np.float32)
    if kind == "few":                                     # many equal ones
        x = np.floor(np.abs(x) * 1.5).astype(np.float32)
    if kind == "odd":
        x = rng.choice(np.array([0.0, -0.0, np.inf, -np.inf, np.nan, -np.nan, 1e-45, -1e-45, 3e38, 1.0, -1.0], np.float32), shape)
    scores = torch.from_numpy(x).to(DEV)
    keep, count, moved = amk.amk_evict_select(scores, i32(lens), budget, first, recent)
    k, c, m = evict_plain(x, lens, budget, first, recent)
    assert np.array_equal(count.cpu().numpy(), c) and np.array_equal(keep.cpu().numpy(), k)
    assert same_bits(moved.cpu().numpy(), m) and same_bits(scores.cpu().numpy(), x)
    again = amk.amk_evict_select(scores, i32(lens), budget, first, recent, moved=scores)       # in place
    assert again[2] is scores and same_bits(scores.cpu().numpy(), m) and torch.equal(again[0], keep)


def test_evict_select_impossible_lengths_and_strides(amk):
    g = gen(2)
    wide = torch.rand(2, 5, 3, 120, generator=g, device=DEV).transpose(1, 2)[..., 3:103]       # [2][3][5][100] strided
    scores = wide[1].transpose(0, 1)                                                             # [5][3][100]
    lens = [100, -1, 101, 50, 2147483647]
    x = scores.cpu().numpy().copy()
    keep, count, moved = amk.amk_evict_select(scores, i32(lens), 20, 2, 3)
    k, c, m = evict_plain(x, lens, 20, 2, 3)
    assert np.array_equal(count.cpu().numpy(), c) and np.array_equal(keep.cpu().numpy(), k) and same_bits(moved.cpu().numpy(), m)
    amk.amk_evict_select(scores, i32(lens), 20, 2, 3, moved=scores)
    assert same_bits(scores.cpu().numpy(), m)
    assert amk.amk_evict_select(scores[:0], i32([]), 20)[0].shape == (0, 3, 20)


# ---- verification -----------------------------------------------------------------------------------------------

def verify_plain(logits, tokens, u, parents, draft, temperature, length):
    """The definition, sequence by sequence, in 64 bits."""
    seqs, rows, vocab = logits.shape
    logits = logits.double().cpu().numpy()
    draft = None if draft is None else draft.double().cpu().numpy()
    tokens, u = tokens.tolist(), u.double().cpu().numpy()
    count, keep, chosen = [], np.full((seqs, rows), -1), []

    def target(x, t):
        if not (0 <= t < math.inf) or np.isnan(x).any() or not np.isfinite(x.max()):
            return None
        if t == 0:
            p = np.zeros(len(x))
            p[int(x.argmax())] = 1
            return p
        e = np.exp((x - x.max()) / t)
        return e / e.sum()

    for s in range(seqs):
        t = 1.0 if temperature is None else float(temperature[s])
        base = 0 if length is None else int(length[s])
        node, path = 0, [0]
        while True:
            p = target(logits[s, node], t)
            found = None
            for c in range(node + 1, rows) if p is not None else ():
                parent = c - 1 if parents is None else int(parents[s, c])
                tok = tokens[s][c]
                if parent != node or not 0 <= tok < vocab:
                    continue
                q = np.zeros(vocab) if draft is None else draft[s, node]
                if draft is None:
                    q[tok] = 1
                if u[s, c] * q[tok] < p[tok]:
                    found = c
                    break
                rest = np.maximum(p - q, 0)
                if rest.sum() > 0:
                    p = rest / rest.sum()
            if found is None:
                break
            node = found
            path.append(node)
        count.append(len(path))
        keep[s, :len(path)] = np.array(path) + base
        if p is None:
            chosen.append(-1)
        else:
            sums = np.cumsum(p)
            over = np.nonzero(sums > u[s, 0] * sums[-1])[0]
            chosen.append(int(over[0]) if len(over) else int(np.nonzero(p > 0)[0][-1]))
    return count, keep, chosen


def verified(amk, logits, tokens, u, parents=None, draft=None, temperature=None, length=None):
    got = amk.amk_verify_draft(logits, tokens, u, parents, draft, temperature, length)
    want = verify_plain(logits, tokens, u, parents, draft, temperature, length)
    assert got[0].tolist() == want[0]
    assert got[1].tolist() == want[1].tolist()
    assert got[2].tolist() == want[2]
    return got


def draft_case(g, seqs, rows, vocab, dtype, kind, tree, near=0.4, temperature=1.0):
    x = randn(g, seqs, rows, vocab, dtype=torch.float32) * 2.5
    likely = torch.randint(0, vocab, (seqs, rows, 1), generator=g, device=DEV)
    x.scatter_(2, likely, torch.logsumexp(x, 2, keepdim=True) + 0.3)
    rng = np.random.default_rng(seqs * 1000 + rows * 10 + vocab)
    parents = np.array([[-1] + [int(rng.integers(max(0, i - 4), i)) if tree else i - 1 for i in range(1, rows)] for _ in range(seqs)])
    above = torch.from_numpy(parents.clip(0)).to(DEV)
    probs = None
    if kind == "probs":
        probs = torch.softmax((x + near * randn(g, seqs, rows, vocab, dtype=torch.float32)) / temperature, 2)
        drawn = torch.multinomial(probs.view(-1, vocab), rows, replacement=True, generator=g).view(seqs, rows, rows)
        tokens = drawn[torch.arange(seqs, device=DEV)[:, None], above, torch.arange(rows, device=DEV)[None]]
    else:
        right = torch.rand(seqs, rows, generator=g, device=DEV) < 0.5
        tokens = torch.where(right, torch.gather(likely[..., 0], 1, above), torch.randint(0, vocab, (seqs, rows), generator=g, device=DEV))
    u = torch.rand(seqs, rows, generator=g, device=DEV)
    return x.to(dtype), tokens.to(torch.int32), u, i32(parents.tolist()) if tree else None, probs


@pytest.mark.parametrize("seqs,rows,vocab", [(1, 1, 1), (3, 4, 2), (2, 6, 500), (40, 9, 1001), (9, 30, 777), (1, 5, 32000), (4, 5, 50001),
                                             (2, 3, 128256), (1, 2, 300007), (150, 3, 4096)])
@pytest.mark.parametrize("kind", ["probs", "point"])
@pytest.mark.parametrize("tree", [False, True])
def test_verify_draft(amk, seqs, rows, vocab, kind, tree):
    g = gen(seqs * 77 + rows + vocab)
    dtype = torch.float32 if (rows + vocab) % 2 else torch.bfloat16
    logits, tokens, u, parents, probs = draft_case(g, seqs, rows, vocab, dtype, kind, tree)
    temperature = torch.tensor([1.0, 0.7, 0.0, 1.5], device=DEV).repeat(seqs)[:seqs].contiguous()
    verified(amk, logits, tokens, u, parents, probs, temperature, i32(list(range(100, 100 + seqs))))
    verified(amk, logits, tokens, u, parents, probs)


def test_verify_draft_many_rejections(amk):
    """Drafts that are mostly wrong: several rejected children of a node, the same token twice among them."""
    for seed in range(6):
        g = gen(seed)
        for kind in ("probs", "point"):
            logits, tokens, u, _, probs = draft_case(g, 12, 20, 40, torch.float32, kind, False, near=2.0)
            parents = torch.randint(0, 3, (12, 20), generator=g, device=DEV).to(torch.int32)
            tokens[:, 5] = tokens[:, 4]
            logits = (logits - logits.amax(2, keepdim=True)) * 0.3         # nothing is likely
            verified(amk, logits, tokens, u, parents, probs)


def test_verify_draft_odd_inputs(amk):
    """Tokens out of range, parents that are none, masked logits, rows without a distribution, temperatures that are none, numbers
    at the ends of [0, 1), strides and alignments."""
    g = gen(11)
    logits, tokens, u, parents, probs = draft_case(g, 8, 7, 333, torch.float32, "point", True)
    tokens[0, 1], tokens[1, 2], tokens[2, 3] = -1, 333, 1 << 30
    parents[3, 2], parents[3, 3], parents[4, 4], parents[5, 1] = 2, 6, -7, 1 << 30
    logits[0, :, 5:] = -math.inf
    logits[1, :, 1:] = -math.inf                                            # one token has all
    logits[2, 1, 7] = math.nan
    logits[6, 0] = -math.inf
    logits[7, 0, 3] = math.inf
    verified(amk, logits, tokens, u, parents)
    verified(amk, logits, tokens, u, parents, temperature=torch.tensor([0.0, 0.0, 0.0, math.nan, -1.0, math.inf, 0.0, 1e-30], device=DEV))
    for end in (0.0, 1.0 - 2.0 ** -24):
        verified(amk, logits, tokens, torch.full_like(u, end), parents)
    # bf16, every alignment of the rows
    for skew in range(9):
        wide = torch.zeros(2, 4, 700 + skew, dtype=torch.bfloat16, device=DEV)
        x, t, u2, _, probs = draft_case(gen(skew), 2, 4, 501, torch.bfloat16, "probs", False)
        wide[:, :, skew:skew + 501] = x
        pw = torch.zeros(4, 2, 509, device=DEV).transpose(0, 1)
        pw[:, :, 3:504] = probs
        verified(amk, wide[:, :, skew:skew + 501], t, u2, draft=pw[:, :, 3:504])
    assert [t.shape[0] for t in amk.amk_verify_draft(logits[:0], tokens[:0], u[:0])] == [0, 0, 0]


@pytest.mark.parametrize("kind", ["probs", "point"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_verify_draft_temperatures_beyond_32_bits(amk, kind, dtype):
    """Logits and temperatures so large that differences of logits overflow fp32, and so small that 1 / T does."""
    for size in (1e38, 1e37, 1e31, 1e-36, 1e-38, 1e-39):
        for seed in range(4):
            x, tokens, u, parents, probs = draft_case(gen(40 + seed), 12, 8, 300, torch.float32, kind, seed % 2 == 0)
            logits = (x.clamp(-3, 3) * size).to(dtype)
            verified(amk, logits, tokens, u, parents, probs, torch.full((12,), size, device=DEV))


def test_verify_draft_same_distribution_accepts_all(amk):
    """A draft with the target's own probabilities: u q < p holds for every u below 1, so that everything is accepted; and with
    probabilities next to each other the answer is that of 64 bits."""
    g = gen(21)
    x = randn(g, 6, 8, 5000, dtype=torch.float32)
    probs = torch.softmax(x.double(), 2).float()
    tokens = torch.multinomial(probs.view(-1, 5000), 8, replacement=True, generator=g).view(6, 8, 8)[:, :, 0].to(torch.int32)
    tokens[:, 1:] = tokens[:, :-1].clone()                                  # node i's token comes from row i - 1
    u = torch.full((6, 8), 1.0 - 2.0 ** -24, device=DEV)
    u[:, 0] = 0.5
    assert verified(amk, x, tokens, u, draft=probs)[0].tolist()[0] >= 1
    u[:, 1:] = 0.999
    assert verified(amk, x, tokens, u, draft=probs)[0].tolist() == [8] * 6


@pytest.mark.parametrize("kind", ["probs", "point"])
def test_verify_draft_keeps_the_targets_distribution(amk, kind):
    """The first token behind node 0, accepted or drawn, is distributed as the target says, whatever the draft: 60000 draws of
    12 tokens, each count within six standard deviations."""
    g = gen(5)
    n, vocab = 60000, 12
    row = randn(g, vocab, dtype=torch.float32)
    p = torch.softmax(row.double(), 0)
    q = torch.softmax(randn(g, vocab, dtype=torch.float32), 0)
    logits = row.expand(n, 4, vocab).contiguous()
    tokens = torch.multinomial(q, 4 * n, replacement=True, generator=g).view(n, 4).to(torch.int32)
    parents = torch.zeros(n, 4, dtype=torch.int32, device=DEV)              # three children of node 0
    u = torch.rand(n, 4, generator=g, device=DEV)
    draft = q.expand(n, 4, vocab).contiguous() if kind == "probs" else None
    count, keep, token = amk.amk_verify_draft(logits, tokens, u, parents, draft)
    first = torch.where(count > 1, tokens.gather(1, keep[:, 1:2].clamp(min=0).long())[:, 0], token)
    seen = torch.bincount(first.long(), minlength=vocab).double()
    assert bool(((seen - n * p).abs() <= 6 * torch.sqrt(n * p * (1 - p))).all())


# ---- together ---------------------------------------------------------------------------------------------------

def test_streams_graphs_and_order(amk):
    """The operators in a row on another stream, captured into a graph and replayed on new inputs: each waits for the one before."""
    g = gen(9)
    rows, nq, nkv, hd, slots, vocab = 6, 8, 2, 64, 640, 3001
    x = randn(g, rows, nq + 2 * nkv, hd)
    pos, where = torch.arange(500, 506, device=DEV, dtype=torch.int32), torch.arange(500, 506, device=DEV)
    kc, vc = randn(g, 1, nkv, slots, hd), randn(g, 1, nkv, slots, hd)
    lse, n = torch.empty(1, rows, nq, device=DEV), i32([500])
    before = torch.rand(1, nkv, slots, generator=g, device=DEV)
    logits, tokens, u, _, probs = draft_case(g, 1, rows, vocab, torch.float32, "probs", False)
    kept = i32([506])

    def all_of_them():
        q = amk.amk_norm_rope_append(x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:], pos, kc, vc, where, theta=1e4)
        out = amk.amk_tree_attention(q[None], kc, vc, n, lse=lse)
        w = amk.amk_attention_weights(q[None], kc, lse, n, before, 0.9)
        return (q, out, w, *amk.amk_evict_select(w, kept, 100, 4, 16), *amk.amk_verify_draft(logits, tokens, u, draft=probs))

    eager = [t.clone() for t in all_of_them()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        on_side = all_of_them()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, on_side))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = all_of_them()
    fresh = randn(g, rows, nq + 2 * nkv, hd)
    x.copy_(fresh)
    u.fill_(0.999)
    graph.replay()
    torch.cuda.synchronize()
    replayed = [t.clone() for t in captured]
    again = all_of_them()
    assert all(torch.equal(a, b) for a, b in zip(replayed, again)) and not torch.equal(replayed[0], eager[0])


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("nq,nkv,hd,rows,slots,seqs", [(7, 1, 128, 2500, 3600, 2), (8, 2, 64, 3, 260, 40), (4, 1, 64, 90, 330, 40), (12, 4, 128, 43, 500, 70)])
def test_attention_weights_long_and_many(amk, nq, nkv, hd, rows, slots, seqs, cache):
    """Many tiles of queries, units cut between blocks; more sequences than a warp looks at once, some of impossible length."""
    g = gen(rows + seqs)
    q, k = randn(g, seqs, rows, nq, hd), randn(g, seqs, nkv, slots, hd)
    k = code(k) if cache == "fp8" else k
    rng = np.random.default_rng(rows)
    lens = [int(x) for x in rng.integers(0, slots - rows + 1, seqs)]
    if seqs > 2:
        lens[1], lens[5], lens[-1] = -3, slots, 0
    lse = true_lse(q, k, lens, hd ** -0.5)
    want, tol = weights64(q, k, lse, lens, None, 1, hd ** -0.5)
    got = amk.amk_attention_weights(q, k, lse, i32(lens))
    weights_agree(got, want, tol)
    assert torch.equal(torch.nan_to_num(got, 7.0), torch.nan_to_num(amk.amk_attention_weights(q, k, lse, i32(lens)), 7.0))


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("rows,tiles", [(3, 0), (3, 1), (200, 0), (200, 1)])
def test_attention_weights_expired_wait(amk, rows, tiles, cache):
    """Tiles that never come: the waits run out, the status says so once, and the next call is right."""
    g = gen(1)
    q, k, lens = randn(g, 2, rows, 8, 128), randn(g, 2, 1, 1500, 128), [1300, 900]
    k = code(k) if cache == "fp8" else k
    lse = true_lse(q, k, lens, 128 ** -0.5)
    q, k, lse = (t.repeat(24, *[1] * (t.dim() - 1)) for t in (q, k, lse))     # several units for each block
    lens = lens * 24
    call = lambda: amk.amk_attention_weights(q, k, lse, i32(lens))
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


def test_first_calls_of_a_process_may_be_captured():
    """Everything that a call sets up once happens in the call itself, and capture allows it."""
    code_ = """
import torch
from paper_2606_09682_b200 import binding as amk
g = torch.Generator(device="cuda").manual_seed(1)
r = lambda *s: torch.randn(*s, device="cuda", generator=g)
x, pos = r(6, 8, 64).bfloat16(), torch.arange(6, device="cuda", dtype=torch.int32)
kc, vc, n = r(1, 2, 700, 64).bfloat16(), r(1, 2, 700, 64).bfloat16(), torch.full((1,), 500, dtype=torch.int32, device="cuda")
q2, lse2 = r(1, 150, 4, 64).bfloat16(), r(1, 150, 4) + 9
lse, logits, tok, u = r(1, 6, 4) + 9, r(1, 6, 9000), torch.zeros(1, 6, dtype=torch.int32, device="cuda"), torch.rand(1, 6, device="cuda", generator=g)
sc = r(2, 3, 40000).abs()
two = torch.full((2,), 39999, dtype=torch.int32, device="cuda")
def run():
    q = amk.amk_norm_rope_append(x[:, :4], x[:, 4:6], x[:, 6:], pos, kc, vc, pos.long() + 500)
    return [q, amk.amk_attention_weights(q[None], kc, lse, n), amk.amk_attention_weights(q2, kc, lse2, n), *amk.amk_evict_select(sc, two, 90, 2, 3),
            *amk.amk_evict_select(sc[:, :, :30000], two - 10000, 20000), *amk.amk_verify_draft(logits, tok, u)]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    a = run()
graph.replay()
assert all(torch.equal(b, c) for b, c in zip(a, run())) and amk.amk_operator_status() == 0
print("fine")
"""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code_], capture_output=True, text=True, timeout=300, cwd=root)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]


def test_scratch_of_two_graphs(amk):
    """Two captured calls with a workspace each, replayed on two streams at once, again and again."""
    g = gen(12)
    q, k = randn(g, 2, 300, 8, 64), randn(g, 2, 2, 900, 64)
    lens = [[500, 31], [0, 600]]
    lse = [true_lse(q, k, n, 0.125) for n in lens]
    logits, tokens, u, _, probs = draft_case(g, 3, 6, 20000, torch.float32, "probs", False)
    want, graphs, streams, outs = [], [], [], []
    for i in range(2):
        n, uu = i32(lens[i]), u if i else (1 - u) * 0.999
        want.append([amk.amk_attention_weights(q, k, lse[i], n), *amk.amk_verify_draft(logits, tokens, uu, draft=probs)])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append([amk.amk_attention_weights(q, k, lse[i], n), *amk.amk_verify_draft(logits, tokens, uu, draft=probs)])
        graphs.append((graph, n, uu))
        streams.append(torch.cuda.Stream())
    for _ in range(20):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph[0].replay()
    torch.cuda.synchronize()
    for a, b in zip(want, outs):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


# ---- with the decode step ---------------------------------------------------------------------------------------

def layers(shape, w, tokens, attend):
    """The model in plain fp32 torch around ``attend(layer, q, k, v)``: q, k, v bf16 [tokens][heads][hd], not rotated yet."""
    f = lambda t: t.float()
    norm = lambda x, g: x * torch.rsqrt((x * x).mean(-1, keepdim=True) + shape.rms_eps) * f(g)
    x = f(w["embed"])[tokens.long()]
    n = len(tokens)
    for l in range(shape.n_layers):
        h = norm(x, w["attn_norm"][l])
        q, k, v = ((h @ f(w[m][l]).t()).view(n, -1, shape.head_dim).to(torch.bfloat16) for m in ("wq", "wk", "wv"))
        x = x + attend(l, q, k, v).float().reshape(n, -1) @ f(w["wo"][l]).t()
        h = norm(x, w["mlp_norm"][l])
        x = x + (torch.nn.functional.silu(h @ f(w["wgate"][l]).t()) * (h @ f(w["wup"][l]).t())) @ f(w["wdown"][l]).t()
    return norm(x, w["final_norm"]) @ f(w["embed"] if shape.tied else w["lm_head"]).t()


@pytest.mark.parametrize("name,kv_dtype", [("mini", "bf16"), ("mini_hd128", "bf16"), ("mini_ragged", "bf16"), ("mini", "fp8")])
def test_prompt_draft_verify_evict_and_decode(amk, name, kv_dtype):
    """A prompt rotated and stored in a decoder's cache, a draft chain verified over it, the accepted tokens kept and the decode step
    going on; then the positions with the least attention weight leave, and the tree attention goes on over what stays.
    4e-2 for logits: q, k and v rounded to bf16 before the rotation and after it, the attention's output once (2^-8 each),
    through the layers; 4.4e-2 more for the 8-bit cache, whose entries may fall on the other side of a border (a step of 2^-3
    for 2^-3 of them)."""
    shape = inp.SHAPES[name]
    w = inp.make_weights(shape, 99, device=DEV, std=0.05, norm_jitter=0.1)
    dec = amk.Decoder(shape, w, "bf16", kv_dtype=kv_dtype)
    nkv, hd = shape.n_kv_heads, shape.head_dim
    n, n_new = 37, 9
    prompt = torch.randint(0, shape.vocab, (n,), generator=gen(3), device=DEV)
    kv_ref, toks, logits_ref = dec.new_cache(), prompt.tolist(), []
    for pos in range(n + n_new):
        dec.amk_decode_step(toks[pos], pos, kv_ref)
        assert dec.amk_last_status()[0] == 0
        logits_ref.append(dec.logits.clone())
        if pos + 1 >= len(toks):
            toks.append(int(dec.next_token))
    kv = dec.new_cache()
    K, V = dec.cache_views(kv)
    bf16 = lambda t: t.contiguous().view(torch.float8_e4m3fn).to(torch.bfloat16) if t.dtype == torch.uint8 else t
    near = lambda a, b: float((a - b).norm() / b.norm())
    tol = 4e-2 + (4.4e-2 if kv_dtype == "fp8" else 0.0)

    # the prompt
    at = torch.arange(n, device=DEV)
    cu = i32([0, n])
    sums = torch.zeros(shape.n_layers, nkv, shape.max_seq, device=DEV)       # attention weights of every layer's positions

    def prompt_layer(l, q, k, v):
        q = amk.amk_norm_rope_append(q, k, v, at.to(torch.int32), K[l][None], V[l][None], at, theta=shape.rope_theta)
        lse = torch.empty(n, shape.n_q_heads, device=DEV)
        out = amk.amk_prompt_attention(q, bf16(K[l])[:, :n].transpose(0, 1), bf16(V[l])[:, :n].transpose(0, 1), cu, lse=lse)
        amk.amk_attention_weights(q[None], K[l][None], lse[None], i32([0]), out=sums[l][None])
        return out

    logits = layers(shape, w, prompt, prompt_layer)
    assert near(logits[-1], logits_ref[n - 1]) < tol
    assert bool(((sums.sum(2) / (n * shape.n_q_heads / nkv) - 1).abs() < 1e-3).all())

    # a chain: the token that the prompt ends in (true[0] is already chosen), three true ones and a wrong one
    true = toks[n:n + n_new]
    draft = true[:4] + [(true[4] + 1) % shape.vocab, true[5]]
    rows, length = len(draft), i32([n])
    where = n + torch.arange(rows, device=DEV)

    def draft_layer(l, q, k, v):
        q = amk.amk_norm_rope_append(q, k, v, where.to(torch.int32), K[l][None], V[l][None], where, theta=shape.rope_theta)
        lse = torch.empty(1, rows, shape.n_q_heads, device=DEV)
        out = amk.amk_tree_attention(q[None], K[l][None], V[l][None], length, lse=lse)[0]
        drafted.append((q, lse))
        return out

    drafted = []
    logits = layers(shape, w, torch.tensor(draft, device=DEV), draft_layer)
    for i in range(4):
        assert near(logits[i], logits_ref[n + i]) < tol, i
    count, keep, token = amk.amk_verify_draft(logits[None].contiguous(), i32([draft]), torch.rand(1, rows, device=DEV), cache_len=length,
                                              temperature=torch.zeros(1, device=DEV))
    best = logits.argmax(1).tolist()
    kept = 1
    while kept < rows and draft[kept] == best[kept - 1]:
        kept += 1
    assert count.tolist() == [kept] and keep.tolist() == [[n + i if i < kept else -1 for i in range(rows)]] and token.tolist() == [best[kept - 1]]
    assert kept == 4                                     # (what the decode step itself chose)
    # the accepted tokens' weights count, the others' are left out
    for l, (q, lse) in enumerate(drafted):
        lse[0, kept:] = -math.inf
        amk.amk_attention_weights(q[None], K[l][None], lse, length, sums[l][None], out=sums[l][None])
    total = n * shape.n_q_heads / nkv + kept * shape.n_q_heads / nkv
    assert bool(((sums.sum(2) / total - 1).abs() < 1e-3).all())
    dec.amk_kv_compact(kv, length, keep, count)
    for pos in range(n + kept, n + n_new):
        dec.amk_decode_step(toks[pos], pos, kv)
        assert near(dec.logits, logits_ref[pos]) < tol, pos

    # a budget for every layer and head; the rows behind the kept ones are free again
    have, budget = n + kept, 20
    before = (bf16(K).double(), bf16(V).double())
    lens = i32([have] * shape.n_layers)
    keep, count, moved = amk.amk_evict_select(sums, lens, budget, 2, 5)
    assert count.unique().tolist() == [budget]
    lists, counts = keep.view(-1, budget), count.view(-1)
    for half in (K, V):
        amk.amk_kv_compact(half.view(shape.n_layers * nkv, 1, shape.max_seq, hd), torch.zeros_like(counts), lists, counts)
    assert torch.equal(moved[:, :, :budget], torch.gather(sums, 2, keep.long()))
    old = [torch.gather(b, 2, keep.long()[..., None].expand(-1, -1, -1, hd)) for b in before]
    for half, want in zip((K, V), old):
        assert torch.equal(bf16(half[:, :, :budget]).double(), want)
    new = torch.tensor([have], device=DEV)
    slot = i32([budget])

    def tree(l, q, k, v):
        q = amk.amk_norm_rope_append(q, k, v, new.to(torch.int32), K[l][None], V[l][None], torch.full((1,), budget, device=DEV), theta=shape.rope_theta)
        return amk.amk_tree_attention(q[None], K[l][None], V[l][None], slot)[0]

    def plain(l, q, k, v):
        qr, kr = rotated64(q, None, new, shape.rope_theta, 0)[0], rotated64(k, None, new, shape.rope_theta, 0)[0]
        rep = shape.n_q_heads // nkv
        keys, values = (torch.cat([o[l], t.double().transpose(0, 1)], 1).repeat_interleave(rep, 0) for o, t in zip(old, (kr, v)))
        x = qr.permute(1, 0, 2) @ keys.transpose(1, 2) * hd ** -0.5
        return (torch.softmax(x, 2) @ values).permute(1, 0, 2).to(torch.bfloat16)

    token = torch.tensor([toks[have]], device=DEV)
    got, want = layers(shape, w, token, tree), layers(shape, w, token, plain)
    assert near(got, want) < (2e-2 if kv_dtype == "bf16" else 6.4e-2)
    dec.close()


def test_refused(amk):
    """What the Python layer and the library refuse, with the reason; a CPU tensor among CUDA ones too."""
    x, pos = torch.zeros(4, 8, 64, dtype=torch.bfloat16, device=DEV), i32([0, 1, 2, 3])
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    kc = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16, device=DEV)
    where = torch.arange(4, device=DEV)
    rope, weights, evict, verify = amk.amk_norm_rope_append, amk.amk_attention_weights, amk.amk_evict_select, amk.amk_verify_draft
    q4, lse, n = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(1, 2, 4, device=DEV), i32([0])
    sc, logits, tok, u = torch.zeros(1, 2, 8, device=DEV), torch.zeros(1, 2, 10, device=DEV), i32([[0, 0]]), torch.zeros(1, 2, device=DEV)
    calls = [lambda: rope(q.float(), k, v, pos), lambda: rope(q, k[:3], v, pos), lambda: rope(q, k, v, pos.long()),
             lambda: rope(q, k, v, pos, kc, None, where), lambda: rope(q, k, None, pos, kc, kc.clone(), where),
             lambda: rope(q, k, v, pos, kc, kc.clone(), where.to(torch.int32)), lambda: rope(q, k, v, pos, kc, kc.clone()[:, :1], where),
             lambda: rope(q, k, v, pos, kc, kc.float(), where), lambda: rope(q, k, v, pos, q_weight=torch.ones(64, device=DEV)),
             lambda: rope(q, k, v, pos, eps=-1.0), lambda: rope(q, k, v, pos, eps=math.nan), lambda: rope(q, k, v, pos, theta=0.0),
             lambda: rope(q, k, v, pos, theta=1e300), lambda: rope(q[:, :, :32], k[:, :, :32], None, pos),
             lambda: rope(x.flatten()[4:4 + 1024].view(4, 4, 64), k, v, pos), lambda: rope(q, k, v, pos.cpu()),
             lambda: rope(q, k, v, pos, q_out=q.clone()[:, :3]), lambda: rope(q.transpose(1, 2), k, v, pos),
             lambda: weights(q4.float(), kc, lse, n), lambda: weights(q4, kc, lse[:, :1], n), lambda: weights(q4, kc, lse, n.long()),
             lambda: weights(q4, kc, lse, n, scale=-1.0), lambda: weights(q4, kc, lse, n, decay=math.inf),
             lambda: weights(q4, kc, lse, n, before=sc[:, :1]), lambda: weights(q4, kc[:, :, :1], lse, n),
             lambda: weights(q4, kc.expand(1, 2, 8, 64)[..., ::1].repeat(1, 2, 1, 1)[:, :3], lse, n), lambda: weights(q4.cpu(), kc, lse, n),
             lambda: evict(sc, n, 0), lambda: evict(sc, n, 9), lambda: evict(sc, n, 4, 3, 2), lambda: evict(sc, n, 4, -1, 2),
             lambda: evict(sc.double(), n, 4), lambda: evict(sc, n.long(), 4), lambda: evict(sc[:, :, ::2], n, 4),
             lambda: verify(logits.half(), tok, u), lambda: verify(logits, tok.long(), u), lambda: verify(logits, tok, u.double()),
             lambda: verify(logits, tok, u, parents=tok[:, :1]), lambda: verify(logits, tok, u, draft=logits.bfloat16()),
             lambda: verify(logits, tok, u, temperature=u), lambda: verify(logits, tok, u, workspace=torch.empty(4, dtype=torch.uint8, device=DEV)),
             lambda: verify(torch.zeros(1, 1025, 4, device=DEV), torch.zeros(1, 1025, dtype=torch.int32, device=DEV), torch.zeros(1, 1025, device=DEV)),
             lambda: weights(q4.requires_grad_(), kc, lse, n)]
    for i, call in enumerate(calls):
        with pytest.raises(amk.AmkError):
            call()
            raise AssertionError(f"call {i} was not refused")
    torch.cuda.synchronize()
