"""GPU tests of the operators between projection, attention and cache at the ends of what their calls allow, against the same plain
implementations in 64 bits and with the same tolerances as test_more_operators_gpu.py."""
import math

import numpy as np
import pytest
import torch

from test_more_operators_gpu import (DEV, code, draft_case, evict_plain, gen, i32, near16, randn, rotated64, same_bits, true_lse,
                                     verified, weights64, weights_agree)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amk():
    from paper_2606_09682_b200 import binding
    return binding


# ---- norm, rotation, storing ------------------------------------------------------------------------------------

@pytest.mark.parametrize("hd", [64, 128])
def test_norm_rope_append_small_elements_of_heads_beyond_32_bits(amk, hd):
    """Heads whose squares are beyond fp32, with elements so much smaller that the normed ones are barely normal bf16 numbers: those
    that are 2^-125 or more at position 0, and those whose rotated sums keep 2^-19 of themselves above bf16's least step elsewhere."""
    g = gen(hd)
    for position, least in ((0, -58), (777, -41)):
        for largest in (69, 100, 127):
            # rms: 2^largest / sqrt(hd), between 2^64 and 2^124
            x = (1 + torch.rand(4, 3, hd, generator=g, device=DEV)) * torch.pow(2.0, torch.randint(least, 60, (4, 3, hd), generator=g, device=DEV) + float(largest - 69))
            x[:, :, 5], x[:, :, 5 + hd // 2] = 2.0 ** largest, -(2.0 ** largest)
            x = x.to(torch.bfloat16)
            q, k = x[:, :2], x[:, 2:]
            w = (1 + 0.3 * torch.rand(hd, generator=g, device=DEV)).to(torch.bfloat16)
            pos = torch.full((4,), position, dtype=torch.int32, device=DEV)
            k_out = torch.empty_like(k)
            got = amk.amk_norm_rope_append(q, k, None, pos, q_weight=w, k_weight=w, k_out=k_out)
            for out, y in ((got, q), (k_out, k)):
                want, both = rotated64(y, w, pos, 10000.0, float(np.float32(1e-5)))
                near16(out, want, both)


# ---- attention weights ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("nq,nkv,hd,rows,slots", [(8, 2, 64, 300, 900), (16, 1, 128, 70, 700), (4, 2, 64, 3, 700)])
@pytest.mark.parametrize("bad", [-320, -1000, -20000000, -(1 << 31), 2147483647])
def test_attention_weights_impossible_lengths_among_others(amk, nq, nkv, hd, rows, slots, cache, bad):
    """A sequence of impossible length gets NaN, and the others their weights, wherever it stands."""
    g = gen(rows)
    for lens in ([bad, 500, 31], [500, bad, 0], [slots - rows, 31, bad], [bad, 77, bad, bad, 200, bad]):
        q, k = randn(g, len(lens), rows, nq, hd), randn(g, len(lens), nkv, slots, hd)
        k = code(k) if cache == "fp8" else k
        lse = true_lse(q, k, lens, hd ** -0.5)
        want, tol = weights64(q, k, lse, lens, None, 1, hd ** -0.5)
        # in the middle of a larger tensor: what lies around out stays as it is
        room = torch.full((len(lens) + 2, nkv, slots), 7.0, device=DEV)
        got = amk.amk_attention_weights(q, k, lse, i32(lens), out=room[1:-1])
        assert [bool(torch.isnan(got[s]).all()) for s in range(len(lens))] == [n == bad for n in lens]
        weights_agree(got, want, tol)
        assert bool((room[0] == 7).all()) and bool((room[-1] == 7).all())


@pytest.mark.parametrize("nq,nkv,hd", [(9, 3, 64), (32, 8, 128), (16, 1, 128), (7, 1, 128)])
@pytest.mark.parametrize("rows,slots,lens", [(1, 300, [0, 299, 127, 128]), (5, 700, [0, 600, 123, 695]), (200, 1000, [0, 1, 800]), (700, 700, [0])])
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_attention_weights_of_a_row_add_up_to_one(amk, nq, nkv, hd, rows, slots, lens, cache):
    """A row's weights add up to exp(its true log-sum-exp - the given one in 32 bits): to 1 within half a step of that, and what the
    positions may be off by."""
    g = gen(rows * 5 + nq)
    q, k = randn(g, len(lens), rows, nq, hd), randn(g, len(lens), nkv, slots, hd)
    k = code(k) if cache == "fp8" else k
    lse = true_lse(q, k, lens, hd ** -0.5)
    _, tol = weights64(q, k, lse, lens, None, 1, hd ** -0.5)
    n = rows * nq // nkv
    off = (amk.amk_attention_weights(q, k, lse, i32(lens)).double().sum(2) / n - 1).abs()
    allowed = tol.sum(2) / n + 1.01 * 2.0 ** -24 * lse.abs().amax((1, 2), keepdim=False)[:, None].double()
    assert bool((off <= allowed).all()) and float(allowed.max()) < 1e-3


# ---- choice of what stays ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("slots", [4096, 4097, 8192, 8193, 16384, 16385, 32767, 32768, 32769, 65536, 65537])
@pytest.mark.parametrize("kind", ["normal", "few", "odd", "same"])
def test_evict_select_at_the_kernels_limits(amk, slots, kind):
    """The largest and smallest lists of each kernel, at budgets that leave nearly all and nearly none, lists at odd addresses."""
    rng = np.random.default_rng(slots)
    shape = (2, 2, slots)
    x = rng.standard_normal(shape).astype(np.float32)
    if kind == "few":
        x = np.floor(np.abs(x) * 1.5).astype(np.float32)
    if kind == "odd":
        x = rng.choice(np.array([0.0, -0.0, np.inf, -np.inf, np.nan, -np.nan, 1e-45, -1e-45, 3e38, 1.0, -1.0], np.float32), shape)
    if kind == "same":
        x = np.full(shape, 0.125, np.float32)
    wide = torch.zeros(2, 2, slots + 3, device=DEV)
    wide[:, :, 1:-2] = torch.from_numpy(x).to(DEV)
    scores = wide[:, :, 1:-2]
    for budget, first, recent in ((1, 0, 0), (slots // 3, 4, 100), (slots - 1, 0, 0), (slots - 1, 5, slots - 10), (slots, 1, 2)):
        lens = [slots, slots - 1 if budget == slots // 3 else slots]
        k, c, m = evict_plain(x, lens, budget, first, recent)
        for s in (scores, scores.contiguous()):
            keep, count, moved = amk.amk_evict_select(s, i32(lens), budget, first, recent)
            assert np.array_equal(count.cpu().numpy(), c) and np.array_equal(keep.cpu().numpy(), k)
            assert same_bits(moved.cpu().numpy(), m) and same_bits(s.cpu().numpy(), x)
        assert amk.amk_evict_select(s, i32(lens), budget, first, recent, moved=s)[2] is s and same_bits(s.cpu().numpy(), m)
    assert not bool(wide[:, :, 0].any()) and not bool(wide[:, :, -2:].any())


# ---- verification -----------------------------------------------------------------------------------------------

def test_verify_draft_sums_of_many_parts(amk):
    """A vocabulary of 2^26 whose small probabilities come to 3e-5 of the row's sum, though any 2^17 of them in a row are less than
    half a step of it in 32 bits: a guess of the likely token is accepted up to its probability and no further."""
    vocab = 1 << 26
    logits = torch.full((1, 2, vocab), math.log(0.99) - 41 * math.log(2), device=DEV)
    logits[0, 0, 0] = 0.0
    logits[0, 1], logits[0, 1, 5] = -math.inf, 0.0
    tokens = i32([[0, 0]])
    rest = float(torch.exp(logits[0, 0, 1:].double()).sum())
    assert 2.9e-5 < rest < 3.1e-5
    for below in (2e-5, 2.8e-5, 3.2e-5, 4e-5):
        u = torch.tensor([[0.0, 1.0 - below]], device=DEV)                  # the draw: the first token with a probability
        accepted = float(u[0, 1].double()) < 1 / (1 + rest)
        assert accepted == (below > rest)
        count, keep, token = amk.amk_verify_draft(logits, tokens, u)
        assert (count.tolist(), keep.tolist(), token.tolist()) == (([2], [[0, 1]], [5]) if accepted else ([1], [[0, -1]], [1])), below


@pytest.mark.parametrize("kind", ["probs", "point"])
@pytest.mark.parametrize("seqs,rows,vocab", [(1, 6, 300007), (3, 5, 140001), (80, 4, 60011), (150, 5, 20000), (76, 4, 128256)])
def test_verify_draft_rejections_in_long_rows(amk, seqs, rows, vocab, kind):
    """Several rejected children of node 0 where a block's share of a row is more than its threads keep: the rest is read and
    rejected again for each of them."""
    g = gen(seqs + rows)
    logits, tokens, u, _, probs = draft_case(g, seqs, rows, vocab, torch.float32, kind, False, near=2.0)
    logits = (logits - logits.amax(2, keepdim=True)) * 0.3                  # nothing is likely
    parents = torch.zeros(seqs, rows, dtype=torch.int32, device=DEV)
    parents[::3, rows - 1] = 1
    u[:, 1] = torch.where(torch.rand(seqs, generator=g, device=DEV) < 0.8, 0.999, u[:, 1])
    tokens[1::4, 3] = tokens[1::4, 2]
    count, _, token = verified(amk, logits, tokens, u, parents, probs)
    assert kind == "probs" or bool((count == 1).any())                      # all children rejected, the token from what they left
    temperature = torch.tensor([0.7, 1.3, 0.0], device=DEV).repeat(seqs)[:seqs].contiguous()
    verified(amk, logits.to(torch.bfloat16), tokens, u, parents, probs, temperature)


@pytest.mark.parametrize("seqs,children,vocab", [(1, 6, 300007), (2, 3, 140001), (80, 3, 60011), (150, 4, 20000)])
def test_verify_draft_every_child_rejected_in_long_rows(amk, seqs, children, vocab):
    """Drafted tokens that the draft likes better than the target does, all below node 0: each one is rejected, and the token is drawn
    from what `children` rejections leave."""
    g = gen(vocab)
    logits = randn(g, seqs, children + 1, vocab, dtype=torch.float32)
    probs = torch.softmax(logits + randn(g, seqs, children + 1, vocab, dtype=torch.float32), 2)
    more = probs[:, 0].double() - torch.softmax(logits[:, 0].double(), 1)
    tokens = torch.cat([torch.zeros(seqs, 1, dtype=torch.long, device=DEV), more.topk(children, 1).indices], 1).to(torch.int32)
    u = torch.full((seqs, children + 1), 1.0 - 2.0 ** -23, device=DEV)
    u[:, 0] = torch.rand(seqs, generator=g, device=DEV)
    count = verified(amk, logits, tokens, u, torch.zeros(seqs, children + 1, dtype=torch.int32, device=DEV), probs)[0]
    assert count.tolist() == [1] * seqs


def test_verify_draft_of_the_targets_own_distribution_is_accepted(amk):
    """q = p rounded to 32 bits, off by 2^-24 of itself at most, is accepted by every number up to 1 - 2^-23: all of a chain, and in the
    target's order where a node has several children, the first one."""
    g = gen(31)
    for vocab in (5000, 128256):
        x = randn(g, 6, 8, vocab, dtype=torch.float32)
        probs = torch.softmax(x.double(), 2).float()
        drawn = torch.multinomial(probs.view(-1, vocab), 1, generator=g).view(6, 8).to(torch.int32)
        chain = torch.cat([drawn[:, :1], drawn[:, :-1]], 1).contiguous()                # node i's token comes from row i - 1
        u = torch.full((6, 8), 1.0 - 2.0 ** -23, device=DEV)
        u[:, 0] = 0.5
        assert verified(amk, x, chain, u, draft=probs)[0].tolist() == [8] * 6
        below = drawn[:, :1].expand(6, 8).contiguous()
        count, keep, _ = verified(amk, x, below, u, torch.zeros(6, 8, dtype=torch.int32, device=DEV), probs)
        assert count.tolist() == [2] * 6 and keep[:, 1].tolist() == [1] * 6


# ---- forms of a call --------------------------------------------------------------------------------------------

def test_given_workspaces_and_8_bit_types(amk):
    """A workspace that the caller keeps gives the same bits as one that is allocated, and an 8-bit cache may be called e4m3."""
    g = gen(17)
    q, k = randn(g, 2, 300, 8, 64), code(randn(g, 2, 2, 900, 64))
    lens = [500, 31]
    lse, n = true_lse(q, k, lens, 0.125), i32(lens)
    space = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    want = amk.amk_attention_weights(q, k, lse, n)
    for cache in (k, k.view(torch.float8_e4m3fn)):
        for rows in (300, 5):
            a = amk.amk_attention_weights(q[:, :rows], cache, lse[:, :rows].contiguous(), n, workspace=space.fill_(255))
            assert torch.equal(a, want if rows == 300 else amk.amk_attention_weights(q[:, :rows], k, lse[:, :rows].contiguous(), n))
    logits, tokens, u, _, probs = draft_case(g, 3, 6, 20000, torch.float32, "probs", False)
    for a, b in zip(amk.amk_verify_draft(logits, tokens, u, draft=probs, workspace=space.fill_(255)), amk.amk_verify_draft(logits, tokens, u, draft=probs)):
        assert torch.equal(a, b)
    x, pos = randn(g, 4, 8, 64), i32([5, 6, 7, 8])
    caches = [torch.zeros(1, 2, 9, 64, dtype=torch.uint8, device=DEV) for _ in range(4)]
    typed = [c.view(torch.float8_e4m3fn) for c in caches[2:]]
    for kc, vc in (caches[:2], typed):
        amk.amk_norm_rope_append(x[:, :4], x[:, 4:6], x[:, 6:], pos, kc, vc, pos.long())
    assert torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3]) and bool(caches[0].any())
