"""Operators between the projections, the attentions and the cache, as they are measured.

  rope     queries and keys normed for each head (or not) and rotated to their positions, the rotated keys and the values
           stored in their cache rows (bf16 or fp8 e4m3), in one pass over the projection
  weights  what attention weight the queries of some tokens put on every cached position, added up for each kv head
  evict    which positions of a cache stay, by those weights: the first ones, the recent ones and the heaviest
  verify   a chain or tree of drafted tokens accepted or rejected against the target's probabilities, from given uniform
           numbers, and the next token drawn

``run`` computes them in their plain form, in elementary torch operations (64 bits for angles, and for sums next to whose
borders a token is chosen), or, where ``own`` is true, by the calls that a user makes of the package.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
THETA, EPS = 500000.0, 1e-5


def listed():
    return [
        # one new token at the SmolLM2 shape, a layer's step of a chat: nothing but latency
        dict(name="rope_one_token", op="rope", nq=9, nkv=3, hd=64, norm=False, cache="bf16", slots=2048, lens="777", rows=1),
        # eight conversations with a 26-node draft each, normed heads, 8-bit cache
        dict(name="rope_draft_fp8", op="rope", nq=32, nkv=8, hd=128, norm=True, cache="fp8", slots=2048,
             lens="2001,1097,513,1600,777,222,0,1310", rows=26),
        # a prompt that fills most of a context, normed heads
        dict(name="rope_prompt", op="rope", nq=32, nkv=8, hd=128, norm=True, cache="bf16", slots=8192, lens="0", rows=8111),
        # one token of a chat: its weights over 1026 positions
        dict(name="weights_one_token", op="weights", nq=32, nkv=4, hd=64, rows=1, slots=2048, lens="1025", cache="bf16",
             decay=1.0),
        # the last 32 tokens of four long prompts look back over their caches
        dict(name="weights_window", op="weights", nq=32, nkv=8, hd=128, rows=32, slots=8192, lens="8001,5310,6999,4097",
             cache="bf16", decay=0.0),
        # the same over the 8-bit cache, a draft's worth of tokens
        dict(name="weights_window_fp8", op="weights", nq=32, nkv=8, hd=128, rows=13, slots=8192,
             lens="8111,7903,64,6403,8000,3333,7212,0", cache="fp8", decay=0.9),
        # every token of a whole prompt
        dict(name="weights_prompt", op="weights", nq=32, nkv=8, hd=128, rows=7001, slots=7168, lens="0", cache="bf16",
             decay=0.0),
        # one layer of a chat's cache
        dict(name="evict_chat", op="evict", seqs=1, nkv=4, slots=2048, budget=512, first=4, recent=64),
        # every layer and head of a long context at once
        dict(name="evict_layers", op="evict", seqs=32, nkv=8, slots=8192, budget=2048, first=4, recent=256),
        # a greedy chat with four guessed tokens
        dict(name="verify_greedy", op="verify", seqs=1, rows=5, vocab=32000, dtype="f32", draft="point", tree=False,
             temperature=0.0),
        # a batch with drafts from a small model
        dict(name="verify_chain", op="verify", seqs=8, rows=6, vocab=128256, dtype="f32", draft="probs", tree=False,
             temperature=0.8),
        # draft trees of a batch, 16-bit logits
        dict(name="verify_tree", op="verify", seqs=6, rows=26, vocab=128256, dtype="bf16", draft="probs", tree=True,
             temperature=1.0),
    ]


HEADS = [(9, 3, 64), (32, 4, 64), (32, 8, 128), (32, 8, 64), (4, 2, 64), (8, 2, 128), (16, 2, 64), (3, 1, 64),
         (8, 8, 64), (16, 1, 128)]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["rope", "rope", "weights", "weights", "weights", "evict", "verify", "verify", "verify"])
    nq, nkv, hd = rng.choice(HEADS)
    if op == "rope":
        seqs, rows = _log(rng, 1, 8), _log(rng, 1, 1000)
        slots = _log(rng, rows, 8192)
        lens = [rng.randint(0, slots - rows) for _ in range(seqs)]
        return dict(op=op, nq=nq, nkv=nkv, hd=hd, norm=rng.random() < 0.5, cache=rng.choice(["bf16", "fp8"]), slots=slots,
                    lens=",".join(map(str, lens)), rows=rows)
    if op == "weights":
        seqs = _log(rng, 1, 8)
        rows = _log(rng, 1, 4096 // seqs)
        slots = _log(rng, rows + 1, 8192)
        lens = [rng.choice([0, slots - rows]) if rng.random() < 0.2 else rng.randint(0, slots - rows) for _ in range(seqs)]
        return dict(op=op, nq=nq, nkv=nkv, hd=hd, rows=rows, slots=slots, lens=",".join(map(str, lens)),
                    cache=rng.choice(["bf16", "bf16", "fp8"]), decay=rng.choice([0.0, 0.9, 1.0]))
    if op == "evict":
        slots = _log(rng, 64, 16384)
        budget = _log(rng, 8, slots)
        return dict(op=op, seqs=_log(rng, 1, 16), nkv=nkv, slots=slots, budget=budget, first=rng.randint(0, budget // 4),
                    recent=rng.randint(0, budget // 2))
    rows = _log(rng, 1, 32)
    return dict(op=op, seqs=_log(rng, 1, 160 // rows if rows > 20 else 8), rows=rows, vocab=_log(rng, 500, 150000),
                dtype=rng.choice(["f32", "bf16"]), draft=rng.choice(["probs", "point"]), tree=rng.random() < 0.5,
                temperature=rng.choice([0.0, 0.6, 1.0, 1.3]))


# ---- inputs -----------------------------------------------------------------------------------------------------

def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32).to(DEV)


def _parents(rng, rows, tree):
    """Node 0 is the token that is already chosen; a drafted token follows the one before it, or one of a few before it."""
    return [-1] + [int(rng.integers(max(0, i - 4), i)) if tree else i - 1 for i in range(1, rows)]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 29)
    rng = np.random.default_rng(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)

    op = case["op"]
    if op == "rope":
        # q, k and v as the fused projection leaves them: slices of one row per token; the sequences' tokens one behind
        # the other, each to be stored behind its own context
        nq, nkv, hd, lens, rows, slots = case["nq"], case["nkv"], case["hd"], _lens(case), case["rows"], case["slots"]
        x = (normal(len(lens) * rows, nq + 2 * nkv, hd) * 1.7).to(torch.bfloat16)
        cache = normal(2, len(lens), nkv, slots, hd)
        cache = cache.to(torch.float8_e4m3fn).view(torch.uint8) if case["cache"] == "fp8" else cache.to(torch.bfloat16)
        at = np.concatenate([n + np.arange(rows) for n in lens])
        where = np.concatenate([s * slots + n + np.arange(rows) for s, n in enumerate(lens)])
        weight = lambda: (1 + 0.2 * normal(hd)).to(torch.bfloat16) if case["norm"] else None
        return dict(op=op, q=x[:, :nq], k=x[:, nq:nq + nkv], v=x[:, nq + nkv:], kc=cache[0], vc=cache[1],
                    at=_i32(at), where=torch.from_numpy(where).to(DEV), wq=weight(), wk=weight())
    if op == "weights":
        nq, nkv, hd, lens, rows, slots = case["nq"], case["nkv"], case["hd"], _lens(case), case["rows"], case["slots"]
        k = normal(len(lens), nkv, slots, hd)
        k = k.to(torch.float8_e4m3fn).view(torch.uint8) if case["cache"] == "fp8" else k.to(torch.bfloat16)
        q = normal(len(lens), rows, nq, hd).to(torch.bfloat16)
        lse = torch.empty(len(lens), rows, nq, device=DEV)        # as the attention over this cache leaves it
        for s, n in enumerate(lens):
            kf = _values(k[s, :, :n + rows])
            hidden = torch.arange(n + rows, device=DEV)[None] > n + torch.arange(rows, device=DEV)[:, None]
            for h in range(nq):
                x = (q[s, :, h].float() @ kf[h // (nq // nkv)].T) / math.sqrt(hd)
                lse[s, :, h] = torch.logsumexp(x.masked_fill_(hidden, -math.inf), 1)
        before = torch.rand(len(lens), nkv, slots, generator=g, device=DEV) if case["decay"] else None
        return dict(op=op, q=q, k=k, lse=lse, len=_i32(lens), before=before, decay=case["decay"])
    if op == "evict":
        # added-up weights have a long tail: few positions carry most
        scores = torch.exp(2 * normal(case["seqs"], case["nkv"], case["slots"]))
        lens = [case["slots"] - int(rng.integers(0, case["slots"] // 8 + 1)) for _ in range(case["seqs"])]
        return dict(op=op, scores=scores, len=_i32(lens), budget=case["budget"], first=case["first"], recent=case["recent"])
    seqs, rows, vocab = case["seqs"], case["rows"], case["vocab"]
    x = normal(seqs, rows, vocab) * 2.5
    likely = torch.randint(0, vocab, (seqs, rows, 1), generator=g, device=DEV)
    x.scatter_(2, likely, torch.logsumexp(x, 2, keepdim=True) + 0.5)     # one token has more than half of each row
    parents = np.array([_parents(rng, rows, case["tree"]) for _ in range(seqs)])
    above = torch.from_numpy(parents.clip(0)).to(DEV)
    probs = None
    if case["draft"] == "probs":                                         # a draft model that nearly agrees
        probs = torch.softmax((x + 0.4 * normal(seqs, rows, vocab)) / max(case["temperature"], 0.5), 2)
        drawn = torch.multinomial(probs.view(seqs * rows, vocab), rows, replacement=True, generator=g).view(seqs, rows, rows)
        tokens = drawn[torch.arange(seqs, device=DEV)[:, None], above, torch.arange(rows, device=DEV)[None]]
    else:                                                                # guesses: the likely token, or another
        wrong = torch.randint(0, vocab, (seqs, rows), generator=g, device=DEV)
        right = torch.rand(seqs, rows, generator=g, device=DEV) < 0.6
        tokens = torch.where(right, torch.gather(likely[..., 0], 1, above), wrong)
    return dict(op=op, logits=x.to(torch.bfloat16) if case["dtype"] == "bf16" else x, tokens=tokens.to(torch.int32),
                u=torch.rand(seqs, rows, generator=g, device=DEV), parents=_i32(parents) if case["tree"] else None,
                probs=probs, temperature=torch.full((seqs,), case["temperature"], device=DEV),
                len=_i32([int(rng.integers(0, 8000)) for _ in range(seqs)]))


# ---- the operators ----------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _package(s)
    return {"rope": _rope, "weights": _weights, "evict": _evict, "verify": _verify}[s["op"]](s)


def _package(s):
    from paper_2606_09682_b200 import binding as amk
    op = s["op"]
    if op == "rope":
        q = amk.amk_norm_rope_append(s["q"], s["k"], s["v"], s["at"], s["kc"], s["vc"], s["where"], q_weight=s["wq"],
                                     k_weight=s["wk"], eps=EPS, theta=THETA)
        return q, _coded(s["kc"]), _coded(s["vc"])
    if op == "weights":
        return amk.amk_attention_weights(s["q"], s["k"], s["lse"], s["len"], s["before"], s["decay"])
    if op == "evict":
        return amk.amk_evict_select(s["scores"], s["len"], s["budget"], s["first"], s["recent"])
    return amk.amk_verify_draft(s["logits"], s["tokens"], s["u"], s["parents"], s["probs"], s["temperature"], s["len"])


def _values(t):
    return t.view(torch.float8_e4m3fn).float() if t.dtype == torch.uint8 else t.float()


def _coded(t):
    return t.view(torch.float8_e4m3fn) if t.dtype == torch.uint8 else t


def _rope(s):
    q, k, v, kc, vc, where = s["q"], s["k"], s["v"], s["kc"], s["vc"], s["where"]
    hd = q.shape[2]
    inv = THETA ** (-torch.arange(0, hd, 2, device=q.device, dtype=torch.float64) / hd)
    angle = s["at"].double()[:, None] * inv
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x, weight):
        x = x.float()
        if weight is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
        a, b = x[..., :hd // 2], x[..., hd // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    slots = kc.shape[2]
    for cache, rows in ((kc, turned(k, s["wk"])), (vc, v.float())):
        if cache.dtype == torch.uint8:
            rows = rows.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        cache[where // slots, :, where % slots] = rows.to(cache.dtype)
    return turned(q, s["wq"]).to(torch.bfloat16), _coded(kc), _coded(vc)


def _weights(s):
    q, k, lse, length, before = s["q"], _values(s["k"]), s["lse"], s["len"], s["before"]
    seqs, rows, nq, hd = q.shape
    nkv, slots = k.shape[1], k.shape[2]
    at = torch.arange(slots, device=q.device)
    allowed = at[None, None] <= length[:, None, None] + torch.arange(rows, device=q.device)[None, :, None]
    qf = q.float().reshape(seqs, rows, nkv, nq // nkv, hd).permute(0, 2, 3, 1, 4) / math.sqrt(hd)
    x = qf @ k[:, :, None].transpose(-1, -2)                             # [seqs][nkv][rep][rows][slots]
    x -= lse.reshape(seqs, rows, nkv, nq // nkv).permute(0, 2, 3, 1)[..., None]
    out = x.exp_().mul_(allowed[:, None, None]).sum((2, 3))
    if before is not None:
        out = out + s["decay"] * before.masked_fill((at >= length[:, None])[:, None], 0)
    return out


def _evict(s):
    scores, length, budget, first, recent = s["scores"], s["len"].long(), s["budget"], s["first"], s["recent"]
    seqs, heads, slots = scores.shape
    at = torch.arange(slots, device=scores.device)
    n = length[:, None, None]
    # one 64-bit key each: what stays anyway, then the heaviest, the lowest index first among equal ones
    bits = scores.view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    order = torch.where((at < first) | (at >= n - recent), 0x7FFFFFFF, order)
    key = torch.where(at < n, (order << 31) | (0x7FFFFFFF - at), torch.iinfo(torch.int64).min)
    count = torch.minimum(length, torch.full_like(length, budget))[:, None].expand(seqs, heads)
    best = torch.topk(key, budget, dim=2).indices
    i = torch.arange(budget, device=scores.device)
    stays = torch.sort(torch.where(i < count[..., None], best, slots), dim=2).values
    inside = stays < slots
    moved = torch.zeros_like(scores)
    moved[..., :budget] = torch.gather(scores, 2, stays.clamp(max=slots - 1)) * inside
    return torch.where(inside, stays, -1).to(torch.int32), count.to(torch.int32), moved


def _verify(s):
    logits, tokens, u, probs, temperature = s["logits"], s["tokens"].long(), s["u"].double(), s["probs"], s["temperature"].double()
    seqs, rows, vocab = logits.shape
    all_ = torch.arange(seqs, device=logits.device)
    parents = torch.arange(-1, rows - 1, device=logits.device).expand(seqs, rows) if s["parents"] is None else s["parents"].long()

    def target(row):                                                     # probabilities of one row of each sequence
        x = logits[all_, row].double()
        best = x.argmax(1, keepdim=True)
        e = torch.exp((x - x.gather(1, best)) / torch.where(temperature > 0, temperature, 1.0)[:, None])
        one = torch.zeros_like(e).scatter_(1, best, 1.0)
        return torch.where((temperature > 0)[:, None], e / e.sum(1, keepdim=True), one)

    at = torch.zeros(seqs, dtype=torch.long, device=logits.device)       # the last accepted node
    p = target(at)
    kept = [all_ >= 0]
    for i in range(1, rows):
        here = parents[:, i] == at
        token = tokens[:, i]
        if probs is None:
            q = torch.zeros_like(p).scatter_(1, token[:, None], 1.0)
        else:
            q = probs[all_, at].double()
        took = here & (u[:, i] * q[all_, token] < p[all_, token])
        rest = torch.clamp(p - q, min=0)
        total = rest.sum(1, keepdim=True)
        p = torch.where((here & ~took)[:, None] & (total > 0), rest / total, p)
        at = torch.where(took, i, at)
        p = torch.where(took[:, None], target(at), p)
        kept.append(took)
    sums = p.cumsum(1)
    over = sums > u[:, :1] * sums[:, -1:]
    last = vocab - 1 - (p > 0).flip(1).int().argmax(1)
    token = torch.where(over.any(1), over.int().argmax(1), last)
    kept = torch.stack(kept, 1)
    place = torch.where(kept, torch.arange(rows, device=logits.device), rows).sort(1).values
    keep = torch.where(place < rows, place + s["len"][:, None], -1)
    return kept.sum(1).to(torch.int32), keep.to(torch.int32), token.to(torch.int32)


# ---- what they cannot do without --------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "rope":
        nq, nkv, hd, tokens = case["nq"], case["nkv"], case["hd"], len(_lens(case)) * case["rows"]
        size = 1 if case["cache"] == "fp8" else 2
        return dict(bytes=tokens * hd * (4 * nq + 4 * nkv + 2 * size * nkv) + 12 * tokens + (4 * hd if case["norm"] else 0),
                    flops=tokens * hd * (nq + nkv) * (7 if case["norm"] else 3))
    if op == "weights":
        nq, nkv, hd, rows, lens = case["nq"], case["nkv"], case["hd"], case["rows"], _lens(case)
        size = 1 if case["cache"] == "fp8" else 2
        cached = sum(lens) + len(lens) * rows
        pairs = sum(n * rows + rows * (rows + 1) // 2 for n in lens)
        return dict(bytes=size * cached * nkv * hd + len(lens) * (rows * nq * (2 * hd + 4) + 4) + 4 * len(lens) * nkv * case["slots"] +
                    (4 * sum(lens) * nkv if case["decay"] else 0), flops=2 * pairs * nq * hd)
    if op == "evict":
        lists, n = case["seqs"] * case["nkv"], case["slots"] * 15 // 16          # (the mean length)
        return dict(bytes=lists * 4 * (n + case["budget"] + 1 + case["slots"]) + 4 * case["seqs"], flops=0)
    # the rows of the nodes that are reached, and of the draft's the ones where something was rejected: about 0.8 of the
    # drafted tokens are accepted from one node to the next (0.6 of the guesses), through the depth of the chain or tree
    seqs, rows, vocab = case["seqs"], case["rows"], case["vocab"]
    share = 0.8 if case["draft"] == "probs" else 0.6
    depth = max(1, rows // 3) if case["tree"] else rows - 1
    reached = 1 + sum(share ** i for i in range(1, depth + 1))
    drafted = 4 * vocab if case["draft"] == "probs" and rows > 1 else 0
    return dict(bytes=int(seqs * (reached * (2 if case["dtype"] == "bf16" else 4) * vocab + drafted + 16 * rows)),
                flops=int(seqs * reached * 4 * vocab))


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rope":
        hd, slots = case["hd"], case["slots"]
        i = np.arange(hd // 2)
        angle = torch.from_numpy(s["at"].cpu().numpy()[:, None].astype(np.float64) * THETA ** (-2.0 * i / hd)).to(DEV)
        turn = torch.complex(angle.cos(), angle.sin())[:, None]

        def rotated(x, w):
            x = x.double()
            if w is not None:
                x = x * torch.rsqrt(x.square().mean(2, keepdim=True) + EPS) * w.double()
            z = torch.complex(x[:, :, :hd // 2].contiguous(), x[:, :, hd // 2:].contiguous()) * turn
            return torch.cat([z.real, z.imag], 2)

        kc, vc = _values(s["kc"]).double(), _values(s["vc"]).double()
        k, v, rows = rotated(s["k"], s["wk"]), s["v"].double(), case["rows"]
        if case["cache"] == "fp8":
            k, v = k.clamp(-448, 448), v.clamp(-448, 448)
        for b, n in enumerate(_lens(case)):
            kc[b, :, n:n + rows] = k[b * rows:(b + 1) * rows].transpose(0, 1)
            vc[b, :, n:n + rows] = v[b * rows:(b + 1) * rows].transpose(0, 1)
        return rotated(s["q"], s["wq"]), kc, vc
    if op == "weights":
        rep, rows = case["nq"] // case["nkv"], case["rows"]
        out = torch.zeros(s["k"].shape[:3], dtype=torch.float64, device=DEV)
        for b, n in enumerate(_lens(case)):
            hidden = torch.ones(rows, n + rows, dtype=torch.bool, device=DEV).triu(n + 1)
            if s["before"] is not None:
                out[b, :, :n] = s["before"][b, :, :n].double() * case["decay"]
            for h in range(case["nq"]):
                x = s["q"][b, :, h].double() @ _values(s["k"][b, h // rep, :n + rows]).double().T * case["hd"] ** -0.5
                w = torch.exp(x - s["lse"][b, :, h].double()[:, None]).masked_fill(hidden, 0)
                out[b, h // rep, :n + rows] += w.sum(0)
        return out
    if op == "evict":
        seqs, heads, slots, budget = case["seqs"], case["nkv"], case["slots"], case["budget"]
        scores, lens = s["scores"].cpu().numpy(), s["len"].tolist()
        keep = np.full((seqs, heads, budget), -1, dtype=np.int32)
        count = np.zeros((seqs, heads), dtype=np.int32)
        moved = np.zeros(scores.shape, dtype=np.float64)
        for b, n in enumerate(lens):
            for h in range(heads):
                if n <= budget:
                    rows = np.arange(n)
                else:
                    tail = n - case["recent"]
                    middle = case["first"] + np.argsort(-scores[b, h, case["first"]:tail], kind="stable")
                    rows = np.sort(np.concatenate([np.arange(case["first"]), np.arange(tail, n),
                                                   middle[:budget - case["first"] - case["recent"]]]))
                count[b, h] = len(rows)
                keep[b, h, :len(rows)] = rows
                moved[b, h, :len(rows)] = scores[b, h, rows]
        return torch.from_numpy(keep), torch.from_numpy(count), torch.from_numpy(moved)
    seqs, rows, vocab = case["seqs"], case["rows"], case["vocab"]
    count, keep, chosen = [], torch.full((seqs, rows), -1, dtype=torch.int32), []
    for b in range(seqs):
        node, path, children = 0, [0], {}
        for i in range(1, rows):
            children.setdefault(int(s["parents"][b, i]) if s["parents"] is not None else i - 1, []).append(i)
        while True:
            x = s["logits"][b, node].double()
            if case["temperature"] > 0:
                p = torch.softmax(x / float(s["temperature"][b]), 0)
            else:
                p = torch.zeros_like(x)
                p[int(torch.nonzero(x == x.max())[0])] = 1
            found = None
            for c in children.get(node, []):
                t, u = int(s["tokens"][b, c]), float(s["u"][b, c])
                q = torch.zeros_like(p) if s["probs"] is None else s["probs"][b, node].double()
                if s["probs"] is None:
                    q[t] = 1
                if u * float(q[t]) < float(p[t]):
                    found = c
                    break
                rest = (p - q).clamp(min=0)
                if float(rest.sum()) > 0:
                    p = rest / rest.sum()
            if found is None:
                break
            node = found
            path.append(node)
        sums = torch.cumsum(p, 0)
        over = torch.nonzero(sums > float(s["u"][b, 0]) * sums[-1])
        chosen.append(int(over[0]) if len(over) else int(torch.nonzero(p > 0)[-1]))
        count.append(len(path))
        keep[b, :len(path)] = torch.tensor(path, dtype=torch.int32) + int(s["len"][b])
    return torch.tensor(count, dtype=torch.int32), keep, torch.tensor(chosen, dtype=torch.int32)
