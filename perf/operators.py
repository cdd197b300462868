"""The operators around the decode step, as they are measured: what a serving program calls between the prompt and
the next decode step.

  prompt   attention over whole prompts, packed one behind the other, causal, grouped heads
  tree     attention of a tree of drafted tokens over each sequence's KV cache (bf16 or fp8 e4m3); one token is the
           smallest tree
  logprob  log probabilities of given tokens, with the entropy of each row and its top alternatives
  compact  the accepted drafted tokens (or the kept positions) moved together in every plane of the caches

``run`` computes them in their plain form, in elementary torch operations and 32 bits, or, where ``own`` is true, by
the calls that a user makes of the package.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
WORD = 64                                             # drafted tokens per word of a tree mask


def listed():
    return [
        # a seven-token prompt at the SmolLM2 shape: nothing but latency
        dict(name="prompt_tiny", op="prompt", nq=9, nkv=3, hd=64, lens="7"),
        # a batch of prompts of a chat service at the TinyLlama shape, lengths as they come
        dict(name="prompt_packed", op="prompt", nq=32, nkv=4, hd=64, lens="517,1,1291,250,33,777,64,129"),
        # one prompt that fills the Llama-3-8B context
        dict(name="prompt_long", op="prompt", nq=32, nkv=8, hd=128, lens="8192"),
        # one token after a short chat, no tree: the smallest call over a cache
        dict(name="tree_one_token", op="tree", nq=32, nkv=4, hd=64, rows=1, slots=2048, lens="1025", cache="bf16"),
        # a 26-node draft tree behind a long context
        dict(name="tree_draft", op="tree", nq=32, nkv=8, hd=128, rows=26, slots=8192, lens="8099", cache="bf16"),
        # eight conversations at once, each with 32 drafted tokens, ragged contexts
        dict(name="tree_batch", op="tree", nq=32, nkv=8, hd=128, rows=32, slots=8192,
             lens="8001,4097,513,6000,7777,2222,0,5310", cache="bf16"),
        # the same kind of batch over the 8-bit cache
        dict(name="tree_batch_fp8", op="tree", nq=32, nkv=8, hd=128, rows=16, slots=8192,
             lens="8111,7903,5001,6403,8000,3333,7212,64", cache="fp8"),
        # the log probability of one sampled token
        dict(name="logprob_one", op="logprob", rows=1, vocab=32000, dtype="f32", top=5),
        # the rows of a 64-node draft, with the alternatives that an API reports
        dict(name="logprob_draft", op="logprob", rows=64, vocab=128256, dtype="f32", top=20),
        # scoring a prompt: every position's token, 16-bit logits
        dict(name="logprob_prompt", op="logprob", rows=2001, vocab=128256, dtype="bf16", top=5),
        # six accepted tokens of a draft, every layer of a Llama-3-8B cache
        dict(name="compact_draft", op="compact", layers=32, nkv=8, hd=128, slots=2048, caches=1, most=26, kind="draft"),
        # a long conversation's cache with its middle dropped: the first tokens and a recent window stay
        dict(name="compact_window", op="compact", layers=22, nkv=4, hd=64, slots=8192, caches=2, most=5000,
             kind="window"),
    ]


HEADS = [(9, 3, 64), (32, 4, 64), (32, 8, 128), (32, 8, 64), (4, 2, 64), (8, 2, 128), (16, 2, 64), (3, 1, 64),
         (8, 8, 64), (16, 1, 128)]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "tree", "tree", "tree", "logprob", "logprob", "compact"])
    if op == "prompt":
        nq, nkv, hd = rng.choice(HEADS)
        total, lens = _log(rng, 1, 8000), []
        for _ in range(_log(rng, 1, 12)):
            n = min(total, _log(rng, 1, 8000))
            if n:
                lens.append(n)
                total -= n
        if rng.random() < 0.3:
            lens.insert(rng.randrange(len(lens) + 1), 0)
        return dict(op=op, nq=nq, nkv=nkv, hd=hd, lens=",".join(map(str, lens)))
    if op == "tree":
        nq, nkv, hd = rng.choice(HEADS)
        rows, seqs = _log(rng, 1, 128), _log(rng, 1, 8)
        slots = _log(rng, rows + 1, 8192)
        lens = [rng.choice([0, slots - rows, min(slots - rows, _log(rng, 1, slots))]) if rng.random() < 0.4 else
                rng.randint(0, slots - rows) for _ in range(seqs)]
        return dict(op=op, nq=nq, nkv=nkv, hd=hd, rows=rows, slots=slots, lens=",".join(map(str, lens)),
                    cache=rng.choice(["bf16", "bf16", "fp8"]))
    if op == "logprob":
        return dict(op=op, rows=_log(rng, 1, 850), vocab=_log(rng, 500, 150000), dtype=rng.choice(["f32", "bf16"]),
                    top=rng.choice([0, 1, 5, 20, 32]))
    nq, nkv, hd = rng.choice(HEADS)
    slots = _log(rng, 64, 2048)
    return dict(op=op, layers=rng.randint(1, 16), nkv=nkv, hd=hd, slots=slots, caches=_log(rng, 1, 4),
                most=_log(rng, 1, slots // 2), kind=rng.choice(["draft", "window"]))


# ---- inputs -----------------------------------------------------------------------------------------------------

def _lens(case):
    return [int(x) for x in case["lens"].split(",")]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32).to(DEV)


def _tree(rng, rows):
    """Random draft tree: every token's parent is an earlier one or the context.  Words of its ancestors' bits."""
    words = np.zeros((rows, (rows + WORD - 1) // WORD), dtype=np.uint64)
    for i in range(rows):
        parent = int(rng.integers(-1, i)) if i else -1
        if parent >= 0:
            words[i] = words[parent]
        words[i, i // WORD] |= np.uint64(1) << np.uint64(i % WORD)
    return words.view(np.int64)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 17)
    rng = np.random.default_rng(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)

    op = case["op"]
    if op == "prompt":
        # q, k and v as the fused projection leaves them: slices of one row per token
        nq, nkv, hd, lens = case["nq"], case["nkv"], case["hd"], _lens(case)
        total = sum(lens)
        rows = normal(total, nq + 2 * nkv, hd).to(torch.bfloat16)
        cu = _i32([0] + list(np.cumsum(lens)))
        return dict(op=op, q=rows[:, :nq], k=rows[:, nq:nq + nkv], v=rows[:, nq + nkv:], cu=cu)
    if op == "tree":
        nq, nkv, hd, rows, slots, lens = case["nq"], case["nkv"], case["hd"], case["rows"], case["slots"], _lens(case)
        kv = normal(2, len(lens), nkv, slots, hd)
        kv = kv.to(torch.float8_e4m3fn).view(torch.uint8) if case["cache"] == "fp8" else kv.to(torch.bfloat16)
        mask = torch.from_numpy(np.stack([_tree(rng, rows) for _ in lens])).to(DEV)
        return dict(op=op, q=normal(len(lens), rows, nq, hd).to(torch.bfloat16), k=kv[0], v=kv[1], len=_i32(lens),
                    mask=mask)
    if op == "logprob":
        rows, vocab = case["rows"], case["vocab"]
        x = (normal(rows, vocab) * 2.5).to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
        tokens = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
        tokens[::2] = x[::2].argmax(dim=1)            # half of them are what a greedy choice takes
        return dict(op=op, logits=x, tokens=tokens.to(torch.int32), top=case["top"])
    caches, slots, most = case["caches"], case["slots"], case["most"]
    kv = normal(caches, 2, case["layers"], case["nkv"], slots, case["hd"]).to(torch.bfloat16)
    base, keep, count = _kept(rng, case)
    return dict(op=op, kv=kv, base=_i32(base), keep=_i32(keep), count=_i32(count), most=most)


def _kept(rng, case):
    """Per cache: where the kept rows go, their slots in ascending order (rows behind the count: 0), how many."""
    slots, most = case["slots"], case["most"]
    base, keep, count = [], [], []
    for _ in range(case["caches"]):
        first = int(rng.integers(0, slots - most + 1)) if case["kind"] == "draft" else min(4, slots - most)
        n = int(rng.integers(max(1, most // 4), most // 2 + 2)) if case["kind"] == "draft" else most - int(rng.integers(0, most // 8 + 1))
        n = min(n, most)
        if case["kind"] == "draft":                   # some of the `most` drafted rows
            rows = first + np.sort(rng.choice(most, n, replace=False))
        else:                                         # the last n rows of the cache
            rows = np.arange(slots - n, slots)
        base.append(first)
        count.append(n)
        keep.append(list(map(int, rows)) + [0] * (most - n))
    return base, keep, count


# ---- the operators ----------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _package(s)
    return {"prompt": _prompt, "tree": _tree_attention, "logprob": _logprob, "compact": _compact}[s["op"]](s)


def _package(s):
    from paper_2606_09682_b200 import binding as amk
    op = s["op"]
    if op == "prompt":
        return amk.amk_prompt_attention(s["q"], s["k"], s["v"], s["cu"])
    if op == "tree":
        return amk.amk_tree_attention(s["q"], s["k"], s["v"], s["len"], s["mask"])
    if op == "logprob":
        return amk.amk_token_logprobs(s["logits"], s["tokens"], s["top"])
    amk.amk_kv_compact(s["kv"], s["base"], s["keep"], s["count"])
    return s["kv"]


def _prompt(s):
    q, k, v, cu = s["q"], s["k"], s["v"], s["cu"]
    total, nq, hd = q.shape
    nkv = k.shape[1]
    at = torch.arange(total, device=q.device)
    seq = torch.bucketize(at, cu[1:].long(), right=True)
    allowed = (seq[:, None] == seq[None, :]) & (at[None, :] <= at[:, None])
    qf = q.float().reshape(total, nkv, nq // nkv, hd).permute(1, 2, 0, 3) / math.sqrt(hd)
    kf, vf = k.float().permute(1, 0, 2)[:, None], v.float().permute(1, 0, 2)[:, None]
    x = (qf @ kf.transpose(-1, -2)).masked_fill(~allowed, -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    o = (p @ vf) / p.sum(-1, keepdim=True)
    return o.permute(2, 0, 1, 3).reshape(total, nq, hd).to(torch.bfloat16)


def _values(t):
    return t.view(torch.float8_e4m3fn).float() if t.dtype == torch.uint8 else t.float()


def _tree_attention(s):
    q, k, v, length, mask = s["q"], _values(s["k"]), _values(s["v"]), s["len"], s["mask"]
    seqs, rows, nq, hd = q.shape
    nkv, slots = k.shape[1], k.shape[2]
    bits = (mask[..., None] >> torch.arange(WORD, device=q.device)) & 1
    bits = bits.reshape(seqs, rows, -1)[:, :, :rows].bool()
    rel = torch.arange(slots, device=q.device)[None] - length[:, None]
    drafted = torch.gather(bits, 2, rel.clamp(0, rows - 1).long()[:, None].expand(seqs, rows, slots))
    allowed = (rel < 0)[:, None] | ((rel >= 0) & (rel < rows))[:, None] & drafted
    qf = q.float().reshape(seqs, rows, nkv, nq // nkv, hd).permute(0, 2, 3, 1, 4) / math.sqrt(hd)
    x = (qf @ k[:, :, None].transpose(-1, -2)).masked_fill(~allowed[:, None, None], -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    o = (p @ v[:, :, None]) / p.sum(-1, keepdim=True)
    return o.permute(0, 3, 1, 2, 4).reshape(seqs, rows, nq, hd).to(torch.bfloat16)


def _logprob(s):
    x, top = s["logits"].float(), s["top"]
    rows, vocab = x.shape
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    logs = torch.log(total)
    lp = x.gather(1, s["tokens"].long()[:, None]) - m - logs
    entropy = logs - (e * (x - m)).sum(1, keepdim=True) / total
    # the largest logits, the lowest index first among equal ones: one 64-bit key for each
    bits = x.view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    key = (order << 32) | (0x7FFFFFFF - torch.arange(vocab, device=x.device))
    best = torch.topk(key, min(top, vocab), dim=1).indices
    return lp[:, 0], entropy[:, 0], best.to(torch.int32), x.gather(1, best) - m - logs


def _compact(s):
    kv, base, keep, count, most = s["kv"], s["base"].long(), s["keep"].long(), s["count"].long(), s["most"]
    caches, slots, hd = kv.shape[0], kv.shape[-2], kv.shape[-1]
    planes = kv.view(caches, -1, slots, hd)
    i = torch.arange(most, device=kv.device)[None]
    to = base[:, None] + i
    src = torch.where(i < count[:, None], keep, to)
    shape = (caches, planes.shape[1], most, hd)
    moved = torch.gather(planes, 2, src[:, None, :, None].expand(shape))
    planes.scatter_(2, to[:, None, :, None].expand(shape), moved)
    return kv


# ---- what they cannot do without --------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "prompt":
        nq, nkv, hd, lens = case["nq"], case["nkv"], case["hd"], _lens(case)
        pairs = sum(n * (n + 1) // 2 for n in lens)
        return dict(bytes=2 * sum(lens) * hd * (2 * nq + 2 * nkv) + 4 * (len(lens) + 1), flops=4 * pairs * nq * hd)
    if op == "tree":
        nq, nkv, hd, rows, lens = case["nq"], case["nkv"], case["hd"], case["rows"], _lens(case)
        size = 1 if case["cache"] == "fp8" else 2
        cached = sum(lens) + len(lens) * rows
        words = (rows + WORD - 1) // WORD
        return dict(bytes=2 * size * cached * nkv * hd + 4 * len(lens) * rows * nq * hd + len(lens) * (4 + 8 * rows * words),
                    flops=4 * cached * rows * nq * hd)
    if op == "logprob":
        size = 2 if case["dtype"] == "bf16" else 4
        rows, vocab = case["rows"], case["vocab"]
        return dict(bytes=rows * (size * vocab + 12 + 8 * min(case["top"], vocab)), flops=5 * rows * vocab)
    # the rows that move, read once and written once; draft: about 3/8 of `most`, window: about 15/16
    share = 0.375 if case["kind"] == "draft" else 0.9375
    row = 2 * case["layers"] * case["nkv"] * case["hd"] * 2
    return dict(bytes=case["caches"] * (2 * max(1, share * case["most"]) * row + 4 * (case["most"] + 2)), flops=0)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "prompt":
        q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
        out = torch.zeros_like(q)
        rep, at = case["nq"] // case["nkv"], 0
        for n in _lens(case):
            if not n:
                continue
            hidden = torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1)
            for h in range(case["nq"]):
                x = torch.einsum("id,jd->ij", q[at:at + n, h], k[at:at + n, h // rep]) * case["hd"] ** -0.5
                x[hidden] = -math.inf
                out[at:at + n, h] = torch.softmax(x, 1) @ v[at:at + n, h // rep]
            at += n
        return out
    if op == "tree":
        q, k, v = s["q"].double(), _values(s["k"]).double(), _values(s["v"]).double()
        out = torch.zeros_like(q)
        rep, rows = case["nq"] // case["nkv"], case["rows"]
        words = s["mask"].cpu().numpy().view(np.uint64)
        for b, n in enumerate(_lens(case)):
            sees = torch.ones(rows, n + rows, dtype=torch.bool)
            for i in range(rows):
                for j in range(rows):
                    sees[i, n + j] = bool((int(words[b, i, j // WORD]) >> (j % WORD)) & 1)
            sees = sees.to(DEV)
            for h in range(case["nq"]):
                x = torch.einsum("id,jd->ij", q[b, :, h], k[b, h // rep, :n + rows]) * case["hd"] ** -0.5
                out[b, :, h] = torch.softmax(x.masked_fill(~sees, -math.inf), 1) @ v[b, h // rep, :n + rows]
        return out
    if op == "logprob":
        lp, entropy, ids, tops = [], [], [], []
        top = min(case["top"], case["vocab"])
        for row, token in zip(s["logits"], s["tokens"].tolist()):
            x = torch.log_softmax(row.double(), 0)
            lp.append(x[token])
            entropy.append(-(x.exp() * x).sum())
            first = torch.sort(row, descending=True, stable=True).indices[:top]
            ids.append(first)
            tops.append(x[first])
        return torch.stack(lp), torch.stack(entropy), torch.stack(ids).to(torch.int32), torch.stack(tops)
    kv = s["kv"]
    out = kv.clone()
    for c in range(case["caches"]):
        n, base = int(s["count"][c]), int(s["base"][c])
        out[c, ..., base:base + n, :] = kv[c].index_select(-2, s["keep"][c, :n].long())
    return out.double()
