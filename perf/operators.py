"""Measured cases of the worker-side operators: embedding lookup and its gradient, dropout from a counter-based
generator and its gradient, attention and its gradient.

`listed()` names the cases, `draw()` gives further ones of the same ranges, `prepare()` makes what a training program
holds before the call, `run()` is one pass: with `own` set through the library's entry points, otherwise in plain torch
operations in 32 bits, rounded once at the end.  `exact()` states the same results in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
PHILOX_STREAM = 5                 # purpose word of a dropout draw


# --------------------------------------------------------------------------------------------------------------
# Cases.  Widths, vocabularies, heads and lengths are those of the GPT-2-XL-shaped (50257 x 1600, 25 heads of 64,
# 1024 tokens) and BERT-large-shaped (30522 x 1024, 16 heads of 64, 512 tokens) workloads, or generic.
# --------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token's row: generation, or the last token of a stream; latency alone
        {"name": "embed_one", "op": "embed", "n": 1, "V": 50257, "D": 1600, "table": "bf16", "act": "bf16", "pad": False},
        # a worker's batch of 8 x 1024 tokens, fp32 throughout
        {"name": "embed_batch", "op": "embed", "n": 8192, "V": 50257, "D": 1600, "table": "f32", "act": "f32", "pad": False},
        # dense embedding gradient of 16 x 512 padded tokens, bf16 gradients as the transport of that workload carries
        {"name": "embed_grad_padded", "op": "embed_grad", "n": 8192, "V": 30522, "D": 1024, "table": "bf16", "act": "bf16",
         "pad": True},
        # dense embedding gradient of 32 x 1024 tokens, fp32: the largest tensor of that model's gradient
        {"name": "embed_grad_batch", "op": "embed_grad", "n": 32768, "V": 50257, "D": 1600, "table": "f32", "act": "f32",
         "pad": False},
        # a few rows of odd width: latency, and rows whose groups of draws straddle row ends
        {"name": "dropout_odd", "op": "dropout", "rows": 7, "cols": 1601, "act": "bf16", "p": 0.1, "residual": False,
         "grad": False},
        # residual dropout behind a block of 8 x 1024 tokens
        {"name": "dropout_residual", "op": "dropout", "rows": 8192, "cols": 1600, "act": "bf16", "p": 0.1, "residual": True,
         "grad": False},
        # gradient through dropout of a feed-forward activation of 32 x 1024 tokens, fp32
        {"name": "dropout_grad_large", "op": "dropout", "rows": 32768, "cols": 6400, "act": "f32", "p": 0.1,
         "residual": False, "grad": True},
        # one new token per sequence against 1024 cached ones
        {"name": "attention_one", "op": "attention", "B": 8, "Sq": 1, "Sk": 1024, "Hq": 25, "Hkv": 25, "D": 64, "act": "bf16",
         "causal": True, "lens": False, "packed": False},
        # an encoder's batch of padded sequences, one slot of the batch empty
        {"name": "attention_padded", "op": "attention", "B": 32, "Sq": 512, "Sk": 512, "Hq": 16, "Hkv": 16, "D": 64,
         "act": "f16", "causal": False, "lens": True, "packed": False},
        # a decoder's training forward, q, k and v as one projection wrote them
        {"name": "attention_causal", "op": "attention", "B": 8, "Sq": 1024, "Sk": 1024, "Hq": 25, "Hkv": 25, "D": 64,
         "act": "bf16", "causal": True, "lens": False, "packed": True},
        # its backward pass, the three gradients written as one tensor
        {"name": "attention_grad_causal", "op": "attention_grad", "B": 8, "Sq": 1024, "Sk": 1024, "Hq": 25, "Hkv": 25,
         "D": 64, "act": "bf16", "causal": True, "lens": False, "packed": True},
        # a long sequence with shared key heads
        {"name": "attention_grad_long", "op": "attention_grad", "B": 1, "Sq": 8192, "Sk": 8192, "Hq": 16, "Hkv": 4,
         "D": 128, "act": "bf16", "causal": True, "lens": False, "packed": False},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "dropout", "attention", "attention_grad"])
    if op in ("embed", "embed_grad"):
        D = rng.choice([64, 769, 1024, 1600, _log(rng, 8, 4096)])
        V = rng.choice([30522, 50257, _log(rng, 100, 130000)])
        n = _log(rng, 1, min(65536, 32768 * 1600 // D))
        while V * D > 50257 * 1600:
            V = V // 2
        table = rng.choice(["f32", "bf16", "f16"])
        act = table if rng.random() < 0.7 else rng.choice(["f32", "bf16"])
        return {"op": op, "n": n, "V": V, "D": D, "table": table, "act": act, "pad": rng.random() < 0.4}
    if op == "dropout":
        cols = rng.choice([1024, 1600, 4096, 6400, _log(rng, 1, 8192)])
        rows = _log(rng, 1, max(1, 32768 * 6400 // cols // 4))
        grad = rng.random() < 0.4
        return {"op": op, "rows": rows, "cols": cols, "act": rng.choice(["f32", "bf16", "f16"]),
                "p": rng.choice([0.0, 0.05, 0.1, 0.5, round(0.9 * rng.random(), 3)]), "residual": not grad and rng.random() < 0.5,
                "grad": grad}
    D = rng.choice([64, 64, 128, 128, 80, 40])
    Hkv = rng.choice([1, 2, 4, 8, 12, 16, 25])
    Hq = Hkv * rng.choice([1, 1, 2, 4])
    Sk = _log(rng, 1, 8192)
    Sq = rng.choice([Sk, Sk, Sk, 1, _log(rng, 1, 8192)])
    most = 8 * 8192 * 8192                                   # scores held at once by the plain form
    while Hq > Hkv and Hq * Sq * Sk > most:
        Hq = max(Hkv, Hq // 2)
    while Hq * Sq * Sk > most:
        Hq = Hkv = max(1, Hkv // 2)
    B = _log(rng, 1, max(1, min(32, most // (Hq * Sq * Sk))))
    return {"op": op, "B": B, "Sq": Sq, "Sk": Sk, "Hq": Hq, "Hkv": Hkv, "D": D, "act": rng.choice(["bf16", "bf16", "f16"]),
            "causal": rng.random() < 0.6, "lens": rng.random() < 0.4, "packed": Sq == Sk and Hq == Hkv and rng.random() < 0.5}


# --------------------------------------------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 17)
    return g


def _randn(g, shape, dtype, sigma=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(sigma).to(dtype)


def _embed_scale(case):
    return math.sqrt(case["D"])


def _embed_inputs(case, seed):
    """Token ids by a power law (the k-th most frequent id has a share of about 1 / k), spread over the vocabulary; with
    `pad`, the last fifth of the list is the padding id 0."""
    g = _gen(seed)
    n, V, D = case["n"], case["V"], case["D"]
    rank = torch.exp(torch.rand(n, generator=g, device=DEV, dtype=torch.float64) * math.log(V)).long().sub_(1).clamp_(0, V - 1)
    stride = next(s for s in range(9973, 9973 + V + 1) if math.gcd(s, V) == 1)
    tokens = rank * stride % V
    if case["pad"]:
        tokens[n - n // 5:] = 0
    tokens = tokens.to(torch.int32)
    if case["op"] == "embed":
        return tokens, _randn(g, (V, D), TORCH[case["table"]], 0.02)
    return tokens, _randn(g, (n, D), TORCH[case["act"]], 1e-3)


def _lens(case):
    """(query lengths, key lengths) of the batch, or None: between a tenth of the length and all of it, and one sequence
    of the batch (where it has several) empty.  They go by the case alone."""
    if not case["lens"]:
        return None
    r = random.Random(case["Sq"] * 1000003 + case["Sk"] * 101 + case["B"])
    frac = [r.uniform(0.1, 1.0) for _ in range(case["B"])]
    if case["B"] > 2:
        frac[case["B"] // 2] = 0.0
    return ([int(math.ceil(f * case["Sq"])) for f in frac], [int(math.ceil(f * case["Sk"])) for f in frac])


def _attention_inputs(case, seed):
    """q [B, Sq, Hq, D], k and v [B, Sk, Hkv, D] (views of one tensor with `packed`), dout, and the lengths."""
    g = _gen(seed)
    B, Sq, Sk, Hq, Hkv, D, dt = (case[x] for x in ("B", "Sq", "Sk", "Hq", "Hkv", "D", "act"))
    if case["packed"]:
        q, k, v = _randn(g, (B, Sq, 3, Hq, D), TORCH[dt]).unbind(2)
    else:
        q = _randn(g, (B, Sq, Hq, D), TORCH[dt])
        k, v = _randn(g, (B, Sk, Hkv, D), TORCH[dt]), _randn(g, (B, Sk, Hkv, D), TORCH[dt])
    dout = _randn(g, (B, Sq, Hq, D), TORCH[dt]) if case["op"] == "attention_grad" else None
    lens = _lens(case)
    if lens is not None:
        lens = tuple(torch.tensor(x, dtype=torch.int32, device=DEV) for x in lens)
    return q, k, v, dout, lens


def prepare(case, seed):
    s = dict(case)
    if own:
        from paper_2605_01989_b200 import binding
        s["dblp"] = binding
    if case["op"] in ("embed", "embed_grad"):
        n, V, D = case["n"], case["V"], case["D"]
        s["tokens"], s["data"] = _embed_inputs(case, seed)
        s["padding"] = 0 if case["pad"] else -1
        s["scale"] = _embed_scale(case)
        if case["op"] == "embed":
            s["out"] = torch.empty((n, D), dtype=TORCH[case["act"]], device=DEV)
        else:
            s["out"] = torch.empty((V, D), dtype=TORCH[case["table"]], device=DEV)
            if own:
                s["ws"] = torch.empty(s["dblp"].dblp_embed_grad_workspace_bytes(n, V, D), dtype=torch.uint8, device=DEV)
    elif case["op"] == "dropout":
        g = _gen(seed)
        s["x"] = _randn(g, (case["rows"], case["cols"]), TORCH[case["act"]])
        s["res"] = _randn(g, (case["rows"], case["cols"]), TORCH[case["act"]]) if case["residual"] else None
        s["out"] = torch.empty_like(s["x"])
        s["key"], s["step"], s["site"] = seed * 2654435761 + 12345, seed % 1000, 3
    else:
        s["q"], s["k"], s["v"], s["dout"], s["len"] = _attention_inputs(case, seed)
        q, k = s["q"], s["k"]
        s["out"] = torch.empty(q.shape, dtype=q.dtype, device=DEV)
        s["lse"] = torch.empty((case["B"], case["Hq"], case["Sq"]), dtype=torch.float32, device=DEV)
        if case["op"] == "attention_grad":
            s["out"], s["lse"] = _plain_attention(s)
            if case["packed"]:
                s["dq"], s["dk"], s["dv"] = torch.empty((case["B"], case["Sq"], 3, case["Hq"], case["D"]), dtype=q.dtype,
                                                        device=DEV).unbind(2)
            else:
                s["dq"], s["dk"], s["dv"] = (torch.empty(t.shape, dtype=t.dtype, device=DEV) for t in (q, k, k))
        if own:
            fwd, bwd = s["dblp"].dblp_attention_workspace_bytes(q, k, causal=case["causal"])
            s["ws"] = torch.empty(bwd if case["op"] == "attention_grad" else fwd, dtype=torch.uint8, device=DEV)
    return s


# --------------------------------------------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else PLAIN[s["op"]](s)


def _run_own(s):
    d = s["dblp"]
    if s["op"] == "embed":
        d.dblp_embed(s["data"], s["tokens"], s["out"], scale=s["scale"], padding=s["padding"])
        return s["out"]
    if s["op"] == "embed_grad":
        d.dblp_embed_grad(s["data"], s["tokens"], s["out"], s["ws"], scale=s["scale"], padding=s["padding"])
        return s["out"]
    if s["op"] == "dropout":
        if s["grad"]:
            d.dblp_dropout_grad(s["x"], s["out"], s["p"], s["key"], s["step"], s["site"])
        else:
            d.dblp_dropout(s["x"], s["out"], s["p"], s["key"], s["step"], s["site"], residual=s["res"])
        return s["out"]
    ql, kl = s["len"] if s["len"] is not None else (None, None)
    if s["op"] == "attention":
        d.dblp_attention(s["q"], s["k"], s["v"], s["out"], s["lse"], s["ws"], causal=s["causal"], q_lens=ql, k_lens=kl)
        return {"out": s["out"], "lse": s["lse"]}
    d.dblp_attention_grad(s["q"], s["k"], s["v"], s["out"], s["dout"], s["lse"], s["dq"], s["dk"], s["dv"], s["ws"],
                          causal=s["causal"], q_lens=ql, k_lens=kl)
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _plain_embed(s):
    tok = s["tokens"].long()
    keep = (tok != s["padding"]).unsqueeze(1)
    return torch.where(keep, s["data"][tok].float() * s["scale"], 0.0).to(s["out"].dtype)


def _plain_embed_grad(s):
    tok = s["tokens"].long()
    live = (tok != s["padding"]).unsqueeze(1)
    acc = torch.zeros((s["V"], s["D"]), dtype=torch.float32, device=DEV)
    acc.index_add_(0, tok, torch.where(live, s["data"].float(), 0.0))
    return (acc * s["scale"]).to(s["out"].dtype)


def _philox_words(n_groups, key, step, site):
    """Philox4x32-10 of counters (group, purpose | site << 8, step): four 32-bit words per group, in int64 tensors
    (products wrap modulo 2^64, which keeps their low and high 32-bit halves)."""
    mask = 0xFFFFFFFF
    g = torch.arange(n_groups, dtype=torch.int64, device=DEV)
    c0, c1 = g & mask, g >> 32
    c2, c3 = torch.full_like(g, PHILOX_STREAM | site << 8), torch.full_like(g, step)
    k0, k1 = key & mask, key >> 32 & mask
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (p1 >> 32 & mask) ^ c1 ^ k0, p1 & mask, (p0 >> 32 & mask) ^ c3 ^ k1, p0 & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return torch.stack((c0, c1, c2, c3), dim=1)


def _plain_dropout(s):
    """Element i draws half i % 2 of word i % 8 // 2 of group i // 8; it is dropped iff the 16 bits are below
    floor(p 65536), and kept elements are scaled by the inverse of the share that is kept."""
    x = s["x"]
    t = math.floor(s["p"] * 65536)
    words = _philox_words((x.numel() + 7) // 8, s["key"], s["step"], s["site"])
    u = torch.stack((words & 0xFFFF, words >> 16), dim=2).reshape(-1)[:x.numel()].reshape(x.shape)
    y = torch.where(u >= t, x.float() * (65536.0 / (65536 - t)), 0.0)
    if s["res"] is not None:
        y = y + s["res"].float()
    return y.to(x.dtype)


def _visible(s):
    """[B or 1, 1, Sq, Sk]: which key a query sees.  With `causal`, query i of a sequence of lq queries and lk keys sees
    keys 0 .. i + lk - lq."""
    Sq, Sk = s["Sq"], s["Sk"]
    i, j = torch.arange(Sq, device=DEV).view(1, 1, Sq, 1), torch.arange(Sk, device=DEV).view(1, 1, 1, Sk)
    if s["len"] is None:
        return j <= i + (Sk - Sq) if s["causal"] else torch.ones((1, 1, Sq, Sk), dtype=torch.bool, device=DEV)
    lq, lk = (t.long().view(-1, 1, 1, 1) for t in s["len"])
    seen = (i < lq) & (j < lk)
    return seen & (j <= i + lk - lq) if s["causal"] else seen


def _heads_first(s, *names):
    """The named tensors as [B, Hq, S, D] in 32 bits, shared heads repeated."""
    rep = s["Hq"] // s["Hkv"]
    return [s[n].float().transpose(1, 2).repeat_interleave(rep if n in ("k", "v") else 1, dim=1) for n in names]


def _plain_attention(s):
    q, k, v = _heads_first(s, "q", "k", "v")
    x = (q @ k.transpose(2, 3)).mul_(1.0 / math.sqrt(s["D"])).masked_fill_(~_visible(s), -math.inf)
    m = x.amax(dim=3, keepdim=True)
    m = torch.where(torch.isinf(m), 0.0, m)
    p = x.sub_(m).exp_()
    total = p.sum(dim=3, keepdim=True)
    out = (p @ v) / torch.where(total > 0, total, 1.0)
    lse = (m + total.log()).squeeze(3)
    return out.transpose(1, 2).to(s["q"].dtype).contiguous(), lse


def _plain_attention_pass(s):
    out, lse = _plain_attention(s)
    return {"out": out, "lse": lse}


def _plain_attention_grad(s):
    scale = 1.0 / math.sqrt(s["D"])
    q, k, v, out, dout = _heads_first(s, "q", "k", "v", "out", "dout")
    lse = torch.where(torch.isinf(s["lse"]), 0.0, s["lse"]).unsqueeze(3)
    p = (q @ k.transpose(2, 3)).mul_(scale).sub_(lse).exp_().masked_fill_(~_visible(s), 0.0)
    dv = p.transpose(2, 3) @ dout
    ds = (dout @ v.transpose(2, 3)).sub_((dout * out).sum(dim=3, keepdim=True)).mul_(p)
    dq, dk = ds @ k * scale, ds.transpose(2, 3) @ q * scale
    dk, dv = (t.view(s["B"], s["Hkv"], -1, s["Sk"], s["D"]).sum(dim=2) for t in (dk, dv))
    return {n: t.transpose(1, 2).to(s["q"].dtype).contiguous() for n, t in (("dq", dq), ("dk", dk), ("dv", dv))}


PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "dropout": _plain_dropout,
         "attention": _plain_attention_pass, "attention_grad": _plain_attention_grad}


# --------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------------------------------------------
def _pairs(case):
    """(query, key) pairs that are not masked, over the batch, for one head."""
    lens = _lens(case)
    total = 0
    for b in range(case["B"]):
        lq, lk = (case["Sq"], case["Sk"]) if lens is None else (lens[0][b], lens[1][b])
        if not case["causal"]:
            total += lq * lk
            continue
        first = max(0, lq - lk)                             # earlier queries see nothing
        n = lq - first
        total += n * (first + lk - lq + 1) + n * (n - 1) // 2
    return total


def _distinct(case):
    """Expected number of different rows that a lookup reads under the power law of the token ids."""
    n, V = case["n"] - (case["n"] // 5 if case["pad"] else 0), case["V"]
    share = np.diff(np.log(np.arange(1, V + 1))) / math.log(V)
    return float(np.sum(-np.expm1(n * np.log1p(-share))))


def work(case):
    if case["op"] in ("embed", "embed_grad"):
        n, V, D = case["n"], case["V"], case["D"]
        tb, ab = BYTES[case["table"]], BYTES[case["act"]]
        if case["op"] == "embed":
            return {"bytes": 4 * n + n * D * ab + _distinct(case) * D * tb, "flops": n * D}
        return {"bytes": 4 * n + n * D * ab + V * D * tb, "flops": n * D + V * D}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * BYTES[case["act"]] * (3 if case["residual"] else 2), "flops": n * (3 if case["residual"] else 2)}
    B, Sq, Sk, Hq, Hkv, D = (case[x] for x in ("B", "Sq", "Sk", "Hq", "Hkv", "D"))
    q, kv, stat = B * Sq * Hq * D * 2, B * Sk * Hkv * D * 2, B * Hq * Sq * 4
    if case["op"] == "attention":
        return {"bytes": 2 * q + 2 * kv + stat, "flops": 4 * D * Hq * _pairs(case)}
    return {"bytes": 4 * q + 4 * kv + stat, "flops": 10 * D * Hq * _pairs(case)}


# --------------------------------------------------------------------------------------------------------------
# The results in 64 bits, from the definitions
# --------------------------------------------------------------------------------------------------------------
def _exact_embed(case, seed):
    tokens, data = _embed_inputs(case, seed)
    pad = 0 if case["pad"] else -1
    if case["op"] == "embed":
        out = data.double().index_select(0, tokens.long()) * _embed_scale(case)
        out[tokens == pad] = 0
        return out
    live = (tokens != pad).nonzero().squeeze(1)
    order = live[torch.argsort(tokens[live].long(), stable=True)]
    ids, counts = torch.unique_consecutive(tokens[order].long(), return_counts=True)
    sums = torch.cat((torch.zeros((1, case["D"]), dtype=torch.float64, device=DEV), data[order].double().cumsum(0)))
    ends = counts.cumsum(0)
    out = torch.zeros((case["V"], case["D"]), dtype=torch.float64, device=DEV)
    out[ids] = (sums[ends] - sums[ends - counts]) * _embed_scale(case)
    return out


def _exact_dropout(case, seed):
    s = prepare({**case, "name": ""}, seed)
    n, t = s["x"].numel(), int(s["p"] * 65536)
    g = np.arange((n + 7) // 8, dtype=np.uint64)
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [g & low, g >> sh, np.full_like(g, PHILOX_STREAM + 256 * s["site"]), np.full_like(g, s["step"])]
    key = [s["key"] % 2 ** 32, s["key"] // 2 ** 32 % 2 ** 32]
    for r in range(10):
        k0, k1 = ((k + r * w) % 2 ** 32 for k, w in zip(key, (0x9E3779B9, 0xBB67AE85)))
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> sh) ^ c[1] ^ np.uint64(k0), b & low, (a >> sh) ^ c[3] ^ np.uint64(k1), a & low]
    u = np.stack([w >> np.uint64(16 * h) & np.uint64(0xFFFF) for w in c for h in (0, 1)], axis=1).reshape(-1)[:n]
    keep = torch.from_numpy((u >= np.uint64(t)).astype(np.float64)).to(DEV).view(s["x"].shape)
    y = keep * s["x"].double() / (1 - t / 65536) if t < 65536 else keep
    return y if s["res"] is None else y + s["res"].double()


def _exact_attention(case, seed):
    """Head by head: softmax over the visible keys and, for the gradient, its derivative with the given out and lse."""
    q, k, v, dout, lens = _attention_inputs(case, seed)
    B, Sq, Sk, Hq, Hkv, D = (case[x] for x in ("B", "Sq", "Sk", "Hq", "Hkv", "D"))
    grad = case["op"] == "attention_grad"
    if grad:
        s = prepare({**case, "name": ""}, seed)
        given_out, given_lse = s["out"], s["lse"]
    f64 = {"dtype": torch.float64, "device": DEV}
    res = ({"dq": torch.zeros((B, Sq, Hq, D), **f64), "dk": torch.zeros((B, Sk, Hkv, D), **f64),
            "dv": torch.zeros((B, Sk, Hkv, D), **f64)} if grad else
           {"out": torch.zeros((B, Sq, Hq, D), **f64), "lse": torch.full((B, Hq, Sq), -math.inf, **f64)})
    for b in range(B):
        lq, lk = (Sq, Sk) if lens is None else (int(lens[0][b]), int(lens[1][b]))
        if lq == 0 or lk == 0:
            continue
        hidden = None
        if case["causal"]:
            hidden = torch.ones((lq, lk), dtype=torch.bool, device=DEV).triu(lk - lq + 1)
        for h in range(Hq):
            hk = h * Hkv // Hq
            Q, K, V = q[b, :lq, h].double(), k[b, :lk, hk].double(), v[b, :lk, hk].double()
            S = torch.mm(Q, K.T) / math.sqrt(D)
            if hidden is not None:
                S[hidden] = -math.inf
            if not grad:
                L = torch.logsumexp(S, dim=1)
                P = torch.exp(S - L.clamp_min(-1e300).unsqueeze(1))
                res["out"][b, :lq, h] = torch.mm(P, V)
                res["lse"][b, h, :lq] = L
                continue
            dO, O = dout[b, :lq, h].double(), given_out[b, :lq, h].double()
            P = torch.exp(S - given_lse[b, h, :lq].double().clamp_min(-1e300).unsqueeze(1))
            dS = P * (torch.mm(dO, V.T) - torch.sum(dO * O, dim=1, keepdim=True)) / math.sqrt(D)
            res["dq"][b, :lq, h] = torch.mm(dS, K)
            res["dk"][b, :lk, hk] += torch.mm(dS.T, Q)
            res["dv"][b, :lk, hk] += torch.mm(P.T, dO)
    return res


def exact(case, seed):
    if case["op"] in ("embed", "embed_grad"):
        return _exact_embed(case, seed)
    if case["op"] == "dropout":
        return _exact_dropout(case, seed) if case["rows"] * case["cols"] <= 1 << 25 else None
    return _exact_attention(case, seed)
