"""Worker-side operators against plain 64-bit statements of their formulas.

Tolerances follow from the formats.  u = half a unit in the last place of the tensor's type, relative (2^-8 bf16, 2^-11
f16, 2^-24 f32).  A value that is rounded once to that type is off by at most u |value|; a rounded factor inside a sum by
at most u times the sum of absolute terms; an fp32 sum of m terms by at most m 2^-24 times that sum.  EXP = 2^-11 bounds
the relative error of a probability: scores reach about 30 in fp32, plus the exponential's own error."""
import math
import os

import numpy as np
import pytest
import torch

from paper_2605_01989_b200 import binding as dblp

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
EXP = 2.0 ** -11
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def randn(shape, dtype, seed, sigma=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * sigma).to(dtype)


def within(got, want, tol, what):
    assert torch.isfinite(got.double()).all(), what
    worst = ((got.double() - want).abs() - tol).max().item() if want.numel() else -1
    assert worst <= 0, "%s: beyond the tolerance by %g" % (what, worst)


def bits(t):
    return t.contiguous().view(torch.uint8)


# ---- embedding -------------------------------------------------------------------------------------------------------
def token_list(n, rows, kind, seed, dtype=torch.int32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if kind == "same":
        t = torch.full((n,), rows // 2, device=DEV)
    elif kind == "each":
        t = torch.arange(n, device=DEV) % rows
    elif kind == "power":
        t = (torch.rand(n, generator=g, device=DEV, dtype=torch.float64) * math.log(rows)).exp().long() - 1
    elif kind == "outside":
        t = torch.randint(-3, rows + 3, (n,), generator=g, device=DEV)
    else:
        t = torch.randint(0, rows, (n,), generator=g, device=DEV)
    return t.to(dtype)


@pytest.mark.parametrize("n,rows,width", [(1, 1, 1), (1, 50257, 1600), (5, 7, 8), (33, 100, 769), (1000, 300, 40), (257, 30522, 1024)])
@pytest.mark.parametrize("table_dtype,out_dtype", [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (BF16, F32)])
def test_embed_is_the_rounded_product(n, rows, width, table_dtype, out_dtype):
    table = randn((rows, width), table_dtype, 1)
    tokens = token_list(n, rows, "any", 2, torch.int64 if n % 2 else torch.int32)
    out = torch.full((n, width), 7.0, dtype=out_dtype, device=DEV)
    scale = math.sqrt(width)
    dblp.dblp_embed(table, tokens, out, scale=scale)
    want = (table[tokens.long()].double() * float(np.float32(scale))).float().to(out_dtype)
    assert torch.equal(bits(out), bits(want))


def test_embed_padding_bad_tokens_and_strides():
    rows, width, n = 50, 24, 400
    wide = randn((rows, 40), BF16, 3)
    tokens = token_list(n, rows, "outside", 4, torch.int64)
    buf = torch.full((n, 48), 9.0, dtype=BF16, device=DEV)
    bad = torch.zeros(1, dtype=torch.int64, device=DEV)
    for first in (0, 1):                               # column 1: rows that no vector load may touch
        dblp.dblp_embed(wide[:, first:first + width], tokens, buf[:, 8:8 + width], padding=4, bad_tokens=bad)
        live = (tokens >= 0) & (tokens < rows) & (tokens != 4)
        want = torch.where(live[:, None], wide[tokens.clamp(0, rows - 1), first:first + width], 0)
        assert torch.equal(buf[:, 8:8 + width], want)
        assert (buf[:, :8] == 9).all() and (buf[:, 8 + width:] == 9).all()
    outside = int(((tokens < 0) | (tokens >= rows)).sum())
    assert outside > 0 and int(bad) == 2 * outside
    dblp.dblp_embed(wide[:, :width], tokens[:0], buf[:0, :width])              # no tokens


def embed_grad(dout, tokens, rows, dtable, **kw):
    ws = torch.empty(dblp.dblp_embed_grad_workspace_bytes(tokens.numel(), rows, dout.shape[1]) + 64, dtype=torch.uint8, device=DEV)
    ws.fill_(0xAB)                                     # contents do not matter
    dblp.dblp_embed_grad(dout, tokens, dtable, ws, **kw)
    return dtable


def grad_and_bound(dout, tokens, rows, scale, out_dtype, padding=-1):
    live = (tokens >= 0) & (tokens < rows) & (tokens != padding)
    t = tokens[live].long()
    width = dout.shape[1]
    total = torch.zeros((rows, width), dtype=torch.float64, device=DEV).index_add_(0, t, dout[live].double())
    mass = torch.zeros((rows, width), dtype=torch.float64, device=DEV).index_add_(0, t, dout[live].double().abs())
    count = torch.bincount(t, minlength=rows).double()[:, None]
    want = total * float(np.float32(scale))
    tol = (count + 2) * 2.0 ** -24 * mass * scale + U[out_dtype] * want.abs() * 1.01
    if out_dtype == F16:
        tol = tol + 2.0 ** -25                         # half the spacing of f16's smallest numbers
    return want, tol


@pytest.mark.parametrize("n,rows,width,kind", [
    (0, 40, 16, "any"), (1, 1, 1, "same"), (1, 50257, 1600, "any"), (31, 64, 8, "any"), (32, 64, 264, "same"), (33, 33, 40, "each"),
    (300, 5, 769, "any"), (1000, 1000, 1024, "power"), (4097, 30522, 256, "power"), (5000, 1, 72, "same"), (8192, 70000, 64, "power"),
    (8193, 255, 64, "power"), (20000, 256, 48, "any"), (40000, 65536, 32, "power"), (30000, 300000, 8, "any"), (20001, 90, 33, "outside"),
    (9000, 11, 264, "same")])
@pytest.mark.parametrize("dout_dtype,table_dtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16)])
def test_embed_grad_sums_every_occurrence(n, rows, width, kind, dout_dtype, table_dtype):
    dout = randn((n, width), dout_dtype, n + rows)
    tokens = token_list(n, rows, kind, n, torch.int64 if rows % 2 else torch.int32)
    scale = 0.75
    dtable = torch.full((rows, width), 5.0, dtype=table_dtype, device=DEV)
    bad = torch.zeros(1, dtype=torch.int64, device=DEV)
    embed_grad(dout, tokens, rows, dtable, scale=scale, padding=2, bad_tokens=bad)
    want, tol = grad_and_bound(dout, tokens, rows, scale, table_dtype, padding=2)
    within(dtable, want, tol, "dtable")
    assert int(bad) == int(((tokens < 0) | (tokens >= rows)).sum())
    again = embed_grad(dout, tokens, rows, torch.empty_like(dtable), scale=scale, padding=2)
    assert torch.equal(bits(again), bits(dtable))


@pytest.mark.parametrize("n", [1, 700, 9001])
@pytest.mark.parametrize("width", [64, 65])
def test_embed_grad_accumulates_and_keeps_strides(n, width):
    rows = 123
    dout = randn((n, width + 16), F32, 5)[:, 8:8 + width]
    tokens = token_list(n, rows, "power", 6)
    buf = randn((rows, width + 24), F32, 7)
    before = buf.clone()
    embed_grad(dout, tokens, rows, buf[:, 8:8 + width], scale=2.0, accumulate=True)
    want, tol = grad_and_bound(dout, tokens, rows, 2.0, F32)
    want = want + before[:, 8:8 + width].double()
    within(buf[:, 8:8 + width], want, tol + 2.0 ** -23 * want.abs(), "accumulated")
    absent = torch.bincount(tokens.long(), minlength=rows) == 0
    assert torch.equal(buf[absent], before[absent])
    assert torch.equal(buf[:, :8], before[:, :8]) and torch.equal(buf[:, 8 + width:], before[:, 8 + width:])


def test_embed_grad_is_the_difference_quotient_of_embed():
    n, rows, width, scale = 500, 60, 32, 1.5
    tokens, dout, step = token_list(n, rows, "power", 8), randn((n, width), F32, 9), randn((rows, width), F32, 10)
    dtable = embed_grad(dout, tokens, rows, torch.empty((rows, width), device=DEV), scale=scale)
    ends = []
    for sign in (1.0, -1.0):                           # the lookup is linear, so a step of any size is exact but for rounding
        out = torch.empty((n, width), device=DEV)
        dblp.dblp_embed(step * sign, tokens, out, scale=scale)
        ends.append((out.double() * dout.double()).sum())
    along = (dtable.double() * step.double()).sum()
    assert abs((ends[0] - ends[1]) / 2 - along) <= 1e-5 * (dout.double().abs().sum() * scale)


# ---- dropout ---------------------------------------------------------------------------------------------------------
def philox(c, k):
    """Philox4x32-10 in plain 64-bit arithmetic; c: four arrays or numbers, k: two numbers."""
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    c, k = [np.asarray(x, dtype=np.uint64) for x in c], [np.asarray(x, dtype=np.uint64) for x in k]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ k[0], b & low, (a >> half) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return c


def draws(n, seed, step, site, first_group=0):
    """The 16 bits of n elements from group first_group on."""
    g = np.arange((n + 7) // 8, dtype=np.uint64) + np.uint64(first_group)
    words = philox((g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), np.full_like(g, 5 | site << 8), np.full_like(g, step)),
                   (seed & 0xFFFFFFFF, seed >> 32))
    u = np.stack([x >> np.uint64(s) & np.uint64(0xFFFF) for x in words for s in (0, 16)], axis=1)
    return torch.from_numpy(u.reshape(-1)[:n].astype(np.int64)).to(DEV)


def test_the_restated_generator_gives_the_published_answers(golden_dir):
    rows = [l.split() for l in open(os.path.join(golden_dir, "philox4x32_10_kat.txt")) if l.strip() and not l.startswith("#")]
    assert len(rows) >= 3
    for row in rows:
        x = [int(w, 16) for w in row[-10:]]
        assert [int(w) for w in philox(x[:4], x[4:6])] == x[6:]


def plain_dropout(x, p, seed, step, site, residual=None):
    t = math.floor(p * 65536)
    keep = (draws(x.numel(), seed, step, site) >= t).view(x.shape)
    inv = float(np.float32(65536 / (65536 - t))) if t < 65536 else 0.0
    y = torch.where(keep, (x.double() * inv).float(), 0.0)
    if residual is not None:
        y = (y.double() + residual.double()).float()
    return y.to(x.dtype)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (1, 8), (3, 9), (7, 1601), (64, 1600), (1000, 24), (5, 100003)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout_matches_the_generator(rows, cols, dtype, p, residual):
    x = randn((rows, cols), dtype, rows * 31 + cols)
    r = randn((rows, cols), dtype, 99) if residual else None
    out = torch.full_like(x, 3.0)
    seed, step, site = 0xDEADBEEF12345678, 41, 9
    dblp.dblp_dropout(x, out, p, seed, step, site, residual=r)
    assert torch.equal(bits(out), bits(plain_dropout(x, p, seed, step, site, r)))


@pytest.mark.parametrize("cols", [24, 13, 64])
def test_dropout_strides_share_one_mask(cols):
    rows, kw = 37, dict(p=0.3, seed=5, step=6, site=7)
    for xo, oo, ro in ((0, 0, 0), (8, 16, 8), (1, 3, 2)):
        x = randn((rows, 96), BF16, 1)[:, xo:xo + cols]
        r = randn((rows, 120), BF16, 2)[:, ro:ro + cols]
        buf = torch.full((rows, 104), 4.0, dtype=BF16, device=DEV)
        dblp.dblp_dropout(x, buf[:, oo:oo + cols], residual=r, **kw)
        assert torch.equal(buf[:, oo:oo + cols], plain_dropout(x, residual=r, **kw))
        assert (buf[:, :oo] == 4).all() and (buf[:, oo + cols:] == 4).all()


def test_dropout_in_place_gradient_and_rate():
    n = 1 << 20
    x, kw = randn((1, n), F32, 3), dict(p=0.1, seed=11, step=2, site=0)
    y = torch.empty_like(x)
    dblp.dblp_dropout(x, y, **kw)
    z = x.clone()
    dblp.dblp_dropout(z, z, **kw)
    assert torch.equal(z, y)
    kept = (y != 0).double().mean().item()
    assert abs(kept - 0.9) < 5 * math.sqrt(0.09 / n)   # five standard deviations
    other = torch.empty_like(x)
    dblp.dblp_dropout(x, other, p=0.1, seed=11, step=2, site=1)
    both = ((y == 0) & (other == 0)).double().mean().item()
    assert abs(both - 0.01) < 5 * math.sqrt(0.01 / n)  # another site: another mask
    g, dx = randn((1, n), F32, 4), torch.empty_like(x)
    dblp.dblp_dropout_grad(g, dx, **kw)
    assert torch.equal(dx, plain_dropout(g, **kw))
    # linear in x, so the difference quotient along x itself is exact but for rounding
    a, b = (g.double() * y.double()).sum(), (dx.double() * x.double()).sum()
    assert abs(a - b) <= 2.0 ** -22 * (g.double() * y.double()).abs().sum()


def test_dropout_groups_beyond_32_bits():
    """Element numbers past 2^32 (a group number's high word is 0 until 2^35 elements, the offsets are not)."""
    rows, cols = 70000, 65536
    x = torch.ones((rows, cols), dtype=F16, device=DEV)
    out = torch.zeros_like(x)
    dblp.dblp_dropout(x, out, 0.5, 3, 4, 5)
    first = (2 ** 32 + 4096) // cols
    want = (draws(cols, 3, 4, 5, first * cols // 8) >= 32768).float() * 2
    assert torch.equal(out[first].float(), want)
    assert out[-1].float().mean().item() == pytest.approx(1.0, abs=0.05)


# ---- attention -------------------------------------------------------------------------------------------------------
def tensors(B, Sq, Sk, Hq, Hkv, D, dtype, layout="plain", seed=1, sigma=1.0):
    """q, k, v, dout and empty out, dq, dk, dv in one of several layouts."""
    def make(tokens, heads, k):
        full = [B, tokens, heads, D]
        if layout == "heads_first":
            return randn((B, heads, tokens, D), dtype, seed + k, sigma).transpose(1, 2)
        if layout == "tokens_first":
            return randn((tokens, B, heads, D), dtype, seed + k, sigma).transpose(0, 1)
        if layout == "wide":                           # sections of wider rows
            return randn((B, tokens, heads + 1, D + 8), dtype, seed + k, sigma)[:, :, :heads, 8:]
        return randn(full, dtype, seed + k, sigma)
    if layout == "packed":
        q, k, v = randn((B, Sq, 3, Hq, D), dtype, seed, sigma).unbind(2)
        dq, dk, dv = torch.full((B, Sq, 3, Hq, D), 7.0, dtype=dtype, device=DEV).unbind(2)
        return q, k, v, randn((B, Sq, Hq, D), dtype, seed + 5), torch.full((B, Sq, Hq, D), 7.0, dtype=dtype, device=DEV), dq, dk, dv
    q, k, v, g = make(Sq, Hq, 0), make(Sk, Hkv, 1), make(Sk, Hkv, 2), make(Sq, Hq, 3)
    out, dq, dk, dv = make(Sq, Hq, 4), make(Sq, Hq, 5), make(Sk, Hkv, 6), make(Sk, Hkv, 7)
    return q, k, v, g, out, dq, dk, dv


def run_attention(q, k, v, out, causal=False, scale=None, lens=(None, None), stream=None):
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), 7.0, device=DEV)
    ws = torch.empty(dblp.dblp_attention_workspace_bytes(q, k, causal)[0], dtype=torch.uint8, device=DEV).fill_(0xFF)
    dblp.dblp_attention(q, k, v, out, lse, ws, causal=causal, scale=scale, q_lens=lens[0], k_lens=lens[1], stream=stream)
    return lse


def run_grad(q, k, v, out, g, lse, dq, dk, dv, causal=False, scale=None, lens=(None, None), stream=None):
    ws = torch.empty(dblp.dblp_attention_workspace_bytes(q, k, causal)[1], dtype=torch.uint8, device=DEV).fill_(0xFF)
    dblp.dblp_attention_grad(q, k, v, out, g, lse, dq, dk, dv, ws, causal=causal, scale=scale, q_lens=lens[0], k_lens=lens[1],
                             stream=stream)


def exact_attention(q, k, v, causal=False, scale=None, lens=(None, None)):
    """(out, lse, p, visible, score mass) in 64 bits, [B, H, ...]."""
    B, Sq, Hq, D = q.shape
    Sk, rep = k.shape[1], Hq // k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    scale = float(np.float32(scale))
    i, j = torch.arange(Sq, device=DEV).view(1, 1, Sq, 1), torch.arange(Sk, device=DEV).view(1, 1, 1, Sk)
    lq = (lens[0].long() if lens[0] is not None else torch.full((B,), Sq, device=DEV)).view(B, 1, 1, 1)
    lk = (lens[1].long() if lens[1] is not None else torch.full((B,), Sk, device=DEV)).view(B, 1, 1, 1)
    lq, lk = lq.clamp(0, Sq), lk.clamp(0, Sk)
    vis = (i < lq) & (j < lk)
    if causal:
        vis = vis & (j <= i + lk - lq)
    Q = torch.where(i.view(1, Sq, 1, 1) < lq, q.double(), 0).transpose(1, 2)
    K, V = (torch.where(j.view(1, Sk, 1, 1) < lk, t.double(), 0).transpose(1, 2).repeat_interleave(rep, 1) for t in (k, v))
    s = (Q @ K.transpose(2, 3) * scale).masked_fill(~vis, -math.inf)
    lse = torch.logsumexp(s, 3)
    p = torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)[..., None]).masked_fill(~vis, 0)
    mass = (Q.abs() @ K.abs().transpose(2, 3) * scale).amax(dim=(2, 3)).max().item() if s.numel() else 0.0
    return p @ V, lse, p, vis, mass, Q, K, V


def check_forward(q, k, v, out, lse, **kw):
    want, wlse, p, vis, mass, Q, K, V = exact_attention(q, k, v, **kw)
    u, D = U[q.dtype], q.shape[3]
    dot = 2.0 ** -24 * (D + 8) * mass                  # fp32 score error
    tol = (u + EXP + 2 * dot) * (p @ V.abs()) + u * want.abs() * 1.01 + 1e-7
    within(out.transpose(1, 2), want, tol, "out")
    empty = torch.isinf(wlse)
    assert torch.equal(torch.isinf(lse) & (lse < 0), empty)
    assert (out.transpose(1, 2)[empty] == 0).all()
    d = (lse.double() - wlse)[~empty].abs()
    assert d.numel() == 0 or (d <= 2 * dot + EXP / 2 + 2.0 ** -22 * wlse[~empty].abs()).all(), d.max().item()


def check_grad(q, k, v, out, g, lse, dq, dk, dv, scale=None, **kw):
    _, wlse, p, vis, mass, Q, K, V = exact_attention(q, k, v, scale=scale, **kw)
    u, D, B = U[q.dtype], q.shape[3], q.shape[0]
    scale = float(np.float32(D ** -0.5 if scale is None else scale))
    row = vis.any(3)[..., None]                        # rows that see nothing contribute nothing, whatever they hold
    G = torch.where(row, g.double().transpose(1, 2), 0)
    O = torch.where(row, out.double().transpose(1, 2), 0)
    s = (Q @ K.transpose(2, 3) * scale)
    given = torch.where(torch.isinf(lse), 0.0, lse.double())[..., None]
    p = torch.exp(s - given).masked_fill(~vis, 0)
    delta = (G * O).sum(3, keepdim=True)
    dp = G @ V.transpose(2, 3)
    ds = p * (dp - delta)
    dot = 2.0 ** -24 * (D + 8)
    perr = EXP + 2 * dot * mass                        # relative error of a probability
    dserr = perr * ds.abs() + p * 4 * dot * (G.abs() @ V.abs().transpose(2, 3) + (G * O).abs().sum(3, keepdim=True)) + u * ds.abs()
    group = lambda t: t.view(B, k.shape[2], -1, *t.shape[2:]).sum(2)  # noqa: E731
    checks = (("dq", dq, ds @ K * scale, dserr @ K.abs() * scale),
              ("dk", dk, group(ds.transpose(2, 3) @ Q) * scale, group(dserr.transpose(2, 3) @ Q.abs()) * scale),
              ("dv", dv, group(p.transpose(2, 3) @ G), group(((u + perr) * p).transpose(2, 3) @ G.abs())))
    for name, got, want, err in checks:
        within(got.transpose(1, 2), want, err + u * want.abs() * 1.01 + 1e-6, name)


SHAPES = [
    # B, Sq, Sk, Hq, Hkv, D, dtype, causal, lengths, layout
    (1, 1, 1, 1, 1, 8, BF16, False, None, "plain"),
    (1, 1, 1, 1, 1, 128, F16, True, None, "plain"),
    (2, 1, 1024, 5, 5, 64, BF16, True, None, "plain"),
    (2, 1, 700, 8, 2, 128, F16, False, None, "plain"),
    (3, 1, 4100, 2, 1, 64, BF16, True, ([1, 0, 1], [4100, 9, 77]), "plain"),
    (1, 3, 5000, 4, 2, 128, BF16, True, None, "heads_first"),
    (1, 700, 1, 2, 2, 64, BF16, False, None, "plain"),
    (1, 128, 128, 2, 2, 64, BF16, False, None, "plain"),
    (1, 128, 128, 2, 2, 64, BF16, True, None, "packed"),
    (1, 256, 256, 1, 1, 128, BF16, True, None, "plain"),
    (2, 129, 257, 4, 2, 64, BF16, True, None, "plain"),
    (2, 257, 129, 2, 2, 64, F16, True, None, "plain"),          # the first queries see nothing
    (1, 500, 20, 2, 1, 128, BF16, True, None, "plain"),
    (2, 200, 200, 3, 3, 40, F16, True, None, "packed"),
    (1, 300, 300, 6, 1, 128, BF16, True, None, "heads_first"),
    (2, 190, 333, 4, 4, 80, BF16, False, None, "wide"),
    (2, 333, 190, 4, 2, 96, F16, False, None, "tokens_first"),
    (1, 1000, 1000, 2, 2, 72, BF16, True, None, "packed"),
    (3, 65, 190, 2, 1, 96, BF16, False, ([65, 0, 7], [190, 33, 0]), "plain"),
    (4, 200, 300, 2, 2, 64, BF16, True, ([200, 150, 128, 1], [300, 100, 128, 1]), "plain"),
    (5, 512, 512, 2, 2, 64, F16, False, ([512, 300, 0, 129, 1000], [512, 300, 0, 129, -4]), "packed"),
    (2, 640, 640, 4, 2, 128, F16, True, ([640, 385], [640, 385]), "plain"),
    (1, 1500, 1500, 3, 1, 64, BF16, False, None, "plain"),
    (1, 2100, 2100, 2, 1, 128, BF16, True, None, "plain"),
    (9, 130, 130, 25, 25, 64, BF16, True, None, "plain"),
    (40, 64, 64, 16, 4, 64, F16, False, None, "plain"),
]


FEW = [
    (1, 1, 200, 4, 1, 40, F16, True, None, "plain"),
    (2, 2, 300, 4, 2, 64, BF16, True, None, "heads_first"),
    (1, 4, 1000, 2, 2, 96, BF16, True, None, "wide"),
    (1, 4, 3, 2, 2, 64, BF16, True, None, "plain"),             # the first query sees nothing
    (3, 2, 150, 2, 1, 128, BF16, False, ([2, 0, 1], [150, 60, 0]), "plain"),
    (2, 3, 9000, 1, 1, 8, F16, True, ([3, 2], [9000, 4097]), "tokens_first"),
    (1, 1, 5000, 8, 1, 128, BF16, True, None, "plain"),
    (1, 8, 600, 1, 1, 64, BF16, True, None, "plain"),
    (1, 9, 600, 1, 1, 64, BF16, True, None, "plain"),
    (33, 1, 70, 25, 25, 64, BF16, True, None, "plain"),
]
SHAPES += FEW


def lengths(lens):
    return (None, None) if lens is None else tuple(torch.tensor(x, dtype=torch.int32, device=DEV) for x in lens)


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hkv,D,dtype,causal,lens,layout", SHAPES)
def test_attention_and_its_gradient(B, Sq, Sk, Hq, Hkv, D, dtype, causal, lens, layout):
    q, k, v, g, out, dq, dk, dv = tensors(B, Sq, Sk, Hq, Hkv, D, dtype, layout)
    kw = dict(causal=causal, lens=lengths(lens))
    lse = run_attention(q, k, v, out, **kw)
    check_forward(q, k, v, out, lse, **kw)
    run_grad(q, k, v, out, g, lse, dq, dk, dv, **kw)
    check_grad(q, k, v, out, g, lse, dq, dk, dv, **kw)
    first = [t.clone() for t in (out, lse, dq, dk, dv)]
    lse = run_attention(q, k, v, out, **kw)
    run_grad(q, k, v, out, g, lse, dq, dk, dv, **kw)
    for a, b in zip(first, (out, lse, dq, dk, dv)):
        assert torch.equal(bits(a), bits(b.clone()))


@pytest.mark.parametrize("dtype,scale,sigma", [(BF16, 0.125, 8.0), (F16, 4.0, 1.0), (BF16, 1e-4, 1.0)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_with_steep_and_flat_scores(dtype, scale, sigma, D):
    """Steep: nearly one-hot rows whose running maximum jumps; flat: all probabilities alike."""
    q, k, v, g, out, dq, dk, dv = tensors(1, 300, 400, 2, 2, D, dtype, sigma=sigma)
    q, k = q.clone(), k.clone()
    k[:, 350] *= 3                                     # a late key that dominates
    lse = run_attention(q, k, v, out, causal=True, scale=scale)
    want, wlse, p, vis, mass, Q, K, V = exact_attention(q, k, v, causal=True, scale=scale)
    dot = 2.0 ** -24 * (D + 8) * mass
    u = U[dtype]
    assert ((lse.double() - wlse).abs() <= 2 * dot + EXP / 2 + 2.0 ** -22 * wlse.abs()).all()
    within(out.transpose(1, 2), want, (u + EXP + 2 * dot) * (p @ V.abs()) + u * want.abs() * 1.01 + 1e-7, "out")
    run_grad(q, k, v, out, g, lse, dq, dk, dv, causal=True, scale=scale)
    check_grad(q, k, v, out, g, lse, dq, dk, dv, scale=scale, causal=True)


@pytest.mark.parametrize("D", [64, 96])
@pytest.mark.parametrize("causal", [False, True])
def test_what_lies_beyond_the_lengths_is_never_used(causal, D):
    B, Sq, Sk, Hq, Hkv = 3, 300, 300, 4, 2
    lens = lengths(([300, 130, 7], [290, 130, 40]))
    q, k, v, g, out, dq, dk, dv = tensors(B, Sq, Sk, Hq, Hkv, D, BF16)
    got = []
    for poison in (0.0, math.nan, math.inf, torch.finfo(BF16).min):
        for t, n in ((q, lens[0]), (g, lens[0]), (k, lens[1]), (v, lens[1])):
            for b in range(B):
                t[b, int(n[b]):] = poison
        lse = run_attention(q, k, v, out, causal=causal, lens=lens)
        o2 = out.clone()
        for b in range(B):
            o2[b, int(lens[0][b]):] = poison
        run_grad(q, k, v, o2, g, lse, dq, dk, dv, causal=causal, lens=lens)
        got.append([t.clone() for t in (out, lse, dq, dk, dv)])
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(bits(a), bits(b))
    for b in range(B):
        assert (dq[b, int(lens[0][b]):] == 0).all() and (dk[b, int(lens[1][b]):] == 0).all() and (dv[b, int(lens[1][b]):] == 0).all()


def test_outputs_keep_to_their_sections():
    B, S, H, D = 2, 150, 3, 40
    q, k, v, g = (randn((B, S, H, D), BF16, i) for i in range(4))
    bufs = [torch.full((B, S, H, 64), 9.0, dtype=BF16, device=DEV) for _ in range(4)]
    out, dq, dk, dv = (b[..., 8:8 + D] for b in bufs)
    lse = run_attention(q, k, v, out, causal=True)
    run_grad(q, k, v, out, g, lse, dq, dk, dv, causal=True)
    check_grad(q, k, v, out, g, lse, dq, dk, dv, causal=True)
    for b in bufs:
        assert (b[..., :8] == 9).all() and (b[..., 8 + D:] == 9).all()


def test_inputs_broadcast_over_heads_and_batch():
    B, S, H, D = 2, 200, 4, 64
    q, g = randn((B, S, H, D), BF16, 1), randn((1, S, 1, D), BF16, 4).expand(B, S, H, D)
    k, v = (randn((1, S, 1, D), BF16, i).expand(B, S, H, D) for i in (2, 3))
    out, dq, dk, dv = (torch.empty((B, S, H, D), dtype=BF16, device=DEV) for _ in range(4))
    lse = run_attention(q, k, v, out)
    check_forward(q, k, v, out, lse)
    run_grad(q, k, v, out, g, lse, dq, dk, dv)         # one gradient per use; the caller sums what it shares
    check_grad(q, k, v, out, g, lse, dq, dk, dv)


def test_key_offsets_beyond_32_bits():
    B, S, H, D = 1, 300, 1, 64
    q, g = randn((B, S, H, D), BF16, 1), randn((B, S, H, D), BF16, 2)
    far = torch.zeros((S, 1 << 23), dtype=BF16, device=DEV)
    far[:, :3 * D] = randn((S, 3 * D), BF16, 3)
    k, v = far[:, :D].view(B, S, H, D), far[:, D:2 * D].view(B, S, H, D)
    out, dq, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
    dk = far[:, 2 * D:3 * D].view(B, S, H, D)
    lse = run_attention(q, k, v, out, causal=True)
    check_forward(q, k, v, out, lse, causal=True)
    run_grad(q, k, v, out, g, lse, dq, dk, dv, causal=True)
    check_grad(q, k, v, out, g, lse, dq, dk, dv, causal=True)


def test_attention_on_another_stream():
    q, k, v, g, out, dq, dk, dv = tensors(2, 400, 400, 4, 4, 64, BF16)
    lse0 = run_attention(q, k, v, out, causal=True)
    run_grad(q, k, v, out, g, lse0, dq, dk, dv, causal=True)
    want = [t.clone() for t in (out, lse0, dq, dk, dv)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [torch.empty_like(t) for t in (out, dq, dk, dv)]
        lse = run_attention(q, k, v, got[0], causal=True)
        run_grad(q, k, v, got[0], g, lse, *got[1:], causal=True)
    s.synchronize()
    for a, b in zip(want, (got[0], lse, *got[1:])):
        assert torch.equal(bits(a), bits(b))


def test_gradient_is_the_difference_quotient():
    """Central differences of the 64-bit loss sum(dout * attention) along random directions, against the returned gradients."""
    B, S, H, D, eps = 1, 150, 2, 64, 1e-4
    q, k, v, g, out, dq, dk, dv = tensors(B, S, S, H, H, D, F16)
    lse = run_attention(q, k, v, out, causal=True)
    run_grad(q, k, v, out, g, lse, dq, dk, dv, causal=True)

    def loss(x):
        return (exact_attention(*x, causal=True)[0] * g.double().transpose(1, 2)).sum().item()

    base = [t.double() for t in (q, k, v)]
    for at, grad in enumerate((dq, dk, dv)):
        d = randn((B, S, H, D), F32, 50 + at).double()
        ends = [loss([t + (sign * eps * d if n == at else 0) for n, t in enumerate(base)]) for sign in (1, -1)]
        along = (grad.double() * d).sum().item()
        # each of the n gradient elements is off by about u of its size with a random sign; 8 standard deviations
        noise = 8 * 2 * U[F16] * (grad.double() * d).square().sum().sqrt().item() + 1e-4 * (grad.double() * d).abs().sum().item()
        assert abs((ends[0] - ends[1]) / (2 * eps) - along) <= noise


@pytest.mark.parametrize("Sq", [1, 260])
def test_attention_without_lse_and_without_a_workspace(Sq):
    q, k, v, g, out, *_ = tensors(1, Sq, 700, 2, 2, 64, BF16)
    run_attention(q, k, v, out)
    want = out.clone()
    need = dblp.dblp_attention_workspace_bytes(q, k)[0]
    assert (need > 0) == (Sq == 1)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    out.fill_(7.0)
    dblp.dblp_attention(q, k, v, out, None, ws)
    assert torch.equal(out, want)
    if need:
        with pytest.raises(dblp.DblpError, match="workspace"):
            dblp.dblp_attention(q, k, v, out)


def test_calls_replay_from_a_graph():
    q, k, v, g, out, dq, dk, dv = tensors(2, 200, 200, 2, 2, 64, BF16)
    one = torch.empty_like(q[:, :1])
    lse, lse1 = run_attention(q, k, v, out, causal=True), run_attention(q[:, :1], k, v, one)
    run_grad(q, k, v, out, g, lse, dq, dk, dv, causal=True)
    tokens, dout = token_list(9000, 500, "power", 3), randn((9000, 64), F32, 4)
    table = torch.empty((500, 64), device=DEV)
    ws = torch.empty(max(dblp.dblp_embed_grad_workspace_bytes(9000, 500, 64), *dblp.dblp_attention_workspace_bytes(q, k, True)), dtype=torch.uint8, device=DEV)
    ws1 = torch.empty(dblp.dblp_attention_workspace_bytes(q[:, :1], k)[0], dtype=torch.uint8, device=DEV)

    def calls():
        dblp.dblp_attention(q, k, v, out, lse, ws, causal=True)
        dblp.dblp_attention_grad(q, k, v, out, g, lse, dq, dk, dv, ws, causal=True)
        dblp.dblp_embed_grad(dout, tokens, table, ws)
        dblp.dblp_attention(q[:, :1], k, v, one, lse1, ws1)

    calls()
    want = [t.clone() for t in (out, lse, dq, dk, dv, table, one, lse1)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for t in (out, lse, dq, dk, dv, table, one, lse1):
        t.fill_(3.0)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, (out, lse, dq, dk, dv, table, one, lse1)):
        assert torch.equal(bits(a), bits(b.clone()))


def test_no_wait_ran_out():
    assert dblp.dblp_wait_timeouts() == 0


@pytest.mark.parametrize("first", [0, 1, 31, 32, 33, 15 * 32, 16 * 32 - 1, 16 * 32 + 1, 63 * 32, 64 * 32, 64 * 32 + 1, 64 * 32 - 1])
@pytest.mark.parametrize("length", [1, 32, 33, 15 * 32, 16 * 32, 16 * 32 + 40, 17 * 32, 63 * 32, 64 * 32, 64 * 32 + 40, 65 * 32, 130 * 32, 200 * 32 + 5])
def test_embed_grad_runs_of_every_length_at_every_place(first, length):
    """One long run between two others, beginning and ending around tile boundaries of the sorted list."""
    rows, width = 5, 16
    tokens = torch.cat([torch.full((c,), v, dtype=torch.int32, device=DEV) for v, c in ((1, first), (2, length), (4, 50))])
    tokens = tokens[torch.randperm(tokens.numel(), generator=torch.Generator().manual_seed(first + length)).to(DEV)]
    dout = randn((tokens.numel(), width), F32, 77)
    dtable = embed_grad(dout, tokens, rows, torch.full((rows, width), 5.0, device=DEV))
    want, tol = grad_and_bound(dout, tokens, rows, 1.0, F32)
    within(dtable, want, tol, "dtable")
