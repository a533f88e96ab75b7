"""dblp_norm_rotate and its gradient against 64-bit statements of their formulas.

Tolerances: u = half a unit in the last place of the tensor's type.  The fp32 part: r from a sum of at most 8 + 5 additions a lane,
cosine and sine off by 2^-21 at most (the angle, below a turn, rounded to fp32, and the function's own error): 2^-20 of the absolute
terms of a result.  A weight's gradient is an fp32 sum of m terms, m 2^-24 more of their absolute sum."""
import pytest
import torch

from paper_2605_01989_b200 import binding as dblp

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 0.0, BF16: 0.0, F16: 2.0 ** -25}


def randn(shape, dtype, seed, sigma=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * sigma).to(dtype)


def within(got, want, tol, what):
    assert torch.isfinite(got.double()).all(), what
    worst = ((got.double() - want).abs() - tol).max().item() if want.numel() else -1
    assert worst <= 0, "%s: beyond the tolerance by %g" % (what, worst)


def partners(x, R, inter):
    """(first members, second members) of the turned pairs, as index lists."""
    i = torch.arange(R // 2, device=DEV)
    return (2 * i, 2 * i + 1) if inter else (i, i + R // 2)


def turned(x, angle, R, inter, back=False):
    """x turned, and the absolute terms of each result."""
    a, b = partners(x, R, inter)
    c, s = angle.cos(), angle.sin() * (-1 if back else 1)
    y, m = x.clone(), x.abs()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    m[..., a] = m[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, m


def case(B, T, Hq, Hk, D, R, dtype, wdtype, far=0, seed=0):
    q, k = randn((B, T, Hq, D), dtype, seed + 1, 2.0), randn((B, T, Hk, D), dtype, seed + 2, 0.3)
    qw, kw = randn((D,), wdtype, seed + 3), randn((D,), wdtype, seed + 4)
    pos = torch.randint(-3, 3, (B, 1), device=DEV, dtype=torch.int32) + far + torch.arange(T, device=DEV, dtype=torch.int32)
    freqs = 10000.0 ** (-torch.arange(R // 2, device=DEV, dtype=torch.float64) / max(1, R // 2))
    return q, k, qw, kw, pos, freqs


def reference(x, w, angle, R, inter, eps):
    x = x.double()
    y = x * (x.pow(2).mean(3, keepdim=True) + eps).rsqrt() * (w.double() if w is not None else 1.0)
    return turned(y, angle, R, inter)


SHAPES = [(1, 1, 1, 1, 8, 0, False), (1, 1, 25, 25, 64, 64, False), (2, 3, 4, 2, 128, 64, True), (3, 37, 5, 1, 80, 80, False), (1, 130, 1, 1, 256, 256, False),
          (2, 65, 3, 3, 40, 40, True), (1, 33, 7, 2, 96, 32, False), (2, 9, 16, 4, 128, 128, False), (4, 1, 12, 3, 64, 16, True), (1, 300, 2, 1, 16, 16, False),
          (1, 5, 3, 0, 72, 48, False), (1, 1000, 1, 1, 8, 8, True), (2, 700, 6, 2, 24, 2, True), (1, 1500, 9, 3, 64, 64, False)]


@pytest.mark.parametrize("B,T,Hq,Hk,D,R,inter", SHAPES)
@pytest.mark.parametrize("dtype,wdtype", [(BF16, F32), (F16, F16), (F32, F32), (BF16, BF16)])
def test_norm_rotate_and_gradient(B, T, Hq, Hk, D, R, inter, dtype, wdtype):
    eps = 1e-5
    q, k, qw, kw, pos, freqs = case(B, T, Hq, max(Hk, 1), D, R, dtype, wdtype, far=1000 * T)
    angle = (pos.double()[..., None] * freqs)[:, :, None]
    sides = [("q", q, qw)] + ([("k", k, kw)] if Hk else [])
    if not Hk:
        k = kw = None
    qo, ko = torch.full_like(q, 7), None if k is None else torch.full_like(k, 7)
    dblp.dblp_norm_rotate(q, k, qw, kw, pos if R else None, freqs if R else None, qo, ko, eps=eps, interleaved=inter)
    for (name, x, w), out in zip(sides, (qo, ko)):
        want, mass = reference(x, w, angle, R, inter, eps)
        within(out, want, 2.0 ** -20 * mass + U[dtype] * want.abs() + U[dtype] * 2.0 ** -20 * mass + TINY[dtype], name)

    douts = [randn(x.shape, dtype, 20 + j) for j, (_, x, _) in enumerate(sides)]
    grads = [torch.full_like(x, 7) for _, x, _ in sides]
    dws = [torch.full_like(w, 7) for _, _, w in sides]
    ws = torch.full((dblp.dblp_norm_rotate_grad_workspace_bytes(q, k),), 0xAB, dtype=torch.uint8, device=DEV)
    two = lambda t: (t[0], t[1] if Hk else None)
    args = (q, k, qw, kw, pos if R else None, freqs if R else None, *two(douts), *two(grads), *two(dws), ws)
    dblp.dblp_norm_rotate_grad(*args, eps=eps, interleaved=inter)
    for (name, x, w), do, dx, dw in zip(sides, douts, grads, dws):
        d, dm = turned(do.double(), angle, R, inter, back=True)
        xd, wd = x.double(), w.double()
        r = (xd.pow(2).mean(3, keepdim=True) + eps).rsqrt()
        want = r * wd * d - xd * r ** 3 * (wd * d * xd).mean(3, keepdim=True)
        mass = r * wd.abs() * dm + xd.abs() * r ** 3 * (wd.abs() * dm * xd.abs()).mean(3, keepdim=True)
        tol = 2.0 ** -19 * mass
        within(dx, want, tol + U[dtype] * (want.abs() + tol) + TINY[dtype], "d" + name)
        sum_, mass = (d * xd * r).sum((0, 1, 2)), (dm * xd.abs() * r).sum((0, 1, 2))
        m = B * T * x.shape[2]
        tol = (2.0 ** -20 + m * 2.0 ** -24) * mass
        within(dw, sum_, tol + U[wdtype] * (sum_.abs() + tol) + TINY[wdtype], "weight of " + name)
    first = [t.clone() for t in dws]
    dblp.dblp_norm_rotate_grad(*args, eps=eps, interleaved=inter, accumulate=True)
    for a, b in zip(dws, first):
        want = 2 * b.double()
        within(a, want, 4 * U[wdtype] * want.abs() + 2 * TINY[wdtype], "accumulated")


@pytest.mark.parametrize("far", [0, 10 ** 6, 2 ** 31 - 100])
def test_far_positions_lose_nothing(far):
    q, k, qw, kw, pos, freqs = case(2, 20, 3, 3, 64, 64, F32, F32)
    pos = pos.clamp_min(0) + far
    out = torch.empty_like(q)
    dblp.dblp_norm_rotate(q, None, None, None, pos, freqs, out, None)
    want, mass = reference(q, None, (pos.double()[..., None] * freqs)[:, :, None], 64, False, 1e-6)
    # the product of position and frequency is off by 2^-53 of itself on both sides, and the division by a turn once more
    angle = far * 2.0 ** -51
    within(out, want, (2.0 ** -20 + angle) * mass, "far")


def test_packed_heads_shared_positions_in_place_and_zero_rows():
    B, T, H, D = 3, 50, 5, 64
    qkv = randn((B, T, 3, H, D), BF16, 1)
    qkv[1, 7] = 0
    freqs = 100.0 ** (-torch.arange(32, device=DEV, dtype=torch.float64) / 32)
    pos = torch.arange(T, device=DEV, dtype=torch.int32).expand(B, T)
    q, k, v = qkv.unbind(2)
    w = randn((D,), F32, 2)
    want = [torch.empty((B, T, H, D), dtype=BF16, device=DEV) for _ in range(2)]
    dblp.dblp_norm_rotate(q, k, w, None, pos, freqs, *want)
    assert (want[0][1, 7] == 0).all()
    angle = (pos.double()[..., None] * freqs)[:, :, None]
    for x, weight, out in ((q, w, want[0]), (k, None, want[1])):
        y, mass = reference(x, weight, angle, 64, False, 1e-6)
        within(out, y, 2.0 ** -19 * mass + U[BF16] * y.abs(), "packed")
    before = v.clone()
    dblp.dblp_norm_rotate(q, k, w, None, pos, freqs, q, k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, before)
    d = [randn((B, T, H, D), BF16, s) for s in (3, 4)]
    dq, dk = (torch.empty_like(t) for t in d)
    dblp.dblp_norm_rotate_grad(q, k, w, None, pos, freqs, *d, dq, dk)             # no gradients of weights: no workspace
    over = [t.clone() for t in d]
    dblp.dblp_norm_rotate_grad(q, k, w, None, pos, freqs, *over, *over)
    assert torch.equal(over[0], dq) and torch.equal(over[1], dk)
    one = randn((1, 1, 1, D), BF16, 5).expand(B, T, H, D)                         # one row, broadcast
    out = torch.empty((B, T, H, D), dtype=BF16, device=DEV)
    dblp.dblp_norm_rotate(one, None, w, None, pos, freqs, out, None)
    y, mass = reference(one, w, angle, 64, False, 1e-6)
    within(out, y, 2.0 ** -19 * mass + U[BF16] * y.abs(), "broadcast")


def test_nothing_to_do_and_gradients_of_nothing():
    q = torch.empty((2, 0, 3, 64), dtype=BF16, device=DEV)
    w, dw = randn((64,), F32, 1), torch.full((64,), 3.0, device=DEV)
    pos, freqs = torch.empty((2, 0), dtype=torch.int32, device=DEV), torch.ones(32, dtype=torch.float64, device=DEV)
    dblp.dblp_norm_rotate(q, q, w, w, pos, freqs, q, q)
    ws = torch.empty(dblp.dblp_norm_rotate_grad_workspace_bytes(q, q), dtype=torch.uint8, device=DEV)
    dblp.dblp_norm_rotate_grad(q, q, w, w, pos, freqs, q, q, q, q, dw, None, ws)
    assert (dw == 0).all()


def test_norm_rotate_from_a_graph_and_on_another_stream():
    q, k, qw, kw, pos, freqs = case(2, 70, 4, 2, 128, 64, BF16, F32)
    d = [randn(t.shape, BF16, 9) for t in (q, k)]
    outs = [torch.empty_like(t) for t in (q, k, q, k, qw, kw)]
    ws = torch.empty(dblp.dblp_norm_rotate_grad_workspace_bytes(q, k), dtype=torch.uint8, device=DEV)

    def calls():
        dblp.dblp_norm_rotate(q, k, qw, kw, pos, freqs, *outs[:2])
        dblp.dblp_norm_rotate_grad(q, k, qw, kw, pos, freqs, *d, *outs[2:], ws)

    calls()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in outs:
            t.fill_(0)
        calls()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    q.copy_(randn(q.shape, BF16, 31))
    graph.replay()
    got = [t.clone() for t in outs]
    calls()
    assert all(torch.equal(a, b) for a, b in zip(got, outs))
