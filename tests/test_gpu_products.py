"""The linear layer, its gradients and the orthogonalised update against plain 64-bit statements of their formulas.

Tolerances follow from the formats.  u = half a unit in the last place of the tensor's type, relative.  An fp32 sum of m terms is
off by at most m 2^-23 of the sum of absolute terms (additions that truncate included).  Activations and their derivatives change by
at most 1.2 times a change of z; computed in fp32 they are off by 2^-17 of their factors at most (the exponential is off by
1.2 |x| units of 2^-24 + 2 of them, which matters up to |x| = 80)."""
import math

import pytest
import torch

from paper_2605_01989_b200 import binding as dblp

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 0.0, BF16: 0.0, F16: 2.0 ** -25}            # half the spacing of a type's smallest numbers, where that shows


def randn(shape, dtype, seed, sigma=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * sigma).to(dtype)


def within(got, want, tol, what):
    assert torch.isfinite(got.double()).all(), what
    worst = ((got.double() - want).abs() - tol).max().item() if want.numel() else -1
    assert worst <= 0, "%s: beyond the tolerance by %g" % (what, worst)


def cdf(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2))


C = math.sqrt(8 / math.pi)
ACT = {None: lambda z: z, "relu": torch.relu, "gelu": lambda z: z * cdf(z), "silu": lambda z: z * torch.sigmoid(z),
       "gelu_tanh": lambda z: z * torch.sigmoid(C * (z + 0.044715 * z ** 3))}


def slope(name, z):
    z = z.clone().requires_grad_()
    return torch.autograd.grad(ACT[name](z).sum(), z)[0]


def space(n):
    return torch.full((n + 256,), 0xAB, dtype=torch.uint8, device=DEV)[:n]          # contents do not matter


def linear(x, w, out_dtype, **kw):
    out = kw.pop("out", None)
    if out is None:
        out = torch.full((x.shape[0], w.shape[1]), 7.0, dtype=out_dtype, device=DEV)
    dblp.dblp_linear(x, w, out, ws=space(dblp.dblp_linear_workspace_bytes(x, w)[0]), **kw)
    return out


def expected(x, w, out_dtype, bias, residual, f):
    """(out, its tolerance, z, its tolerance)"""
    xd, wd = x.double(), w.double()
    z, mass = xd @ wd, xd.abs() @ wd.abs()
    if bias is not None:
        z, mass = z + bias.double(), mass + bias.double().abs()
    ez = (x.shape[1] + 2) * 2.0 ** -23 * mass
    y = ACT[f](z)
    tol = 1.2 * ez + (2.0 ** -17 * z.abs() if f else 0)
    if residual is not None:
        y = y + residual.double()
        tol = tol + 2.0 ** -23 * (y.abs() + residual.double().abs())
    return y, (tol + U[out_dtype] * (y.abs() + tol) + TINY[out_dtype]), z, ez + U[x.dtype] * (z.abs() + ez) + TINY[x.dtype]


SIZES = [(1, 1, 1), (1, 64, 128), (2, 1600, 6400), (3, 257, 129), (4, 512, 1000), (1, 6400, 1600), (3, 40, 72), (4, 8, 8), (7, 33, 260), (8, 4096, 1000), (17, 100, 7), (31, 1601, 515), (64, 512, 1024),
         (65, 40, 129), (100, 1, 300), (127, 129, 1), (128, 64, 64), (129, 520, 260), (300, 72, 2050), (777, 1601, 499), (1100, 1000, 1530),
         (4100, 192, 768)]


@pytest.mark.parametrize("n,i,o", SIZES)
@pytest.mark.parametrize("dtype,out_dtype,turned", [(BF16, BF16, False), (F16, F32, True), (BF16, F32, True), (F16, F16, False)])
def test_linear_is_the_rounded_formula(n, i, o, dtype, out_dtype, turned):
    f = list(ACT)[(n + i + o) % 5]
    x = randn((n, i), dtype, 1)
    w = randn((o, i), dtype, 2, i ** -0.5).t() if turned else randn((i, o), dtype, 2, i ** -0.5)
    bias = randn((o,), F32 if n % 2 else dtype, 3) if o % 3 else None
    residual = randn((n, o), out_dtype, 4) if i % 2 == 0 else None
    pre = torch.full((n, o), 5.0, dtype=dtype, device=DEV)
    out = linear(x, w, out_dtype, bias=bias, residual=residual, pre=pre, activation=f)
    y, tol, z, ez = expected(x, w, out_dtype, bias, residual, f)
    within(out, y, tol, "out")
    within(pre, z, ez, "pre")
    again = linear(x, w, out_dtype, bias=bias, residual=residual, activation=f)
    assert torch.equal(again, out)


@pytest.mark.parametrize("f", list(ACT))
@pytest.mark.parametrize("n", [5, 200])
def test_activations_and_their_derivatives(f, n):
    """x = 1 and one column a value: z takes every value of a type's range that matters."""
    v = torch.cat((torch.linspace(-12, 12, 1199, device=DEV), torch.tensor([-300.0, -88.0, -1e-4, 0.0, 1e-4, 88.0, 300.0, 1e4, -1e4], device=DEV)))
    v = v.to(F16).float()
    x, w = torch.ones((n, 1), dtype=F16, device=DEV), v.to(F16)[None, :]
    out = linear(x, w, F32, activation=f)
    want = ACT[f](v.double()).expand(n, -1)
    within(out, want, 2.0 ** -17 * want.abs() + 1e-30, "act")
    if f is None:
        return
    dx = torch.empty((n, v.numel()), dtype=F16, device=DEV)
    dy, eye = torch.ones((n, 1), dtype=F16, device=DEV), torch.ones((v.numel(), 1), dtype=F16, device=DEV)
    dblp.dblp_linear_grad(dy, dx, eye, dx=dx, pre=v.to(F16).expand(n, -1).contiguous(), activation=f,
                          ws=space(dblp.dblp_linear_workspace_bytes(dx, eye, dy)[1]))
    d = slope(f, v.double()).expand(n, -1)
    if f == "relu":
        d = (v > 0).double().expand(n, -1)
    within(dx, d, (2.0 ** -17 + U[F16]) * (d.abs() + 2.0 ** -7 * (d.abs() < 1e-2)) + TINY[F16], "act'")


@pytest.mark.parametrize("n,i,o", [(5, 96, 200), (70, 200, 136), (600, 264, 520)])
def test_linear_strides_broadcasts_and_places(n, i, o):
    wide, tall = randn((n, i + 24), BF16, 5), randn((i + 3, o + 16), BF16, 6, i ** -0.5)
    buf = torch.full((n, o + 40), 9.0, dtype=BF16, device=DEV)
    for cut in (8, 1):                                  # column 1: rows that start off every boundary
        x, w, out = wide[:, cut:cut + i], tall[1:1 + i, cut:cut + o], buf[:, cut:cut + o]
        buf.fill_(9.0)
        linear(x, w, BF16, out=out, activation="gelu")
        y, tol, _, _ = expected(x, w, BF16, None, None, "gelu")
        within(out, y, tol, "strided")
        assert (buf[:, :cut] == 9).all() and (buf[:, cut + o:] == 9).all()
    one = randn((1, i), BF16, 7).expand(n, i)
    w = randn((o, i), BF16, 8, i ** -0.5).t()
    out = linear(one, w, BF16)
    y, tol, _, _ = expected(one, w, BF16, None, None, None)
    within(out, y, tol, "one row, repeated")
    res = randn((n, o), F32, 9)
    before = res.clone()
    linear(wide[:, :i], w, F32, out=res, residual=res, activation="silu")
    y, tol, _, _ = expected(wide[:, :i], w, F32, None, before, "silu")
    within(res, y, tol, "over the residual")


@pytest.mark.parametrize("n,i,o", [(2, 64, 96), (50, 64, 96), (700, 64, 544)])
@pytest.mark.parametrize("bias_dtype", [F32, BF16, F16])
def test_bias_anywhere_in_a_flat_vector(n, i, o, bias_dtype):
    x, w, flat = randn((n, i), BF16, 1), randn((i, o), BF16, 2, i ** -0.5), randn((o + 3,), bias_dtype, 3)
    for at in (0, 1, 3):
        out = linear(x, w, BF16, bias=flat[at:at + o], activation="silu")
        y, tol, _, _ = expected(x, w, BF16, flat[at:at + o], None, "silu")
        within(out, y, tol, at)


def test_many_tiles_a_block_and_edges_of_them():
    """More tiles than blocks: results by TMA, with rows and columns that end inside a piece, beside untouched neighbours."""
    n, i, o = 4111, 72, 2600
    x, w = randn((n, i), BF16, 1), randn((i, o), BF16, 2, i ** -0.5)
    for odt in (BF16, F32):
        buf, pre = torch.full((n + 1, o + 40), 9.0, dtype=odt, device=DEV), torch.full((n, o), 5.0, dtype=BF16, device=DEV)
        res = randn((n, o), odt, 3)
        linear(x, w, odt, out=buf[:n, :o], residual=res, pre=pre if odt == BF16 else None, activation="gelu")
        y, tol, z, ez = expected(x, w, odt, None, res, "gelu")
        within(buf[:n, :o], y, tol, "out")
        assert (buf[n] == 9).all() and (buf[:, o:] == 9).all()
        if odt == BF16:
            within(pre, z, ez, "pre")
    dy, dw = randn((n, o), BF16, 4), torch.empty((i, o), device=DEV)
    dx, keep = randn((n, i), BF16, 5), randn((n, i), BF16, 6)
    dblp.dblp_linear_grad(dy, x, w, dx=dx, dw=dw, ws=space(dblp.dblp_linear_workspace_bytes(x, w, dy)[1]), residual=keep)
    want, mass = dy.double() @ w.double().t() + keep.double(), dy.double().abs() @ w.double().abs().t() + keep.double().abs()
    tol = (o + 2) * 2.0 ** -23 * mass
    within(dx, want, tol + U[BF16] * (want.abs() + tol), "dx")


def test_elements_beyond_32_bits():
    n, i, o = 43000, 16, 50264
    x, w = randn((n, i), BF16, 1), randn((i, o), BF16, 2, i ** -0.5)
    out = torch.empty((n, o), dtype=BF16, device=DEV)
    assert out.numel() > 1 << 31
    linear(x, w, BF16, out=out, activation="relu")
    for rows in (slice(0, 40), slice(n // 2, n // 2 + 40), slice(n - 40, n)):
        y, tol, _, _ = expected(x[rows], w, BF16, None, None, "relu")
        within(out[rows], y, tol, rows)
    dx = torch.empty((n, i), dtype=BF16, device=DEV)
    dblp.dblp_linear_grad(out, x, w, dx=dx, ws=space(dblp.dblp_linear_workspace_bytes(x, w, out)[1]))
    rows = slice(n - 40, n)
    want, mass = out[rows].double() @ w.double().t(), out[rows].double().abs() @ w.double().abs().t()
    within(dx[rows], want, (o + 2) * 2.0 ** -23 * mass + U[BF16] * (want.abs() + mass * 2.0 ** -8), "dx")


def test_rows_in_reverse():
    """Negative row strides, which the header allows (a tensor cannot have them: raw addresses)."""
    import ctypes as C
    n, i, o = 300, 64, 96
    x, w = randn((n, i), BF16, 1), randn((i, o), BF16, 2, i ** -0.5)
    out, plain = torch.zeros((n, o), dtype=BF16, device=DEV), linear(x, w, BF16)
    m = lambda t, rows: C.byref(dblp.dblp_matrix_t(t.data_ptr() + (rows - 1) * t.stride(0) * 2, -t.stride(0), 1))
    l = dblp.dblp_linear_t(n, i, o, 1, 1, 0, 0, 0)
    f = C.c_size_t()
    assert dblp.lib().dblp_linear_workspace_bytes(C.byref(l), m(x, n), C.byref(dblp.dblp_matrix_t(w.data_ptr(), o, 1)), None, C.byref(f), None) == 0
    ws = space(f.value)
    rc = dblp.lib().dblp_linear(C.byref(l), m(x, n), C.byref(dblp.dblp_matrix_t(w.data_ptr(), o, 1)), None, None, None, m(out, n), ws.data_ptr(), f.value,
                                torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(out, plain)


def test_linear_without_input_columns_or_rows():
    bias, res = randn((40,), F32, 1), randn((9, 40), F32, 2)
    x, w = torch.empty((9, 0), dtype=BF16, device=DEV), torch.empty((0, 40), dtype=BF16, device=DEV)
    out = linear(x, w, F32, bias=bias, residual=res, activation="relu")
    assert torch.equal(out, torch.relu(bias).expand(9, -1) + res)
    linear(x[:0], w, F32)
    linear(x, w[:, :0], F32)


def test_what_is_not_finite_stays_in_its_row():
    x, w = randn((200, 96), BF16, 1), randn((96, 136), BF16, 2)
    x[7, 3], x[150, 90] = math.nan, math.inf
    for f in ACT:
        out = linear(x, w, BF16, activation=f)
        assert out[7].isnan().all() and not torch.isfinite(out[150]).all()
        ok = torch.ones(200, dtype=torch.bool, device=DEV)
        ok[[7, 150]] = False
        assert torch.isfinite(out[ok]).all(), f


# ---- gradients -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,i,o", SIZES + [(9001, 65, 130), (2048, 256, 8), (5000, 8, 8)])
@pytest.mark.parametrize("dtype,dw_dtype,turned", [(BF16, F32, False), (F16, F16, True), (BF16, BF16, False)])
def test_linear_grad_is_the_formula(n, i, o, dtype, dw_dtype, turned):
    f = list(ACT)[(n + i) % 5]
    dy, x = randn((n, o), dtype, 1), randn((n, i), dtype, 2)
    w = randn((o, i), dtype, 3, o ** -0.5).t() if turned else randn((i, o), dtype, 3, o ** -0.5)
    pre = randn((n, i), dtype, 4) if f else None
    residual = randn((n, i), dtype, 5) if o % 2 == 0 else None
    dx = torch.full((n, i), 7.0, dtype=dtype, device=DEV)
    dw = (torch.full((o, i), 7.0, dtype=dw_dtype, device=DEV).t() if turned else torch.full((i, o), 7.0, dtype=dw_dtype, device=DEV))
    db = torch.full((o,), 7.0, dtype=F32 if o % 3 else dtype, device=DEV)
    ws = space(dblp.dblp_linear_workspace_bytes(x, w, dy)[1])
    dblp.dblp_linear_grad(dy, x, w, dx=dx, dw=dw, dbias=db, ws=ws, residual=residual, pre=pre, activation=f)

    y, a, b = dy.double(), x.double(), w.double()
    want, mass = y @ b.t(), y.abs() @ b.abs().t()
    if residual is not None:
        want, mass = want + residual.double(), mass + residual.double().abs()
    tol = (o + 2) * 2.0 ** -23 * mass
    if f:
        d = slope(f, pre.double())
        want, tol = want * d, tol * d.abs() + 2.0 ** -17 * want.abs()
    within(dx, want, tol + U[dtype] * (want.abs() + tol) + TINY[dtype], "dx")
    want, tol = a.t() @ y, (n + 2) * 2.0 ** -23 * (a.abs().t() @ y.abs())
    within(dw, want, tol + U[dw_dtype] * (want.abs() + tol) + TINY[dw_dtype], "dw")
    want, tol = y.sum(0), (n + 2) * 2.0 ** -23 * y.abs().sum(0)
    within(db, want, tol + U[db.dtype] * (want.abs() + tol) + TINY[db.dtype], "dbias")

    first = dw.clone(), db.clone()
    dblp.dblp_linear_grad(dy, x, w, dw=dw, dbias=db, ws=ws, accumulate=True)
    for got, was in zip((dw, db), first):
        want = 2 * was.double()                         # the product again, exactly as before, unless `was` had been rounded
        within(got, want, 4 * U[got.dtype] * want.abs() + 2 * TINY[got.dtype], "accumulated")


def test_a_gradient_against_differences():
    """Loss = <out, c> of a two-layer block in 64 bits, moved a little in a random direction of each argument."""
    n, d, h = 40, 72, 200
    x, w1, w2 = randn((n, d), BF16, 1), randn((d, h), BF16, 2, d ** -0.5), randn((h, d), BF16, 3, h ** -0.5)
    b1, c = randn((h,), F32, 4), randn((n, d), BF16, 5)
    pre = torch.empty((n, h), dtype=BF16, device=DEV)
    mid = linear(x, w1, BF16, bias=b1, pre=pre, activation="gelu")
    dw2, dpre = torch.empty((h, d), device=DEV), torch.empty((n, h), dtype=BF16, device=DEV)
    dblp.dblp_linear_grad(c, mid, w2, dx=dpre, dw=dw2, ws=space(dblp.dblp_linear_workspace_bytes(mid, w2, c)[1]), pre=pre, activation="gelu")
    dw1, db1, dx = torch.empty((d, h), device=DEV), torch.empty(h, device=DEV), torch.empty((n, d), dtype=BF16, device=DEV)
    dblp.dblp_linear_grad(dpre, x, w1, dx=dx, dw=dw1, dbias=db1, residual=c, ws=space(dblp.dblp_linear_workspace_bytes(x, w1, dpre)[1]))

    args = [t.double() for t in (x, w1, b1, w2)]

    def loss(x, w1, b1, w2):
        return ((ACT["gelu"](x @ w1 + b1) @ w2 + x) * c.double()).sum()

    for k, grad in enumerate((dx, dw1, db1, dw2)):
        step = randn(args[k].shape, F32, 10 + k).double() * 1e-4
        up, down = ([a + s * step if j == k else a for j, a in enumerate(args)] for s in (1, -1))
        slope_ = (loss(*up) - loss(*down)) / 2
        # four roundings to bf16 at most on the way, of random sign in sums of many terms: 2^-8 of the root sum of squares
        tol = 4 * 2.0 ** -8 * (grad.double() * step).norm() + 1e-6 * abs(slope_)
        assert abs((grad.double() * step).sum() - slope_) <= 4 * tol, k


def test_linear_grad_with_nothing_to_sum():
    w, x = randn((24, 40), BF16, 1), torch.empty((0, 24), dtype=BF16, device=DEV)
    dy = torch.empty((0, 40), dtype=BF16, device=DEV)
    dw, db = torch.full((24, 40), 3.0, device=DEV), torch.full((40,), 3.0, device=DEV)
    ws = space(dblp.dblp_linear_workspace_bytes(x, w, dy)[1])
    dblp.dblp_linear_grad(dy, x, w, dw=dw, dbias=db, ws=ws, accumulate=True)
    assert (dw == 3).all() and (db == 3).all()
    dblp.dblp_linear_grad(dy, x, w, dw=dw, dbias=db, ws=ws)
    assert (dw == 0).all() and (db == 0).all()
    x, dy, w = randn((9, 24), BF16, 2), torch.empty((9, 0), dtype=BF16, device=DEV), torch.empty((24, 0), dtype=BF16, device=DEV)
    dx = torch.empty_like(x)
    dblp.dblp_linear_grad(dy, x, w, dx=dx, residual=x)
    assert torch.equal(dx, x)


@pytest.mark.parametrize("n,i,o", [(3, 200, 136), (300, 136, 264)])
def test_dx_over_pre_or_the_residual_and_strided_gradients(n, i, o):
    dy, x, w = randn((n, o + 8), F16, 1)[:, 3:3 + o], randn((n, i), F16, 2), randn((i, o), F16, 3, o ** -0.5)
    pre, res = randn((n, i), F16, 4), randn((n, i), F16, 5)
    plain = torch.empty((n, i), dtype=F16, device=DEV)
    ws = space(dblp.dblp_linear_workspace_bytes(x, w, dy)[1])
    kw = dict(ws=ws, activation="silu")
    dblp.dblp_linear_grad(dy, x, w, dx=plain, pre=pre, residual=res, **kw)
    over = pre.clone()
    dblp.dblp_linear_grad(dy, x, w, dx=over, pre=over, residual=res, **kw)
    assert torch.equal(over, plain)
    over = res.clone()
    dblp.dblp_linear_grad(dy, x, w, dx=over, pre=pre, residual=over, **kw)
    assert torch.equal(over, plain)
    flat = torch.full((i * o + 5,), 2.0, device=DEV)       # an fp32 gradient anywhere in a flat buffer
    dw = flat[3:3 + i * o].view(i, o)
    dblp.dblp_linear_grad(dy, x, w, dw=dw, ws=ws)
    want, tol = x.double().t() @ dy.double(), (n + 2) * 2.0 ** -23 * (x.double().abs().t() @ dy.double().abs())
    within(dw, want, tol + 2.0 ** -24 * want.abs(), "dw")
    assert (flat[:3] == 2).all() and (flat[3 + i * o:] == 2).all()


# ---- orthogonalised update ------------------------------------------------------------------------------------------------
def newton_schulz(x, coefficients, eps):
    x = x.double()
    x = x / (x.norm() + eps) if x.norm() + eps > 0 else x
    for a, b, c in coefficients:
        if x.shape[0] <= x.shape[1]:
            A = x @ x.T
            x = a * x + (b * A + c * A @ A) @ x
        else:
            A = x.T @ x
            x = a * x + x @ (b * A + c * A @ A)
    return x


def orthogonalize(x, out_dtype, out=None, **kw):
    if out is None:
        out = torch.full(x.shape, 7.0, dtype=out_dtype, device=DEV)
    dblp.dblp_orthogonalize(x, out, space(dblp.dblp_orthogonalize_workspace_bytes(x, out)), **kw)
    return out


def matrix(b, m, n, dtype, kind, seed):
    g = randn((b, m, n), F32, seed)
    if kind == "strong":
        g = randn((b, m, 3), F32, seed + 1) @ randn((b, 3, n), F32, seed + 2) + 0.1 * g
    elif kind == "low rank":
        g = randn((b, m, 2), F32, seed + 1) @ randn((b, 2, n), F32, seed + 2)
    return (g * 1e-3).to(dtype)


# Of the result's norm.  One f16 product: in each of five steps some six roundings of 2^-12.3 on average, each changing X by at most
# about 8 times itself (the coefficients), adding up at random: sqrt(30) * 2e-4 * 8 = 9e-3; and the rounding of the result.
# Two words: 2^-22 of X may grow with a small singular value, 3.45^5 = 485 times, 1.2e-4.
CLOSE = {BF16: 9e-3 + 2.0 ** -8, F32: 1.2e-4, F16: 1.2e-4 + 2.0 ** -11}


@pytest.mark.parametrize("b,m,n", [(1, 1, 1), (1, 1, 50), (2, 40, 1), (3, 5, 9), (1, 64, 64), (2, 33, 120), (1, 129, 200), (1, 128, 128), (4, 130, 64),
                                   (1, 257, 255), (1, 700, 90), (1, 100, 1500), (2, 384, 640), (1, 1030, 520), (40, 24, 16)])
@pytest.mark.parametrize("kind,dtype,out_dtype", [("noise", F32, BF16), ("strong", BF16, F32), ("low rank", F32, BF16), ("strong", F16, F16)])
def test_orthogonalize_is_the_iteration(b, m, n, kind, dtype, out_dtype):
    x = matrix(b, m, n, dtype, kind, m + n)
    out = orthogonalize(x, out_dtype, scale=1.5)
    for j in range(b):
        want = 1.5 * newton_schulz(x[j], dblp.MUON_COEFFICIENTS, 1e-7)
        rel = ((out[j].double() - want).norm() / want.norm()).item()
        assert rel < CLOSE[out_dtype], rel
    assert torch.equal(orthogonalize(x, out_dtype, scale=1.5), out)


def test_orthogonalize_brings_singular_values_near_one():
    x = matrix(1, 200, 340, F32, "noise", 1)[0]
    s = torch.linalg.svdvals(orthogonalize(x, F32).double())
    assert 0.6 < s.min() and s.max() < 1.3
    cubic = ((1.5, -0.5, 0.0),) * 16                     # converges to the nearest orthogonal matrix from below
    y = orthogonalize(x, F32, coefficients=cubic).double()
    want = newton_schulz(x, cubic, 1e-7)
    assert ((y - want).norm() / want.norm()).item() < 16 / 5 * CLOSE[F32]


def test_orthogonalize_strides_places_and_sizes_of_values():
    wide = matrix(3, 90, 200, F32, "noise", 4)
    for cut in (1, 8):
        x = wide[:, 2:80, cut:cut + 151]
        buf = torch.full((3, 78, 170), 9.0, dtype=BF16, device=DEV)
        out = orthogonalize(x, BF16, out=buf[:, :, cut:cut + 151])
        assert torch.equal(out, orthogonalize(x.contiguous(), BF16))
        assert (buf[:, :, :cut] == 9).all() and (buf[:, :, cut + 151:] == 9).all()
    x = wide[0].clone()
    want = orthogonalize(x, F32)
    assert torch.equal(orthogonalize(x, F32, out=x.clone(), eps=1e-7), want)
    same = x.clone()
    assert torch.equal(orthogonalize(same, F32, out=same), want)
    for size in (1e-30, 1e30):                           # squares beyond fp32
        y = orthogonalize(x * size, F32, eps=0.0)
        assert ((y - orthogonalize(x, F32, eps=0.0)).norm() / want.norm()).item() < CLOSE[F32]


def test_orthogonalize_zeros_and_what_is_not_finite_stay_in_their_matrix():
    x = matrix(4, 70, 40, F32, "noise", 4)
    x[1] = 0
    x[2, 5, 6] = math.nan
    for eps in (0.0, 1e-7):
        out = orthogonalize(x, BF16, eps=eps)
        assert (out[1] == 0).all() and out[2].isnan().all()
        assert torch.equal(out[[0, 3]], orthogonalize(x[[0, 3]], BF16, eps=eps))
    dblp.dblp_orthogonalize(x[:0], out[:0], None)
    dblp.dblp_orthogonalize(x[:, :0], out[:, :0], None)


# ---- streams and graphs ---------------------------------------------------------------------------------------------------
def test_products_on_another_stream_and_from_a_graph():
    x, w, dy = randn((300, 520), BF16, 1), randn((520, 264), BF16, 2), randn((300, 264), BF16, 3)
    f, g = dblp.dblp_linear_workspace_bytes(x, w, dy)
    ws = space(max(f, g))
    upd = torch.empty((520, 264), dtype=BF16, device=DEV)
    dw, dx, out = torch.empty((520, 264), device=DEV), torch.empty_like(x), torch.empty((300, 264), dtype=BF16, device=DEV)
    ws2 = space(dblp.dblp_orthogonalize_workspace_bytes(dw, upd))

    def calls():
        dblp.dblp_linear(x, w, out, ws=ws, activation="gelu")
        dblp.dblp_linear_grad(dy, x, w, dx=dx, dw=dw, ws=ws)
        dblp.dblp_orthogonalize(dw, upd, ws2)

    calls()
    want = [t.clone() for t in (out, dx, dw, upd)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in (out, dx, dw, upd):
            t.fill_(0)
        calls()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, (out, dx, dw, upd)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in (11, 12):
        x.copy_(randn(x.shape, BF16, seed))
        graph.replay()
        got = [t.clone() for t in (out, dx, dw, upd)]
        calls()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, dx, dw, upd)))
    assert dblp.dblp_wait_timeouts() == 0
