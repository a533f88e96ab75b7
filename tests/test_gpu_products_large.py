"""Products of the sizes that training runs: pairs of blocks, wide tiles, several tiles a block, results by TMA, whole tiles beside cut ones.
On the CPU, that the plan sends them there; on the GPU, against 64 bits.

Bounds, in parts of the result's norm.  fp32 results: a run of 512 terms is 32 products of 16; each may truncate its 16 terms and the
sum so far at 2^-23 of it, half of that on average: 32 * 17 / 2 * 2^-23 * 2 / 3 of a run's own size, 2.2e-5, and runs add up at random.
Results of 16 bits: rounding a spread of values, 2^-7 / sqrt(12) of a binade's lower end (bf16), 1.7e-3 of the norm: below 2^-9; f16 an eighth."""
import math

import pytest
import torch

import plans as pl
from paper_2605_01989_b200 import binding as dblp

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NEAR = {F32: 2.2e-5, BF16: 2.0 ** -9, F16: 2.0 ** -12}
UPDATE = {F32: 1.2e-5, BF16: 3e-3}

UPDATES = [(1, 1601, 3100), (1, 3100, 1590), (8, 803, 1109), (8, 1590, 1700), (1, 700, 4000), (1, 6400, 1600), (3, 1310, 1700)]
LONG_UPDATES = [(1, 8200, 8250), (8, 2100, 12000)]       # sums of more than 8192 terms that are not cut
ROWS, WIDE, NARROW = 4207, 6384, 1616                  # a down-projection: a ragged batch, widths that end inside a piece
VOCABULARY = (520, 512, 50257)


def test_the_updates_reach_every_kind_of_tile():
    for precise in (False, True):
        grams, squares, steps = zip(*(pl.plans(pl.update(*s, precise)) for s in UPDATES))
        symmetric = grams + squares
        assert sum(r["cg"] == 2 for r in symmetric) >= 11 and {r["bn"] for r in symmetric if r["cg"] == 2} == {128, 256}
        assert any(r["rest"] and r["whole"] and r["cg"] == 2 for r in symmetric)                    # cut tiles beside whole ones, mirrored
        assert any(r["rest"] and not r["whole"] for r in symmetric)
        assert any(r["items"] > 74 and r["cg"] == 2 for r in symmetric)                             # several a pair
        assert sum(r["several"] and r["cg"] == 2 for r in steps) >= 5 and {r["bn"] for r in steps if r["several"]} >= {128, 256}
    assert any(r["rest"] and r["whole"] and r["several"] for r in steps)


def test_the_long_updates_sum_in_runs():
    for s in LONG_UPDATES:
        assert max(r["longest"] for r in pl.plans(pl.update(*s, False))) * 64 > 8192, s


def test_the_layers_reach_wide_pairs_in_runs_and_by_tma():
    (dx,), (dw,) = pl.plans([pl.grad_x(ROWS, WIDE, NARROW)]), pl.plans([pl.grad_w(ROWS, WIDE, NARROW)])
    for r in (dx, dw):
        assert r["cg"] == 2 and r["bn"] == 256 and r["several"]
    assert dw["whole"] and dw["rest"]
    n, d, v = VOCABULARY
    logits, dx, dw = pl.plans([dict(pl.forward(n, d, v, True), whole=1), dict(pl.grad_x(n, d, v, True), whole=0), dict(pl.grad_w(n, d, v, True), whole=0)])
    assert logits["cg"] == 2 and logits["several"] and dx["copies"] and dw["copies"] and dw["several"]


def randn(shape, dtype, seed, sigma=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).mul_(sigma).to(dtype)


def space(n):
    return torch.full((n + 256,), 0xAB, dtype=torch.uint8, device=DEV)[:n]


def near(got, want, bound, what):
    off = ((got.double() - want).norm() / want.norm()).item()
    assert off < bound, (what, off)
    # a piece in a wrong place is far off by itself: every 32 rows and every 32 columns
    for dim in (0, 1):
        e, w = (t.pow(2).sum(1 - dim) for t in (got.double() - want, want))
        k = len(e) // 32 * 32
        if k:
            worst = (e[:k].view(-1, 32).sum(1) / w[:k].view(-1, 32).sum(1)).max().sqrt().item()
            assert worst < 2 * bound, (what, dim, worst)


def iteration(x):
    x = x.double()
    x = x / (x.norm() + 1e-7)
    for a, b, c in dblp.MUON_COEFFICIENTS:
        if x.shape[0] <= x.shape[1]:
            A = x @ x.T
            x = a * x + (b * A + c * A @ A) @ x
        else:
            A = x.T @ x
            x = a * x + x @ (b * A + c * A @ A)
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("b,m,n", UPDATES + LONG_UPDATES)
def test_large_matrices_are_orthogonalised(b, m, n, out_dtype):
    x = randn((b, m, 8), F32, 1, 0.5) @ randn((b, 8, n), F32, 2) + randn((b, m, n), F32, 3)
    buf = torch.full((b, m + 3, (n + 47) // 16 * 16), 9.0, dtype=out_dtype, device=DEV)
    out = buf[:, :m, :n]
    ws = space(dblp.dblp_orthogonalize_workspace_bytes(x, out))
    dblp.dblp_orthogonalize(x, out, ws, scale=1.25)
    for j in range(b):
        near(out[j], 1.25 * iteration(x[j]), UPDATE[out_dtype], j)
    assert (buf[:, m:] == 9).all() and (buf[:, :, n:] == 9).all()
    first = out.clone()
    dblp.dblp_orthogonalize(x, out, ws, scale=1.25)
    assert torch.equal(out, first)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dw_dtype,turned", [(BF16, F32, False), (F16, F32, True), (BF16, BF16, True), (F16, F16, False)])
def test_a_large_layers_gradients(dtype, dw_dtype, turned):
    n, i, o = ROWS, WIDE, NARROW
    dy, x = randn((n, o), dtype, 1), randn((n, i), dtype, 2)
    w = randn((o, i), dtype, 3, o ** -0.5).t() if turned else randn((i, o), dtype, 3, o ** -0.5)
    pre, keep = randn((n, i), dtype, 4), randn((n, i), dtype, 5)
    dw = torch.full((o, i) if turned else (i, o), 7.0, dtype=dw_dtype, device=DEV)
    dw = dw.t() if turned else dw
    buf, db = torch.full((n + 1, i + 16), 9.0, dtype=dtype, device=DEV), torch.empty(o, device=DEV)
    dx, ws = buf[:n, :i], space(dblp.dblp_linear_workspace_bytes(x, w, dy)[1])
    dblp.dblp_linear_grad(dy, x, w, dx=dx, dw=dw, dbias=db, ws=ws, residual=keep, pre=pre, activation="silu")
    g = torch.sigmoid(pre.double())
    near(dx, (dy.double() @ w.double().t() + keep.double()) * (g * (1 + pre.double() * (1 - g))), NEAR[dtype], "dx")
    near(dw, x.double().t() @ dy.double(), NEAR[dw_dtype], "dw")
    near(db[None], dy.double().sum(0)[None], 2.0 ** -20, "dbias")
    assert (buf[n] == 9).all() and (buf[:, i:] == 9).all()
    alone = torch.empty_like(x)
    dblp.dblp_linear_grad(dy, x, w, dx=alone, ws=ws, residual=keep)
    near(alone, dy.double() @ w.double().t() + keep.double(), NEAR[dtype], "dx without an activation")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_an_output_layer_of_an_odd_vocabulary(dtype):
    """The largest product of a token model's step: fp32 logits, and gradients whose rows are off 16 bytes; the table is [vocabulary, width]."""
    n, d, v = VOCABULARY
    x, table = randn((n, d), dtype, 1), randn((v, d), dtype, 2, d ** -0.5)
    logits = torch.full((n, v), 7.0, device=DEV)
    dlogits = randn((n, v), dtype, 3)
    ws = space(max(dblp.dblp_linear_workspace_bytes(x, table.t(), dlogits)))
    dblp.dblp_linear(x, table.t(), logits, ws=ws)
    near(logits, x.double() @ table.double().t(), NEAR[F32], "logits")
    dx, dtable, db = torch.empty_like(x), torch.full((v, d), 7.0, device=DEV), torch.empty(v, device=DEV)
    dblp.dblp_linear_grad(dlogits, x, table.t(), dx=dx, dw=dtable.t(), dbias=db, ws=ws)
    near(dx, dlogits.double() @ table.double(), NEAR[dtype], "dx")
    near(dtable, dlogits.double().t() @ x.double(), NEAR[F32], "dtable")
    near(db[None], dlogits.double().sum(0)[None], 2.0 ** -20, "dbias")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out_dtype", [(BF16, BF16), (F16, F32)])
def test_a_large_layer_forward(dtype, out_dtype):
    n, i, o = 4100, NARROW, WIDE
    (r,) = pl.plans([pl.forward(n, i, o)])
    assert r["cg"] == 2 and r["bn"] == 256 and r["several"]
    x, w, bias, keep = randn((n, i), dtype, 1), randn((i, o), dtype, 2, i ** -0.5), randn((o,), F32, 3), randn((n, o), out_dtype, 4)
    out, pre = torch.empty((n, o), dtype=out_dtype, device=DEV), torch.empty((n, o), dtype=dtype, device=DEV)
    dblp.dblp_linear(x, w, out, ws=space(dblp.dblp_linear_workspace_bytes(x, w)[0]), bias=bias, residual=keep, pre=pre, activation="gelu")
    z = x.double() @ w.double() + bias.double()
    near(pre, z, NEAR[dtype], "pre")
    near(out, z * 0.5 * torch.special.erfc(-z / math.sqrt(2)) + keep.double(), NEAR[out_dtype], "out")
