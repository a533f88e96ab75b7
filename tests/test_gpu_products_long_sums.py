"""What a long sum loses.  The tensor cores' own additions truncate; sums of one sign lose most.  Against 64 bits."""
import pytest
import torch

import plans as pl
from paper_2605_01989_b200 import binding as dblp

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11}
SIGNED = {"one sign": (0.5, 1.5), "both signs": (-1.5, 1.5)}


def uniform(shape, dtype, seed, lo=0.5, hi=1.5, scale=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.rand(shape, generator=g, device=DEV) * (hi - lo) + lo).mul_(scale).to(dtype)


def space(n):
    return torch.full((n + 256,), 0xAB, dtype=torch.uint8, device=DEV)[:n]


def rounded_once(got, want, dtype):
    """Half a step of the type, and an eighth of one for the sum itself: 8192 terms of f16 in one run lose 8192 * 6e-9 = 4.9e-5, below
    2^-11 / 8 = 6.1e-5; of bf16 eight times as many, 3.9e-4 of 4.9e-4.  Longer sums are taken in runs of 512 terms, which lose less."""
    worst = ((got.double() - want).abs() / want.abs()).max().item()
    assert worst <= U[dtype] * (1 + 1 / 8), worst


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows", [8192, 40000, 1 << 19, 1 << 20])
def test_dw_of_many_rows_is_rounded_once(dtype, rows):
    x, dy, w = uniform((rows, 64), dtype, 1), uniform((rows, 128), dtype, 2, scale=1 / 256), torch.zeros((64, 128), dtype=dtype, device=DEV)
    dw, db = torch.empty((64, 128), dtype=dtype, device=DEV), torch.empty(128, dtype=dtype, device=DEV)
    dblp.dblp_linear_grad(dy, x, w, dw=dw, dbias=db, ws=space(dblp.dblp_linear_workspace_bytes(x, w, dy)[1]))
    rounded_once(dw, x.double().t() @ dy.double(), dtype)
    rounded_once(db, dy.double().sum(0), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n", [3, 40, 300])
@pytest.mark.parametrize("K", [8192, 16448, 1 << 18])
def test_long_rows_are_rounded_once(dtype, n, K):
    x, w = uniform((n, K), dtype, 1), uniform((K, 304), dtype, 2, scale=1 / 512)
    out, pre = (torch.empty((n, 304), dtype=dtype, device=DEV) for _ in range(2))
    ws = space(max(dblp.dblp_linear_workspace_bytes(x, w, torch.empty((n, 304), dtype=dtype, device=DEV))))
    dblp.dblp_linear(x, w, out, ws=ws, pre=pre, activation="relu")
    want = x.double() @ w.double()
    rounded_once(out, want, dtype)
    rounded_once(pre, want, dtype)
    wt, dx = w.t().contiguous(), torch.empty((n, 304), dtype=dtype, device=DEV)      # the same sum as a gradient: dy = x, w^T
    keep = uniform((n, 304), dtype, 3)
    dblp.dblp_linear_grad(x, keep, wt, dx=dx, ws=space(dblp.dblp_linear_workspace_bytes(keep, wt, x)[1]), pre=keep, activation="relu")
    rounded_once(dx, want, dtype)


def long_dw(rows):
    return pl.grad_w(rows, 9472, 512)


def test_the_long_products_are_not_cut():
    for rows in (512, 8192, 16384):
        (r,) = pl.plans([long_dw(rows)])
        assert r["whole"] > 0 and r["cg"] == 2 and r["bn"] == 256


@pytest.mark.gpu
@pytest.mark.parametrize("signs", list(SIGNED))
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_fp32_results_lose_no_more_with_the_sums_length(dtype, signs):
    """Runs of 512 terms each lose what one of them does, and fp32 additions join them: 2^-24 of the sum each at most."""
    lost = {}
    for rows in (512, 8192, 16384):
        x, dy = uniform((rows, 9472), dtype, 1, *SIGNED[signs]), uniform((rows, 512), dtype, 2, *SIGNED[signs])
        w = torch.zeros((9472, 512), dtype=dtype, device=DEV)
        dw = torch.empty((9472, 512), device=DEV)
        dblp.dblp_linear_grad(dy, x, w, dw=dw, ws=space(dblp.dblp_linear_workspace_bytes(x, w, dy)[1]))
        want = x.double().t() @ dy.double()
        lost[rows] = ((dw.double() - want).norm() / want.norm()).item()
    for rows in (8192, 16384):
        assert lost[rows] <= 2 * lost[512] + rows / 512 * 2.0 ** -24, lost
