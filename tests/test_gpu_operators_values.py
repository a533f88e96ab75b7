"""Attention and its gradient where scores are NaN, infinite or very large, in every place of the groups that the kernels take
them in; the exponential by itself."""
import math

import pytest
import torch

import test_gpu_operators as op

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F16 = torch.bfloat16, torch.float16
NAN, INF = math.nan, math.inf


def case(Sq, D, dtype, B=1, Sk=200, H=2, seed=1):
    """Tensors whose first column makes infinite scores on demand: q has a one there, k a zero."""
    ts = [t.clone() for t in op.tensors(B, Sq, Sk, H, H, D, dtype, seed=seed)]
    ts[0][..., 0] = 1.0
    ts[1][..., 0] = 0.0
    return ts


# One head's key at each place of eight, in both halves of a tile and in the last one; Sq = 3: few rows a key head, 150: tiles.
@pytest.mark.parametrize("Sq", [3, 150])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("at", list(range(8)) + [70, 71, 133, 198, 199])
def test_a_score_that_is_no_number_reaches_its_rows(Sq, D, dtype, bad, at):
    q, k, v, g, out, dq, dk, dv = case(Sq, D, dtype)
    clean = torch.empty_like(out)
    lse0 = op.run_attention(q, k, v, clean)
    k[:, at, 0, 0] = bad                               # of head 0 alone
    lse = op.run_attention(q, k, v, out)
    assert torch.isnan(out[:, :, 0]).all()
    assert (torch.isnan(lse[:, 0]) | (lse[:, 0] == INF)).all()
    assert torch.equal(op.bits(out[:, :, 1]), op.bits(clean[:, :, 1])) and torch.equal(lse[:, 1], lse0[:, 1])
    op.run_grad(q, k, v, out, g, lse, dq, dk, dv)
    for t in (dq, dk, dv):
        assert torch.isnan(t[:, :, 0]).all() and torch.isfinite(t[:, :, 1]).all()


@pytest.mark.parametrize("Sq", [4, 150])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("at", list(range(8)) + [70, 71, 133, 149])
def test_a_query_that_is_no_number_reaches_every_key_it_sees(Sq, D, dtype, at):
    at = at % Sq
    q, k, v, g, out, dq, dk, dv = case(Sq, D, dtype)
    q[:, at, 0, 3] = NAN
    lse = op.run_attention(q, k, v, out)
    assert torch.isnan(out[:, at, 0]).all() and torch.isnan(lse[:, 0, at]).all()
    others = [i for i in range(Sq) if i != at]
    assert torch.isfinite(out[:, others]).all() and torch.isfinite(lse[:, :, others]).all() and torch.isfinite(out[:, :, 1]).all()
    op.run_grad(q, k, v, out, g, lse, dq, dk, dv)
    assert torch.isnan(dq[:, at, 0]).all() and torch.isnan(dk[:, :, 0]).all() and torch.isnan(dv[:, :, 0]).all()
    assert torch.isfinite(dq[:, others]).all()
    for t in (dq, dk, dv):
        assert torch.isfinite(t[:, :, 1]).all()


@pytest.mark.parametrize("Sq", [3, 150])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", list(range(8)) + [133, 199])
def test_a_score_of_minus_infinity_is_a_key_of_no_weight(Sq, D, at):
    q, k, v, g, out, dq, dk, dv = case(Sq, D, BF16)
    k[:, at, :, 0] = -INF
    lse = op.run_attention(q, k, v, out)
    rest = [j for j in range(k.shape[1]) if j != at]
    op.check_forward(q, k[:, rest], v[:, rest], out, lse)


@pytest.mark.parametrize("Sq", [3, 150])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_rows_whose_scores_are_all_minus_infinity_weigh_nothing(Sq, D, causal):
    """Such a row has no largest score: out = 0 and lse = -infinity as for a row that sees no key, and so the gradient."""
    q, k, v, g, out, dq, dk, dv = case(Sq, D, BF16)
    rows = list(range(0, Sq, 2))
    q[..., 0] = 0.0
    q[:, rows, :, 0] = -1e30                           # finite, the products are not
    k[..., 0] = 1e30
    lse = op.run_attention(q, k, v, out, causal=causal)
    assert (out[:, rows] == 0).all() and (lse[:, :, rows] == -INF).all()
    op.run_grad(q, k, v, out, g, lse, dq, dk, dv, causal=causal)
    assert (dq[:, rows] == 0).all()
    got = [t.clone() for t in (dk, dv)]
    q[:, rows, :, 0] = 0.0                             # what the other rows give, with no dout for these
    g[:, rows] = 0
    lse = op.run_attention(q, k, v, out, causal=causal)
    out[:, rows] = 0
    op.run_grad(q, k, v, out, g, lse, dq, dk, dv, causal=causal)
    assert torch.isfinite(got[0]).all() and torch.isfinite(got[1]).all()
    assert torch.equal(got[0], dk) and torch.equal(got[1], dv)


# Scores q0 k0 are exact: q0 a small number, k0 a power of two.  Up to 2^28 in f16, to 2^100 in bf16.
@pytest.mark.parametrize("Sq", [3, 150])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,power", [(F16, 10), (F16, 14), (BF16, 10), (BF16, 14), (BF16, 22), (BF16, 27), (BF16, 31), (BF16, 50), (BF16, 100)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("scale", [0.125, 0.7])
def test_very_large_scores_choose_the_largest(Sq, D, dtype, power, sign, scale):
    """Rows of q0 in (1, 2), keys of k0 = +-2^power or, the ones that win, of a quarter more or less; the exact
    result is the mean of the winners' values."""
    head = 2.0 ** 14 if dtype == F16 else 1.0          # f16: a part of the exponent in q
    q, k, v, g, out, *_ = case(Sq, D, dtype)
    q.zero_()
    q[:, :, 0, 0] = (1 + torch.arange(Sq, device=DEV).remainder(128) / 128) * head
    q[:, :, 1, 0] = q[:, :, 0, 0]
    k.zero_()
    k[..., 0] = sign * 2.0 ** power
    winners = [5, 6, 71, 134]
    k[:, winners, 0, 0] = sign * 2.0 ** power * (1.25 if sign > 0 else 0.75)          # head 1: all keys alike
    lse = op.run_attention(q, k, v, out, scale=scale)
    u, x = op.U[dtype], v[0].double()
    for h, who in ((0, winners), (1, list(range(k.shape[1])))):
        want = x[who, h].mean(0)
        op.within(out[0, :, h], want.expand(Sq, D), (u + op.EXP) * x[who, h].abs().mean(0) + 1.01 * u * want.abs(), "head %d" % h)
        s = q[0, :, h, 0].double() * k[0, who[0], h, 0].double() * float(torch.tensor(scale, dtype=torch.float32))
        want = s + math.log(len(who))
        assert ((lse[0, h].double() - want).abs() <= 2.0 ** -21 * want.abs() + op.EXP).all()


@pytest.mark.parametrize("Sq", [3, 150])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [8, 12, 16, 24, 31, 50, 100])
@pytest.mark.parametrize("start", [-1.0, 1.0])
def test_very_large_scores_that_rise_from_tile_to_tile(Sq, D, power, start):
    """The largest score grows with every 32 keys, from small or from far below zero; the last eight keys win."""
    q, k, v, g, out, *_ = case(Sq, D, BF16)
    q.zero_()
    q[..., 0] = (1 + torch.arange(Sq, device=DEV).remainder(128) / 128)[None, :, None]
    k.zero_()
    j = torch.arange(k.shape[1], device=DEV)
    k[..., 0] = ((start + (j // 32) / 8) * 2.0 ** power)[None, :, None]
    lse = op.run_attention(q, k, v, out, scale=0.7)
    u, x = op.U[BF16], v[0, 192:].double()
    want = x.mean(0)
    op.within(out[0], want.expand(Sq, 2, D), (u + op.EXP) * x.abs().mean(0) + 1.01 * u * want.abs(), "out")
    want = q[0, :, 0, 0].double() * k[0, 199, 0, 0].double() * float(torch.tensor(0.7, dtype=torch.float32)) + math.log(8)
    assert ((lse[0].double() - want).abs() <= 2.0 ** -21 * want.abs() + op.EXP).all()


@pytest.mark.parametrize("Sq,Sk,lens", [(4, 3, None), (300, 200, None), (260, 1, None), (130, 2, None), (400, 128, None), (300, 400, ([300, 200, 257, 40], [100, 200, 1, 0]))])
@pytest.mark.parametrize("D", [64, 128])
def test_queries_that_see_nothing_may_hold_anything(Sq, Sk, lens, D):
    """Causal, more queries than keys: the first ones see no key, and what they hold reaches neither result nor gradient."""
    B = len(lens[0]) if lens else 2
    q, k, v, g, out, dq, dk, dv = case(Sq, D, BF16, B=B, Sk=Sk)
    kw = dict(causal=True, lens=op.lengths(lens))
    got = []
    for poison in (0.0, NAN, INF):
        for b in range(B):
            lq, lk = (lens[0][b], lens[1][b]) if lens else (Sq, Sk)
            for t in (q, g):
                t[b, :max(0, lq - lk)] = poison
        lse = op.run_attention(q, k, v, out, **kw)
        op.run_grad(q, k, v, out, g, lse, dq, dk, dv, **kw)
        got.append([t.clone() for t in (out, lse, dq, dk, dv)])
    assert all(torch.isfinite(t).all() for t in got[0] if t.dtype == BF16)
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(op.bits(a), op.bits(b))


def exponents(dtype):
    """Every exponent from 0 down to -7 in steps of 1/256 (both types hold those below -4 in steps of 1/64 and more alike)."""
    x = -torch.arange(0, 7 * 256 + 1, dtype=torch.float64) / 256
    return x.to(dtype).unique()


@pytest.mark.parametrize("place", range(8))
@pytest.mark.parametrize("D", [64, 128])
def test_the_exponential_by_itself(place, D):
    """Two keys count: one with score 0, one with score x ln 2, so that exp(lse) - 1 is the kernel's 2^x.  log2f and the product with
    ln 2 are off by about 2^-23 of values up to 1, exp(lse) doubles that; the polynomial is off by 2.7e-6, ex2 by 2^-22."""
    x = exponents(F16)
    B, Sq, Sk = x.numel(), 9, 64
    q, k = torch.zeros((B, Sq, 1, D), dtype=F16, device=DEV), torch.zeros((B, Sk, 1, D), dtype=F16, device=DEV)
    q[..., 0] = 1.0
    k[..., 0] = -1000.0
    k[:, 8, 0, 0] = 0.0
    k[:, 16 + place, 0, 0] = x.to(DEV)
    v, out = torch.zeros_like(k), torch.empty_like(q)
    lse = op.run_attention(q, k, v, out, scale=math.log(2))
    got = torch.expm1(lse[:, 0, 0].double()).cpu()
    want = torch.exp2(x.double())
    assert ((got - want).abs() <= 3e-6 * want + 4 * 2.0 ** -23).all(), ((got - want).abs() / want).max()
    assert (lse == lse[:, :, :1]).all()
