"""Results that lie over what other blocks still read are refused; neighbours between whose lines they lie are not."""
import ctypes as C

import pytest
import torch

from paper_2605_01989_b200 import binding as dblp

EINVAL = -1
A = 1 << 20                                            # addresses that are never read
FAR = [A + (k << 24) for k in range(10)]
DEV = "cuda:0"


def matrix(data, row=64, col=1):
    return C.byref(dblp.dblp_matrix_t(data, row, col))


def linear(bias=None, residual=None, pre=None, x=FAR[0], w=FAR[1], out=FAR[2], bias_dtype=0, **kw):
    l = dblp.dblp_linear_t(**{**dict(rows=16, in_=64, out=64, dtype=1, out_dtype=1, bias_dtype=bias_dtype, activation=0, flags=0), **kw})
    m = lambda t: t if t is None or not isinstance(t, int) else matrix(t)
    rc = dblp.lib().dblp_linear(C.byref(l), m(x), m(w), bias, m(residual), m(pre), m(out), FAR[9], 1 << 40, None)
    return rc, dblp.lib().dblp_last_error().decode()


@pytest.mark.parametrize("kw,words", [
    (dict(out=FAR[0]), "out lies over x"), (dict(out=FAR[0], residual=FAR[0]), "out lies over x"), (dict(out=FAR[1]), "out lies over w"),
    (dict(out=FAR[0] + 2), "out lies over x"), (dict(out=FAR[0] + 15 * 128 + 126), "out lies over x"), (dict(out=FAR[0] - 15 * 128 - 126), "out lies over x"),
    (dict(pre=FAR[0]), "pre lies over x"), (dict(pre=FAR[1] + 64 * 128 - 2), "pre lies over w"), (dict(pre=FAR[2]), "pre lies over out"),
    (dict(pre=FAR[3], residual=FAR[3]), "pre lies over residual"), (dict(residual=FAR[2] + 16), "out lies over residual"),
    (dict(residual=matrix(FAR[2], 128)), "out lies over residual"), (dict(bias=FAR[2] + 128), "out lies over bias"), (dict(pre=FAR[3], bias=FAR[3] + 4), "pre lies over bias"),
    # lines of one stride: 64 of 160 elements a line, and one element too many
    (dict(x=matrix(FAR[0], 160), out=matrix(FAR[0] + 126, 160)), "out lies over x"), (dict(x=matrix(FAR[0] + 126, 160), out=matrix(FAR[0] + 5 * 320, 160)), "out lies over x"),
    # from the last line up
    (dict(x=matrix(FAR[0] + 15 * 128, -64), out=matrix(FAR[0] + 15 * 128 + 126)), "out lies over x"),
    # the transposed view of weights held as [out, in]
    (dict(w=matrix(FAR[1], 1, 64), out=FAR[1] + 63 * 128 + 126), "out lies over w")])
def test_linear_refuses_results_over_what_it_reads(kw, words):
    rc, text = linear(**kw)
    assert rc == EINVAL and words in text, (rc, text)


def linear_grad(dy=FAR[0], x=FAR[1], w=FAR[2], dx=None, dw=None, db=None, residual=None, pre=None, **kw):
    l = dblp.dblp_linear_t(**{**dict(rows=16, in_=64, out=64, dtype=1, out_dtype=1, bias_dtype=0, activation=2 if pre else 0, flags=0), **kw})
    m = lambda t: t if t is None or not isinstance(t, int) else matrix(t)
    rc = dblp.lib().dblp_linear_grad(C.byref(l), m(dy), m(x), m(w), m(residual), m(pre), m(dx), m(dw), db, FAR[9], 1 << 40, None)
    return rc, dblp.lib().dblp_last_error().decode()


@pytest.mark.parametrize("kw,words", [
    (dict(dx=FAR[0]), "dx lies over dy"), (dict(dx=FAR[0], residual=FAR[0]), "dx lies over dy"), (dict(dx=FAR[2]), "dx lies over w"),
    (dict(dx=FAR[3], residual=FAR[3] + 2), "dx lies over residual"), (dict(dx=FAR[3], pre=FAR[3] + 128), "dx lies over pre"), (dict(dw=FAR[0]), "dw lies over dy"),
    (dict(dw=FAR[1] + 1024), "dw lies over x"), (dict(dx=FAR[3], dw=FAR[2]), "dw lies over w"), (dict(dx=FAR[3], dw=FAR[4], pre=FAR[4]), "dw lies over pre"),
    (dict(dx=FAR[3], dw=FAR[4], residual=FAR[4]), "dw lies over residual"), (dict(dx=FAR[3], dw=FAR[3]), "dx lies over dw"), (dict(db=FAR[0]), "dbias lies over dy"),
    (dict(dw=FAR[3], db=FAR[3] + 128), "dw lies over dbias"), (dict(dx=FAR[3], db=FAR[3] + 128), "dx lies over dbias"), (dict(dx=FAR[3], db=FAR[2]), "dbias lies over w"),
    (dict(dw=FAR[3], db=FAR[1]), "dbias lies over x")])
def test_linear_grad_refuses_results_over_what_it_reads(kw, words):
    rc, text = linear_grad(**kw)
    assert rc == EINVAL and words in text, (rc, text)


def randn(shape, seed, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def space(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("n,d", [(3, 64), (40, 64), (300, 136)])
def test_results_between_the_lines_of_operands(n, d):
    buf, w, bias = randn((n, 4 * d), 1), randn((d, d), 2), randn((d,), 3, torch.float32)
    part = lambda t, k: t[:, k * d:(k + 1) * d]
    want, wpre = torch.empty((n, d), dtype=torch.bfloat16, device=DEV), torch.empty((n, d), dtype=torch.bfloat16, device=DEV)
    keep = buf.clone()
    ws = space(max(dblp.dblp_linear_workspace_bytes(part(buf, 1), w, part(buf, 0))))
    dblp.dblp_linear(part(keep, 1), w, want, ws=ws, bias=bias, residual=part(keep, 2), pre=wpre, activation="gelu")
    dblp.dblp_linear(part(buf, 1), w, part(buf, 2), ws=ws, bias=bias, residual=part(buf, 2), pre=part(buf, 0), activation="gelu")
    assert torch.equal(part(buf, 2), want) and torch.equal(part(buf, 0), wpre)
    assert torch.equal(part(buf, 1), part(keep, 1)) and torch.equal(part(buf, 3), part(keep, 3))
    # dw behind dbias in one flat vector, dx over x beside dy
    buf, flat = keep.clone(), torch.zeros(d * d + d, device=DEV)
    dx, dw, db = torch.empty_like(want), torch.empty((d, d), device=DEV), torch.empty(d, device=DEV)
    dblp.dblp_linear_grad(part(keep, 0), part(keep, 1), w, dx=dx, dw=dw, dbias=db, ws=ws)
    dblp.dblp_linear_grad(part(buf, 0), part(buf, 1), w, dx=part(buf, 1), dw=flat[d:].view(d, d), dbias=flat[:d], ws=ws)
    assert torch.equal(part(buf, 1), dx) and torch.equal(flat[d:].view(d, d), dw) and torch.equal(flat[:d], db)
