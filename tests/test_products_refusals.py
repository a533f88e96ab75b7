"""What dblp_norm_rotate, dblp_linear, dblp_orthogonalize and their gradients refuse, before anything touches a device."""
import ctypes as C

import pytest
import torch

from paper_2605_01989_b200 import binding as dblp

EINVAL, EALIGN, ECAPACITY = -1, -2, -3
A = 1 << 20                                            # an address that is never read


def call(name, *args):
    rc = getattr(dblp.lib(), name)(*args)
    return rc, dblp.lib().dblp_last_error().decode()


# ---- norm and rotation ---------------------------------------------------------------------------------------------------
def heads(data=A, batch=16 * 4 * 64, token=4 * 64, head=64):
    return C.byref(dblp.dblp_heads_t(data, batch, token, head))


ROTATE = dict(batch=2, tokens=16, q_heads=4, k_heads=4, head_dim=64, rotary_dim=64, dtype=1, weight_dtype=0, flags=0, eps=1e-6, positions=A,
              position_stride=16, freqs=A)


def rotate(q=None, q_out=None, k=None, k_out=None, q_weight=A, **kw):
    a = dblp.dblp_norm_rotate_t(**{**ROTATE, **kw})
    return call("dblp_norm_rotate", C.byref(a), q or heads(), q_weight, q_out or heads(), k or heads(), A, k_out or heads(), None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(dtype=4), EINVAL, "dtype"), (dict(weight_dtype=-1), EINVAL, "dtype"), (dict(head_dim=0), EINVAL, "head_dim"), (dict(head_dim=60), EINVAL, "head_dim"),
    (dict(head_dim=264), EINVAL, "head_dim"), (dict(flags=1), EINVAL, "flags"), (dict(flags=4), EINVAL, "flags"), (dict(rotary_dim=72), EINVAL, "rotary_dim"),
    (dict(rotary_dim=24), EINVAL, "rotary_dim"), (dict(rotary_dim=31, flags=2), EINVAL, "rotary_dim"), (dict(eps=0.0), EINVAL, "eps"),
    (dict(eps=float("nan")), EINVAL, "eps"), (dict(eps=float("inf")), EINVAL, "eps"), (dict(tokens=1 << 31), ECAPACITY, "heads"),
    (dict(tokens=1 << 28), ECAPACITY, "heads"), (dict(positions=None), EINVAL, "positions"), (dict(freqs=None), EINVAL, "freqs"),
    (dict(positions=A + 2), EALIGN, "positions"), (dict(freqs=A + 4), EALIGN, "freqs"), (dict(q=heads(data=None)), EINVAL, "q is null"),
    (dict(k=heads(data=A + 8)), EALIGN, "k has"), (dict(q=heads(token=60)), EALIGN, "q has"), (dict(q=heads(token=-256)), EINVAL, "stride"),
    (dict(q_out=heads(head=32)), EINVAL, "overlap"), (dict(k_out=heads(token=0)), EINVAL, "overlap"), (dict(q_weight=A + 2), EALIGN, "q_weight")])
def test_norm_rotate_refuses(kw, status, word):
    rc, text = rotate(**kw)
    assert rc == status and "norm_rotate" in text and word in text


def rotate_grad(ws=A, wb=1 << 30, dw=A, dq=None, **kw):
    a = dblp.dblp_norm_rotate_t(**{**ROTATE, **kw})
    return call("dblp_norm_rotate_grad", C.byref(a), heads(), A, heads(), dq or heads(), dw, heads(), A, heads(), heads(), dw, ws, wb, None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(ws=None), EINVAL, "workspace"), (dict(ws=A + 64), EALIGN, "workspace"), (dict(wb=64), ECAPACITY, "workspace"), (dict(dq=heads(head=0)), EINVAL, "overlap"),
    (dict(dw=A + 1), EALIGN, "weight"), (dict(flags=8), EINVAL, "flags")])
def test_norm_rotate_grad_refuses(kw, status, word):
    rc, text = rotate_grad(**kw)
    assert rc == status and "norm_rotate_grad" in text and word in text


# ---- linear ----------------------------------------------------------------------------------------------------------------
def matrix(data=A, rows=64, cols=1):
    return C.byref(dblp.dblp_matrix_t(data, rows, cols))


LINEAR = dict(rows=16, in_=64, out=64, dtype=1, out_dtype=1, bias_dtype=0, activation=0, flags=0)


def linear(x=None, w=None, bias=None, residual=None, pre=None, out=None, ws=A, wb=1 << 40, **kw):
    l = dblp.dblp_linear_t(**{**LINEAR, **kw})
    return call("dblp_linear", C.byref(l), x or matrix(), w or matrix(), bias, residual, pre, out or matrix(), ws, wb, None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(dtype=0), EINVAL, "dtype"), (dict(out_dtype=2), EINVAL, "out_dtype"), (dict(bias_dtype=7), EINVAL, "bias"), (dict(activation=5), EINVAL, "activation"),
    (dict(activation=-1), EINVAL, "activation"), (dict(flags=1), EINVAL, "flags"), (dict(rows=1 << 31), ECAPACITY, "2^31"), (dict(x=matrix(data=None)), EINVAL, "x is null"),
    (dict(x=matrix(data=A + 1)), EALIGN, "x is not"), (dict(x=matrix(rows=1, cols=64)), EINVAL, "x has strides"), (dict(w=matrix(rows=2, cols=2)), EINVAL, "w has strides"),
    (dict(w=matrix(data=None)), EINVAL, "w is null"), (dict(x=matrix(rows=1 << 38)), EINVAL, "stride"), (dict(out=matrix(rows=63)), EINVAL, "overlap"),
    (dict(out=matrix(rows=0)), EINVAL, "overlap"), (dict(out=matrix(data=None)), EINVAL, "out is null"), (dict(residual=matrix(data=None)), EINVAL, "residual is null"),
    (dict(pre=matrix(rows=8)), EINVAL, "overlap"), (dict(bias=A + 2), EALIGN, "bias"), (dict(x=matrix(data=A + 2), ws=None), EINVAL, "workspace"),
    (dict(x=matrix(data=A + 2), ws=A + 16), EALIGN, "workspace"), (dict(x=matrix(data=A + 2), wb=0), ECAPACITY, "workspace")])
def test_linear_refuses(kw, status, word):
    rc, text = linear(**kw)
    assert rc == status and "linear" in text and word in text


def linear_grad(dy=None, x=None, w=None, residual=None, pre=None, dx=None, dw=None, db=None, ws=A, wb=1 << 40, **kw):
    l = dblp.dblp_linear_t(**{**LINEAR, **kw})
    return call("dblp_linear_grad", C.byref(l), dy or matrix(), x or matrix(), w or matrix(), residual, pre, dx, dw, db, ws, wb, None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(flags=2), EINVAL, "flags"), (dict(dx=matrix(), activation=2), EINVAL, "pre"), (dict(dx=matrix(), pre=matrix()), EINVAL, "pre"),
    (dict(dx=matrix(rows=60)), EINVAL, "overlap"), (dict(dw=matrix(rows=3, cols=2)), EINVAL, "dw has strides"), (dict(dw=matrix(rows=1, cols=60)), EINVAL, "overlap"),
    (dict(dw=matrix(), x=matrix(data=None)), EINVAL, "x is null"), (dict(dx=matrix(), w=matrix(data=None)), EINVAL, "w is null"),
    (dict(dx=matrix(), dy=matrix(data=None)), EINVAL, "dy is null"), (dict(db=A + 1), EALIGN, "dbias"), (dict(db=A, ws=None), EINVAL, "workspace"),
    (dict(db=A, wb=16), ECAPACITY, "workspace"), (dict(dw=matrix(data=A + 2), out_dtype=0), EALIGN, "dw is not")])
def test_linear_grad_refuses(kw, status, word):
    rc, text = linear_grad(**kw)
    assert rc == status and "linear_grad" in text and word in text


def test_linear_workspace_is_for_what_cannot_be_read_in_place():
    size = lambda n, i, o, off: dblp.dblp_linear_workspace_bytes(torch.empty(n * i + 8, dtype=torch.bfloat16)[off:off + n * i].view(n, i),
                                                                torch.empty((i, o), dtype=torch.bfloat16))[0]
    assert size(8192, 1600, 6400, 0) <= size(8192, 1600, 6400, 1) - 8192 * 1600 * 2
    l = dblp.dblp_linear_t(**{**LINEAR, "rows": (1 << 31) - 1, "in_": (1 << 31) - 1, "out": (1 << 31) - 1})
    n = C.c_size_t()
    rc, text = call("dblp_linear_workspace_bytes", C.byref(l), matrix(data=A + 2), matrix(data=A + 2), None, C.byref(n), None)
    assert rc == ECAPACITY or n.value < 1 << 63


# ---- orthogonalised update ---------------------------------------------------------------------------------------------------
def ortho(x=A, out=A, ws=A, wb=1 << 40, coefficients=(1.5, -0.5, 0.0), **kw):
    a = dict(batch=2, rows=8, cols=64, x_dtype=0, out_dtype=1, steps=1, eps=0.0, scale=1.0, x_batch_stride=512, x_row_stride=64, out_batch_stride=512,
             out_row_stride=64)
    a.update(kw)
    c = None if coefficients is None else (C.c_float * len(coefficients))(*coefficients)
    return call("dblp_orthogonalize", C.byref(dblp.dblp_orthogonalize_t(coefficients=c, **a)), x, out, ws, wb, None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(x_dtype=3), EINVAL, "dtype"), (dict(out_dtype=-2), EINVAL, "dtype"), (dict(rows=32769), ECAPACITY, "32768"), (dict(batch=65536), ECAPACITY, "65536"),
    (dict(steps=0), EINVAL, "steps"), (dict(steps=17), EINVAL, "steps"), (dict(coefficients=None), EINVAL, "coefficients"),
    (dict(coefficients=(1.0, float("inf"), 0.0)), EINVAL, "coefficient"), (dict(eps=-1.0), EINVAL, "eps"), (dict(eps=float("nan")), EINVAL, "eps"),
    (dict(scale=float("inf")), EINVAL, "scale"), (dict(x=None), EINVAL, "null"), (dict(out=None), EINVAL, "null"), (dict(x=A + 2), EALIGN, "aligned"),
    (dict(out=A + 1), EALIGN, "aligned"), (dict(x_row_stride=-64), EINVAL, "stride"), (dict(out_row_stride=60), EINVAL, "overlap"),
    (dict(out_batch_stride=100), EINVAL, "overlap"), (dict(ws=None), EINVAL, "workspace"), (dict(ws=A + 128), EALIGN, "workspace"), (dict(wb=1000), ECAPACITY, "workspace")])
def test_orthogonalize_refuses(kw, status, word):
    rc, text = ortho(**kw)
    assert rc == status and "orthogonalize" in text and word in text


def test_nothing_to_do_is_ok():
    assert rotate(batch=0)[0] == 0 and rotate(tokens=0)[0] == 0 and rotate(q_heads=0, k_heads=0)[0] == 0
    assert linear(rows=0)[0] == 0
    none = dblp.dblp_linear_t(**{**LINEAR, "out": 0})
    assert call("dblp_linear", C.byref(none), matrix(), matrix(), None, None, None, None, None, 0, None)[0] == 0
    assert linear_grad()[0] == 0 and linear_grad(rows=0, dx=matrix())[0] == 0
    assert ortho(batch=0)[0] == 0 and ortho(rows=0)[0] == 0 and ortho(cols=0)[0] == 0


def test_the_binding_checks_shapes_types_and_names():
    x, w, out = torch.zeros((4, 8), dtype=torch.bfloat16), torch.zeros((8, 16), dtype=torch.bfloat16), torch.zeros((4, 16), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):
        dblp.dblp_linear(x, w, out)
    with pytest.raises(ValueError, match="rows x in"):
        dblp.dblp_linear_workspace_bytes(x, w.t())
    with pytest.raises(ValueError, match="dtype"):
        dblp.dblp_linear_workspace_bytes(x, w.float())
    with pytest.raises(ValueError, match="activation"):
        dblp._linear(x, w, None, None, "tanh", 0)
    with pytest.raises(ValueError, match="shape"):
        dblp.dblp_orthogonalize_workspace_bytes(x, out)
    with pytest.raises(ValueError, match="triples"):
        dblp._orthogonalize(x, x, [(1.0, 2.0)], 0.0, 1.0)
    with pytest.raises(ValueError, match="batch"):
        dblp.dblp_norm_rotate_grad_workspace_bytes(torch.zeros((1, 2, 3, 64)), torch.zeros((1, 3, 3, 64)))


def test_structs():
    assert C.sizeof(dblp.dblp_norm_rotate_t) == 64 and C.sizeof(dblp.dblp_matrix_t) == 24 and C.sizeof(dblp.dblp_linear_t) == 32
    assert C.sizeof(dblp.dblp_orthogonalize_t) == 72
