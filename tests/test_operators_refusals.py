"""What the worker-side entry points refuse, before anything touches a device: status, and a text that names the reason."""
import ctypes as C

import pytest
import torch

from paper_2605_01989_b200 import binding as dblp

EINVAL, EALIGN, ECAPACITY = -1, -2, -3
A = 1 << 20                                            # an address that is never read


def call(name, *args):
    rc = getattr(dblp.lib(), name)(*args)
    return rc, dblp.lib().dblp_last_error().decode()


def embed(**kw):
    a = dict(table=A, ts=64, rows=10, width=64, tdt=0, tok=A, tb=4, n=5, pad=-1, scale=1.0, out=A, os=64, odt=0)
    a.update(kw)
    return call("dblp_embed", a["table"], a["ts"], a["rows"], a["width"], a["tdt"], a["tok"], a["tb"], a["n"], a["pad"], a["scale"],
                a["out"], a["os"], a["odt"], None, None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(tdt=7), EINVAL, "dtype"), (dict(odt=-1), EINVAL, "dtype"), (dict(tb=2), EINVAL, "tokens"), (dict(tok=A + 2), EALIGN, "tokens"),
    (dict(table=None), EINVAL, "null"), (dict(out=None), EINVAL, "null"), (dict(tok=None), EINVAL, "null"), (dict(os=63), EINVAL, "overlap"),
    (dict(os=0), EINVAL, "overlap"), (dict(rows=1 << 31), ECAPACITY, "rows"), (dict(out=A + 1), EALIGN, "aligned")])
def test_embed_refuses(kw, status, word):
    rc, text = embed(**kw)
    assert rc == status and "embed" in text and word in text


def test_nothing_to_do_is_ok():
    assert embed(n=0, tok=None, out=None)[0] == 0
    assert embed(width=0)[0] == 0
    assert dropout(rows=0, x=None, out=None)[0] == 0
    assert attention(batch=0)[0] == 0
    assert attention(q_tokens=0)[0] == 0


def embed_grad(**kw):
    a = dict(dout=A, ds=64, ddt=0, tok=A, tb=4, n=5, pad=-1, scale=1.0, table=A, ts=64, rows=10, width=64, tdt=0, flags=0, ws=A, wb=1 << 30)
    a.update(kw)
    return call("dblp_embed_grad", a["dout"], a["ds"], a["ddt"], a["tok"], a["tb"], a["n"], a["pad"], a["scale"], a["table"], a["ts"],
                a["rows"], a["width"], a["tdt"], a["flags"], None, a["ws"], a["wb"], None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(ddt=3), EINVAL, "dtype"), (dict(flags=2), EINVAL, "flags"), (dict(n=1 << 31), ECAPACITY, "tokens"), (dict(dout=None), EINVAL, "null"),
    (dict(table=None), EINVAL, "null"), (dict(ts=10), EINVAL, "overlap"), (dict(ws=None), EINVAL, "workspace"), (dict(ws=A + 16), EALIGN, "workspace"),
    (dict(wb=100), ECAPACITY, "workspace"), (dict(tok=A + 1), EALIGN, "tokens")])
def test_embed_grad_refuses(kw, status, word):
    rc, text = embed_grad(**kw)
    assert rc == status and "embed_grad" in text and word in text


def test_embed_grad_workspace_grows_with_the_tokens():
    small, large = (dblp.dblp_embed_grad_workspace_bytes(n, 50257, 1600) for n in (100, 100000))
    assert 0 < small < large
    with pytest.raises(dblp.DblpError):
        dblp.dblp_embed_grad_workspace_bytes(1 << 31, 10, 10)


def dropout(**kw):
    a = dict(x=A, xs=64, res=None, rs=0, out=A, os=64, rows=4, cols=64, dt=1, p=0.1, seed=1, step=2, site=3)
    a.update(kw)
    return call("dblp_dropout", a["x"], a["xs"], a["res"], a["rs"], a["out"], a["os"], a["rows"], a["cols"], a["dt"], a["p"], a["seed"],
                a["step"], a["site"], None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(dt=9), EINVAL, "dtype"), (dict(p=-0.1), EINVAL, "p ="), (dict(p=1.5), EINVAL, "p ="), (dict(p=float("nan")), EINVAL, "p ="),
    (dict(site=1 << 24), EINVAL, "site"), (dict(x=None), EINVAL, "null"), (dict(out=None), EINVAL, "null"), (dict(os=32), EINVAL, "overlap"),
    (dict(rows=1 << 41), ECAPACITY, "elements"), (dict(x=A + 1), EALIGN, "aligned"), (dict(res=A + 1, rs=64), EALIGN, "aligned")])
def test_dropout_refuses(kw, status, word):
    rc, text = dropout(**kw)
    assert rc == status and "dropout" in text and word in text


SHAPE = dict(batch=2, q_tokens=16, k_tokens=16, q_heads=4, kv_heads=2, head_dim=64, dtype=1, flags=0, scale=0.125)


def heads(data=A, batch=16 * 4 * 64, token=4 * 64, head=64):
    return C.byref(dblp.dblp_heads_t(data, batch, token, head))


def attention(q=None, k=None, v=None, out=None, **kw):
    s = dblp.dblp_attention_t(**{**SHAPE, **kw})
    return call("dblp_attention", C.byref(s), q or heads(), k or heads(), v or heads(), out or heads(), None, None, 0, None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(dtype=0), EINVAL, "dtype"), (dict(head_dim=0), EINVAL, "head_dim"), (dict(head_dim=60), EINVAL, "head_dim"),
    (dict(head_dim=136), EINVAL, "head_dim"), (dict(kv_heads=3), EINVAL, "divide"), (dict(kv_heads=0), EINVAL, "divide"),
    (dict(flags=4), EINVAL, "flags"), (dict(scale=0.0), EINVAL, "scale"), (dict(scale=float("nan")), EINVAL, "scale"),
    (dict(scale=float("inf")), EINVAL, "scale"), (dict(q_tokens=1 << 30), ECAPACITY, "tokens"),
    (dict(q=heads(data=None)), EINVAL, "q is null"), (dict(v=heads(data=A + 8)), EALIGN, "v has"), (dict(k=heads(token=60)), EALIGN, "k has"),
    (dict(k=heads(token=-256)), EINVAL, "stride"), (dict(out=heads(token=0)), EINVAL, "overlap"), (dict(out=heads(head=32)), EINVAL, "overlap"),
    (dict(out=heads(batch=256)), EINVAL, "overlap")])
def test_attention_refuses(kw, status, word):
    rc, text = attention(**kw)
    assert rc == status and "attention" in text and word in text


def attention_grad(lse=A, ws=A, wb=1 << 30, dk=None, dq=None, **kw):
    s = dblp.dblp_attention_t(**{**SHAPE, **kw})
    return call("dblp_attention_grad", C.byref(s), heads(), heads(), heads(), heads(), heads(), lse, dq or heads(), dk or heads(), heads(),
                ws, wb, None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(lse=None), EINVAL, "lse"), (dict(ws=None), EINVAL, "workspace"), (dict(ws=A + 8), EALIGN, "workspace"), (dict(wb=8), ECAPACITY, "workspace"),
    (dict(dk=heads(head=0)), EINVAL, "overlap"), (dict(dq=heads(batch=0)), EINVAL, "overlap"), (dict(dtype=5), EINVAL, "dtype")])
def test_attention_grad_refuses(kw, status, word):
    rc, text = attention_grad(**kw)
    assert rc == status and "attention_grad" in text and word in text


def test_f16_is_not_a_plan_type():
    with pytest.raises(dblp.DblpError) as e:
        dblp.Plan([1000], dblp.DBLP_F16, 1024, 2)
    assert e.value.status == EINVAL


def test_the_binding_checks_shapes_types_and_places():
    x = torch.zeros((4, 8))
    with pytest.raises(ValueError, match="current device"):
        dblp.dblp_dropout(x, x, 0.1, 1, 2, 3)


def test_structs_of_the_worker_side():
    assert C.sizeof(dblp.dblp_heads_t) == 32 and C.sizeof(dblp.dblp_attention_t) == 56
