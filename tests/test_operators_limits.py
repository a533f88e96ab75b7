"""Worker-side entry points at the ends of their ranges, before anything touches a device: empty batches, sizes whose products
leave 64 bits."""
import ctypes as C

import pytest
import torch

import test_operators_refusals as refusals
from paper_2605_01989_b200 import binding as dblp

EINVAL, EALIGN, ECAPACITY = -1, -2, -3


def workspace(**kw):
    s = dblp.dblp_attention_t(**{**refusals.SHAPE, **kw})
    f, g = C.c_size_t(77), C.c_size_t(77)
    rc, text = refusals.call("dblp_attention_workspace_bytes", C.byref(s), C.byref(f), C.byref(g))
    return rc, f.value, g.value, text


@pytest.mark.parametrize("q_tokens", [0, 1, 2, 16, 300])
@pytest.mark.parametrize("k_tokens", [0, 1, 300])
def test_an_empty_batch_needs_no_workspace(q_tokens, k_tokens):
    assert workspace(batch=0, q_tokens=q_tokens, k_tokens=k_tokens)[:3] == (0, 0, 0)


@pytest.mark.parametrize("q_tokens", [0, 1, 2, 16, 300])
@pytest.mark.parametrize("k_tokens", [0, 1, 300])
def test_the_workspace_query_knows_every_small_shape(q_tokens, k_tokens):
    rc, f, g, _ = workspace(q_tokens=q_tokens, k_tokens=k_tokens)
    assert rc == 0 and f % 4 == 0 and g % 4 == 0 and max(f, g) < 1 << 24


@pytest.mark.parametrize("rows,cols", [(1 << 39, 1 << 31), (1 << 33, 1 << 31), ((1 << 33) + 1, 1 << 31), ((1 << 40) - 1, 0xFFFFFFFF),
                                       (1 << 40, 2), (1 << 41, 1), (1 << 63, 2), ((1 << 64) - 1, 1)])
def test_dropout_counts_its_elements_beyond_64_bits(rows, cols):
    rc, text = refusals.dropout(rows=rows, cols=cols, xs=cols, os=cols)
    assert rc == ECAPACITY and "elements" in text


@pytest.mark.parametrize("kw", [dict(batch=65535, q_heads=65535, kv_heads=65535, q_tokens=(1 << 30) - 1, k_tokens=1 << 29),
                                dict(batch=65535, q_heads=65535, kv_heads=65535, q_tokens=(1 << 30) - 1, k_tokens=0),
                                dict(batch=65535, q_heads=65535, kv_heads=1, q_tokens=(1 << 30) - 1, k_tokens=1 << 29, head_dim=128)])
def test_a_workspace_beyond_64_bits_is_refused(kw):
    rc, _, _, text = workspace(**kw)
    assert rc == ECAPACITY and "workspace" in text


def test_a_large_workspace_is_counted_in_full():
    """One sequence of 2^29 tokens, 8 heads of 128: at least one fp32 copy of q and 8 bytes a row."""
    n = 1 << 29
    rc, _, g, _ = workspace(batch=1, q_heads=8, kv_heads=8, q_tokens=n, k_tokens=n, head_dim=128)
    assert rc == 0 and g >= n * 8 * (128 * 4 + 8)


A = refusals.A


@pytest.mark.parametrize("name,args", [
    ("dblp_embed", (A, 64, 10, 64, 0, A, 4, 5, -1, 1.0, A, 64, 0, A + 4, None)),
    ("dblp_embed_grad", (A, 64, 0, A, 4, 5, -1, 1.0, A, 64, 10, 64, 0, 0, A + 4, A, 1 << 30, None))])
def test_a_counter_off_its_boundary_is_refused(name, args):
    rc, text = refusals.call(name, *args)
    assert rc == EALIGN and "bad_tokens" in text


@pytest.mark.parametrize("which", ["q_lens", "k_lens"])
def test_lengths_off_their_boundary_are_refused(which):
    for rc, text in (refusals.attention(**{which: A + 2}), refusals.attention_grad(**{which: A + 2})):
        assert rc == EALIGN and "lengths" in text


def test_lse_off_its_boundary_is_refused():
    s, h = dblp.dblp_attention_t(**refusals.SHAPE), refusals.heads
    forward = refusals.call("dblp_attention", C.byref(s), h(), h(), h(), h(), A + 2, None, 0, None)
    for rc, text in (forward, refusals.attention_grad(lse=A + 1)):
        assert rc == EALIGN and "lse" in text


# Calls through the binding with tensors that have shapes and no memory: they end in a refusal, the binding's or the library's
# for the null address.
@pytest.fixture
def anywhere(monkeypatch):
    monkeypatch.setattr(dblp, "_on_device", lambda *t: None)


def meta(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


WIDE = (1 << 32) + 8


@pytest.mark.parametrize("call", [
    lambda: dblp.dblp_dropout(meta(1, WIDE), meta(1, WIDE), 0.1, 1, 2, 3, stream=0),
    lambda: dblp.dblp_dropout_grad(meta(1, WIDE), meta(1, WIDE), 0.1, 1, 2, 3, stream=0),
    lambda: dblp.dblp_dropout(meta(4, 8), meta(4, 8), 0.1, 1, 1 << 32, 3, stream=0),
    lambda: dblp.dblp_dropout(meta(4, 8), meta(4, 8), 0.1, 1, -1, 3, stream=0),
    lambda: dblp.dblp_dropout(meta(4, 8), meta(4, 8), 0.1, 1, 2, (1 << 32) + 3, stream=0),
    lambda: dblp.dblp_dropout_grad(meta(4, 8), meta(4, 8), 0.1, 1, 2, (1 << 32) + 3, stream=0),
    lambda: dblp.dblp_embed(meta(4, WIDE), meta(2, dtype=torch.int32), meta(2, WIDE), stream=0),
    lambda: dblp.dblp_embed_grad(meta(2, WIDE), meta(2, dtype=torch.int32), meta(4, WIDE), None, stream=0),
    lambda: dblp.dblp_embed_grad_workspace_bytes(5, 5, WIDE),
    lambda: dblp.dblp_attention_workspace_bytes(meta(1, 5, 2, 64), meta(1, WIDE, 2, 64))])
def test_what_does_not_fit_in_32_bits_is_refused(anywhere, call):
    with pytest.raises(ValueError, match="32 bits"):
        call()


@pytest.mark.parametrize("call", [
    lambda ws: dblp.dblp_embed_grad(meta(2, 8), meta(2, dtype=torch.int32), meta(4, 8), ws, stream=0),
    lambda ws: dblp.dblp_attention(*(meta(1, 5, 2, 64) for _ in range(4)), ws=ws, stream=0),
    lambda ws: dblp.dblp_attention_grad(*(meta(1, 5, 2, 64) for _ in range(5)), meta(1, 2, 5, dtype=torch.float32),
                                        *(meta(1, 5, 2, 64) for _ in range(3)), ws, stream=0)])
def test_a_workspace_with_gaps_is_refused(anywhere, call):
    """What lies in the gaps is not the workspace's to write."""
    with pytest.raises(ValueError, match="workspace"):
        call(meta(1 << 20, 2, dtype=torch.uint8)[:, 0])
