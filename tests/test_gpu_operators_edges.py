"""Worker-side operators with nothing to do, or nearly: no queries, no keys, no sequences, no tokens."""
import math

import pytest
import torch

import test_gpu_operators as op
from paper_2605_01989_b200 import binding as dblp

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16, F16 = torch.bfloat16, torch.float16


def pieces(B, Sq, Sk, Hq, Hkv, D, dtype):
    return [t.clone() for t in op.tensors(B, Sq, Sk, Hq, Hkv, D, dtype)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [False, True])
def test_gradient_without_queries_is_zero(D, lens):
    q, k, v, g, out, dq, dk, dv = pieces(3, 0, 300, 4, 2, D, BF16)
    kw = dict(causal=True, lens=op.lengths(([0, 0, 0], [300, 7, 0])) if lens else (None, None))
    lse = op.run_attention(q, k, v, out, **kw)
    for t in (dk, dv):
        t.fill_(7.0)
    op.run_grad(q, k, v, out, g, lse, dq, dk, dv, **kw)
    assert (dk == 0).all() and (dv == 0).all()


@pytest.mark.parametrize("Sq", [1, 3, 200])
@pytest.mark.parametrize("D", [40, 128])
def test_attention_without_keys(Sq, D):
    q, k, v, g, out, dq, dk, dv = pieces(2, Sq, 0, 4, 4, D, F16)
    for t in (out, dq):
        t.fill_(7.0)
    lse = op.run_attention(q, k, v, out)
    assert (out == 0).all() and (lse == -math.inf).all()
    op.run_grad(q, k, v, out, g, lse, dq, dk, dv)
    assert (dq == 0).all()


@pytest.mark.parametrize("Sq", [1, 200])
def test_attention_with_lengths_of_zero(Sq):
    q, k, v, g, out, dq, dk, dv = pieces(2, Sq, 300, 4, 4, 64, BF16)
    for a, b in (([0, 0], [300, 9]), ([Sq, Sq], [0, 0])):
        for t in (out, dq, dk, dv):
            t.fill_(7.0)
        kw = dict(lens=op.lengths((a, b)))
        lse = op.run_attention(q, k, v, out, **kw)
        assert (out == 0).all() and (lse == -math.inf).all()
        op.run_grad(q, k, v, out, g, lse, dq, dk, dv, **kw)
        for t in (dq, dk, dv):
            assert (t == 0).all()


def test_no_sequences():
    q, k, v, g, out, dq, dk, dv = pieces(0, 5, 5, 2, 2, 64, BF16)
    lse = torch.empty((0, 2, 5), device=DEV)
    dblp.dblp_attention(q, k, v, out, lse)
    dblp.dblp_attention_grad(q, k, v, out, g, lse, dq, dk, dv, None)


def test_embed_grad_without_tokens_in_a_graph():
    rows, width = 70, 40
    dout, tokens = torch.empty((0, width), device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    table = torch.full((rows, width), 5.0, device=DEV)
    op.embed_grad(dout, tokens, rows, table)
    assert (table == 0).all()
    ws = torch.empty(dblp.dblp_embed_grad_workspace_bytes(0, rows, width), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dblp.dblp_embed_grad(dout, tokens, table, ws)
    table.fill_(5.0)
    ws.fill_(0xFF)
    graph.replay()
    assert (table == 0).all()
    table.fill_(5.0)
    dblp.dblp_embed_grad(dout, tokens, table, ws, accumulate=True)
    assert (table == 5).all()


@pytest.mark.parametrize("Sq,Sk", [(0, 300), (2, 0), (200, 0), (200, 300)])
def test_gradients_in_a_graph(Sq, Sk):
    q, k, v, g, out, dq, dk, dv = pieces(2, Sq, Sk, 4, 2, 64, BF16)
    lse = op.run_attention(q, k, v, out)
    op.run_grad(q, k, v, out, g, lse, dq, dk, dv)
    want = [t.clone() for t in (dq, dk, dv)]
    ws = torch.empty(dblp.dblp_attention_workspace_bytes(q, k)[1], dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dblp.dblp_attention_grad(q, k, v, out, g, lse, dq, dk, dv, ws)
    for t in (dq, dk, dv):
        t.fill_(7.0)
    graph.replay()
    for a, b in zip(want, (dq, dk, dv)):
        assert torch.equal(op.bits(a), op.bits(b))
