"""The decoder block's step: its gradient against 64-bit automatic differentiation of the same model, and rounds of it through the
lossy transport with the orthogonalised update."""
import math

import pytest
import torch

from paper_2605_01989_b200 import binding as dblp
from paper_2605_01989_b200 import worker as wk

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def reference_loss(p, x, want, model, batch, tokens):
    d, n, H, D = model.width, batch * tokens, model.heads, model.head_dim
    x0 = p["table"][x.reshape(-1).long()] * math.sqrt(d)
    q, k, v = (x0 @ p["w_qkv"]).view(batch, tokens, 3, H, D).unbind(2)
    angle = (torch.arange(tokens, device=DEV).double()[:, None] * model.freqs)[:, None]
    c, s = torch.cat((angle.cos(),) * 2, -1), torch.cat((angle.sin(),) * 2, -1)

    def turn(y, w):
        y = y * (y.pow(2).mean(-1, keepdim=True) + 1e-6).rsqrt() * w
        return y * c + torch.cat((-y[..., D // 2:], y[..., :D // 2]), -1) * s

    q, k = turn(q, p["q_norm"]), turn(k, p["k_norm"])
    q, k, v = (t.transpose(1, 2) for t in (q, k, v))
    scores = (q @ k.transpose(2, 3)) / math.sqrt(D)
    scores = scores.masked_fill(torch.ones((tokens, tokens), dtype=torch.bool, device=DEV).triu(1), -math.inf)
    x1 = (scores.softmax(3) @ v).transpose(1, 2).reshape(n, d) @ p["w_out"] + x0
    x2 = torch.nn.functional.gelu(x1 @ p["w_up"] + p["b_up"]) @ p["w_down"] + p["b_down"] + x1
    return torch.nn.functional.cross_entropy(x2 @ p["table"].t(), want.reshape(-1).long())


@pytest.mark.parametrize("batch,tokens,heads,head_dim", [(2, 150, 2, 64), (1, 45, 3, 128)])
def test_the_gradient_is_that_of_the_block(batch, tokens, heads, head_dim):
    torch.cuda.set_device(0)
    rows = 300
    model = wk.BlockModel(rows, heads, head_dim, DEV, seed=3)
    w = wk.BlockWorker(model, batch, tokens)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    x, want = (torch.randint(0, rows, (batch, tokens), generator=g, device=DEV, dtype=torch.int32) for _ in range(2))
    loss = w.step(x, want, 1)
    params = {n: t.detach().double().requires_grad_() for n, t in model.views(model.flat).items()}
    exact = reference_loss(params, x, want, model, batch, tokens)
    exact.backward()
    assert abs(loss.item() - exact.item()) < 2.0 ** -8 * abs(exact.item())
    # A gradient passes at most about 20 roundings to bf16 of random sign, each 2^-8 at most and 2^-9.8 on average: their root sum of
    # squares is below 1 %; three times that.  The norms' gradients are sums of terms that nearly cancel over the batch: ten times.
    for name, got in model.views(w.grad).items():
        rel = ((got.double() - params[name].grad).norm() / params[name].grad.norm()).item()
        assert rel < (0.1 if "norm" in name else 0.03), (name, rel)
    assert dblp.dblp_wait_timeouts() == 0


def test_the_step_replays_from_a_graph():
    torch.cuda.set_device(0)
    model = wk.BlockModel(256, 2, 64, DEV, seed=1)
    w = wk.BlockWorker(model, 2, 64)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    draw = lambda: torch.randint(0, 256, (2, 64), generator=g, device=DEV, dtype=torch.int32)
    x, want = draw(), draw()
    w.step(x, want, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        w.step(x, want, 1)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = w.step(x, want, 1)
    for _ in range(2):
        x.copy_(draw())
        want.copy_(draw())
        graph.replay()
        got, first = w.grad.clone(), loss.clone()
        again = w.step(x, want, 1)
        assert torch.equal(w.grad, got) and torch.equal(again, first)


def test_rounds_with_the_orthogonalised_update_repeat():
    losses = wk.train(4, block=True)
    assert all(math.isfinite(x) for x in losses)
    assert wk.train(4, block=True) == losses
    assert dblp.dblp_wait_timeouts() == 0
