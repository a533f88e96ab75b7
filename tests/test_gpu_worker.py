"""The worker's step: its gradient against 64-bit automatic differentiation of the same model with the same masks, and rounds of
it through the lossy transport."""
import math

import pytest
import torch

from paper_2605_01989_b200 import binding as dblp
from paper_2605_01989_b200 import worker as wk

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def mask(n, d, p, seed, step, site):
    """What dropout does to ones: 0, or the scale of what is kept."""
    out = torch.empty((n, d), device=DEV)
    dblp.dblp_dropout(torch.ones((n, d), device=DEV), out, p, seed, step, site)
    return out.double()


@pytest.mark.parametrize("batch,tokens,heads,head_dim", [(2, 150, 2, 64), (1, 40, 3, 128)])
def test_the_gradient_is_that_of_the_model(batch, tokens, heads, head_dim):
    torch.cuda.set_device(0)
    rows, step, p = 300, 5, 0.1
    model = wk.TokenModel(rows, heads, head_dim, DEV, seed=3)
    w = wk.Worker(model, batch, tokens, p=p, seed=9)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    x, want = (torch.randint(0, rows, (batch, tokens), generator=g, device=DEV, dtype=torch.int32) for _ in range(2))
    loss = w.step(x, want, step)

    d, n = model.width, batch * tokens
    table, w_qkv, w_out = params = [t.detach().double().requires_grad_() for t in model.views(model.flat)]
    x0 = table[x.reshape(-1).long()] * math.sqrt(d) * mask(n, d, p, 9, step, wk.EMBED_SITE)
    q, k, v = (x0 @ w_qkv).view(batch, tokens, 3, heads, head_dim).permute(2, 0, 3, 1, 4)
    s = (q @ k.transpose(2, 3)) / math.sqrt(head_dim)
    s = s.masked_fill(torch.ones((tokens, tokens), dtype=torch.bool, device=DEV).triu(1), -math.inf)
    att = (s.softmax(3) @ v).transpose(1, 2).reshape(n, d)
    x1 = x0 + (att @ w_out) * mask(n, d, p, 9, step, wk.RESIDUAL_SITE)
    exact = torch.nn.functional.cross_entropy(x1 @ table.t(), want.reshape(-1).long())
    exact.backward()

    assert abs(loss.item() - exact.item()) < 2.0 ** -8 * abs(exact.item())
    # A gradient passes at most about 14 roundings to bf16 of random sign, each 2^-8 at most and 2^-9.8 on average: their
    # root sum of squares is below 1 %; three times that
    for got, param, name in zip(model.views(w.grad), params, ("table", "qkv", "out")):
        rel = ((got.double() - param.grad).norm() / param.grad.norm()).item()
        assert rel < 0.03, (name, rel)


def test_rounds_over_a_lossy_transport_learn():
    losses = wk.train(60)
    assert losses[0] > 5.5 and losses[-1] < 0.6 * losses[0]
    assert wk.train(3) == losses[:3]                   # every step of it repeats bit for bit
    assert dblp.dblp_wait_timeouts() == 0
