"""A decoder block's update against its formula in 64 bits, tensor by tensor: momentum of the mean; matrices move by the momentum with its
singular values near 1, times sqrt(max(1, rows / columns)), the rest by the momentum."""
import math

import pytest
import torch

from paper_2605_01989_b200 import binding as dblp
from paper_2605_01989_b200 import worker as wk

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def iteration(x):
    x = x / (x.norm() + 1e-7)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    for a, b, c in dblp.MUON_COEFFICIENTS:
        A = x @ x.T
        x = a * x + (b * A + c * A @ A) @ x
    return x.T if tall else x


@pytest.mark.parametrize("heads,head_dim,lr,mu", [(2, 64, 0.5, 0.9), (3, 40, 0.1, 0.5)])
def test_an_update_moves_every_tensor_as_the_formula_does(heads, head_dim, lr, mu):
    torch.cuda.set_device(0)
    model = wk.BlockModel(200, heads, head_dim, DEV, seed=2)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    momentum = torch.zeros_like(model.flat, dtype=torch.float64)
    for _ in range(3):
        mean = torch.randn(model.flat.shape, generator=g, device=DEV) * 1e-2
        before = model.flat.clone()
        model.update(mean, lr, mu)
        momentum = mu * momentum + mean.double()
        moved = {n: (t.double() - u.double()) for (n, t), u in zip(model.views(model.flat).items(), model.views(before).values())}
        size = {n: t.double().norm().item() for n, t in model.views(before).items()}
        for n, m in model.views(momentum).items():
            if n in model.MATRICES:
                want = -0.02 * lr * math.sqrt(max(1.0, m.shape[0] / m.shape[1])) * iteration(m)
            else:
                want = -lr * m
            # the orthogonalised matrix in bf16: 3e-3 of its norm; the sum rounded to fp32, half a step of the parameter; momentum in fp32
            bound = (3e-3 if n in model.MATRICES else 2.0 ** -22) * want.norm().item() + 2.0 ** -24 * (size[n] + want.norm().item())
            assert (moved[n] - want).norm().item() < bound, n
    # the formula's own sign and size: a step along the gradient makes the loss of a linear function smaller
    assert sum((moved[n] * t).sum().item() for n, t in model.views(momentum).items()) < 0
