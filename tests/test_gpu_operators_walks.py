"""Attention and its gradient at shapes that make a block go on: several key tiles a share in the gradient (the additions to dq
and the accumulators' hand-over from tile to tile), with and without head groups, and several work items a block in the
forward pass, empty ones among them.  Statements and tolerances are those of test_gpu_operators."""
import random

import pytest
import torch

import test_gpu_operators as op
from paper_2605_01989_b200 import binding as dblp

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def mixed(B, Sq, Sk, seed):
    """Lengths of every kind: none, one, a tile's end and just beyond, all, and in between."""
    r = random.Random(seed)
    pick = lambda n: r.choice([0, 1, n, n, min(n, 128), min(n, 129), min(n, 256), r.randint(1, n)])  # noqa: E731
    return [pick(Sq) for _ in range(B)], [pick(Sk) for _ in range(B)]


GRADIENTS = [
    # B, Sq, Sk, Hq, Hkv, D, dtype, causal, lengths; how the library cuts it: key tiles a share, head groups
    (16, 500, 640, 16, 4, 64, BF16, True, True),                # 5, 2
    (16, 500, 640, 16, 4, 64, F16, False, False),               # 5, 2
    (16, 500, 640, 16, 4, 128, BF16, True, False),              # 5, 2
    (16, 500, 640, 16, 4, 128, F16, False, True),               # 5, 2
    (9, 520, 520, 20, 20, 64, BF16, True, False),               # 5, 1
    (9, 520, 520, 20, 20, 128, BF16, False, True),              # 5, 1
    (8, 700, 700, 16, 8, 64, F16, True, True),                  # 3, 1
    (20, 400, 520, 16, 8, 128, BF16, True, True),               # 5, 1
    (10, 400, 650, 30, 15, 64, BF16, False, False),             # 3, 1
    (1, 1500, 1500, 32, 4, 128, BF16, True, False),             # 3, 8
    (20, 100, 520, 32, 16, 64, BF16, True, False),              # 5, 1; two pairs a key tile: each visit follows the last but one
    (20, 100, 520, 16, 16, 128, BF16, False, False),            # 5, 1; one pair a key tile: each visit follows the last at once
]


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hkv,D,dtype,causal,lens", GRADIENTS)
def test_gradients_over_several_key_tiles_a_share(B, Sq, Sk, Hq, Hkv, D, dtype, causal, lens):
    q, k, v, g, out, dq, dk, dv = op.tensors(B, Sq, Sk, Hq, Hkv, D, dtype)
    kw = dict(causal=causal, lens=op.lengths(mixed(B, Sq, Sk, B * Sk + D) if lens else None))
    lse = op.run_attention(q, k, v, out, **kw)
    op.check_forward(q, k, v, out, lse, **kw)
    op.run_grad(q, k, v, out, g, lse, dq, dk, dv, **kw)
    op.check_grad(q, k, v, out, g, lse, dq, dk, dv, **kw)
    first = [t.clone() for t in (dq, dk, dv)]
    for _ in range(3):
        op.run_grad(q, k, v, out, g, lse, dq, dk, dv, **kw)
        for a, b in zip(first, (dq, dk, dv)):
            assert torch.equal(op.bits(a), op.bits(b))
    assert dblp.dblp_wait_timeouts() == 0


@pytest.mark.parametrize("B,Sq,Sk,Hq,Hkv,D,dtype,causal", [
    (30, 300, 500, 8, 4, 128, BF16, True), (40, 200, 333, 9, 3, 128, F16, False), (20, 260, 700, 12, 12, 64, F16, True),
    (40, 150, 400, 12, 4, 64, BF16, False), (50, 129, 200, 8, 8, 96, BF16, True)])
@pytest.mark.parametrize("lens", [False, True])
def test_forward_over_several_items_a_block(B, Sq, Sk, Hq, Hkv, D, dtype, causal, lens):
    assert B * Hq * ((Sq + 127) // 128) > 600                   # two blocks an SM hold 296
    q, k, v, g, out, *_ = op.tensors(B, Sq, Sk, Hq, Hkv, D, dtype)
    kw = dict(causal=causal, lens=op.lengths(mixed(B, Sq, Sk, B + Sq) if lens else None))
    lse = op.run_attention(q, k, v, out, **kw)
    op.check_forward(q, k, v, out, lse, **kw)
    first = out.clone(), lse.clone()
    for _ in range(3):
        lse = op.run_attention(q, k, v, out, **kw)
        assert torch.equal(op.bits(out), op.bits(first[0])) and torch.equal(op.bits(lse), op.bits(first[1]))
    assert dblp.dblp_wait_timeouts() == 0
