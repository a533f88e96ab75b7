"""Which tokens are padding, which are bad, and which count; runs of a token in rows that no vector access may touch."""
import pytest
import torch

import test_gpu_operators as op
from paper_2605_01989_b200 import binding as dblp

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
ROWS = 90


def ids(n, dtype, padding):
    """Tokens in and around the table, the value of `padding` among them."""
    t = torch.randint(-2, ROWS + 3, (n,), generator=torch.Generator().manual_seed(n))
    t[::7] = padding if padding >= -2 ** 31 or dtype == torch.int64 else -1
    return t.to(dtype).to(DEV)


def counter():
    return torch.zeros(1, dtype=torch.int64, device=DEV)


PADDINGS = [None, -1, -100, ROWS, 2 ** 31 - 1, -2 ** 31, -2 ** 63, 0, ROWS - 1]


@pytest.mark.parametrize("padding", PADDINGS)
@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,width", [(5, 8), (500, 64), (500, 33), (5000, 16), (5000, 7)])
def test_only_a_row_of_the_table_is_a_padding_id(padding, dtype, n, width):
    kw = {} if padding is None else dict(padding=padding)
    p = -1 if padding is None else padding
    tokens = ids(n, dtype, p)
    inside = (tokens >= 0) & (tokens < ROWS)
    live = inside & (tokens.long() != p)                        # (an int32 tensor compares with a cut-off number)
    table, dout = op.randn((ROWS, width), F32, 1), op.randn((n, width), F32, 2)
    out, dtable, bad = torch.full((n, width), 7.0, device=DEV), torch.full((ROWS, width), 7.0, device=DEV), counter()
    dblp.dblp_embed(table, tokens, out, bad_tokens=bad, **kw)
    assert torch.equal(out, torch.where(live[:, None], table[tokens.long().clamp(0, ROWS - 1)], 0.0))
    assert int(bad) == int((~inside).sum()) > 0
    op.embed_grad(dout, tokens, ROWS, dtable, bad_tokens=bad.zero_(), **kw)
    want, tol = op.grad_and_bound(dout, tokens.long(), ROWS, 1.0, F32, padding=p)
    op.within(dtable, want, tol, "dtable")
    assert int(bad) == int((~inside).sum())


@pytest.mark.parametrize("first", [0, 31, 32, 33, 16 * 32 - 1, 16 * 32, 16 * 32 + 1, 64 * 32 + 1])
@pytest.mark.parametrize("length", [1, 32, 33, 16 * 32, 17 * 32, 33 * 32 + 5, 130 * 32])
@pytest.mark.parametrize("width,dtype", [(7, F32), (129, BF16)])
def test_embed_grad_runs_at_odd_widths(first, length, width, dtype):
    """One long run between two others, around the boundaries of tiles of 32 and of groups of 16 tiles."""
    rows = 5
    tokens = torch.cat([torch.full((c,), v, dtype=torch.int32) for v, c in ((1, first), (2, length), (4, 50))])
    tokens = tokens[torch.randperm(tokens.numel(), generator=torch.Generator().manual_seed(first + length))].to(DEV)
    dout = op.randn((tokens.numel(), width), dtype, 78)
    dtable = op.embed_grad(dout, tokens, rows, torch.full((rows, width), 5.0, dtype=dtype, device=DEV))
    want, tol = op.grad_and_bound(dout, tokens, rows, 1.0, dtype)
    op.within(dtable, want, tol, "dtable")
