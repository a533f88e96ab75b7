"""How far dblp_orthogonalize's results are from the iteration in 64 bits, in parts of the result's norm, with the usual five steps.

The bounds, from the scheme's own roundings:
F32  X is held to 2^-23 of its entries.  Where the result fills the space (full rank) the error stays small; the tensor cores' runs of 192 terms of
     one sign at most take 1.2e-6 from the diagonal of A, which the polynomial multiplies by up to |b| = 4.8, 6e-6: twice that.
     Of a few directions only, what rounding leaves in the other directions grows by a = 3.4445 a step.  What is lost before step k of five
     arrives 3.4445^(5 - k) times as large, 485 + 141 + 41 + 12 + 3 = 682 together, of an X that is up to 1.2 / 0.68 times the
     result: 682 * 1.77 * 2^-23 = 1.44e-4.  (The iteration in fp32 gives 3e-5 to 1.6e-4 for the
     same matrices.)
F16  the same and the result's rounding, 2^-12.
BF16 products of one f16 word from 512 on the shorter side: roundings of random sign, 2.4e-3 at most by a 64-bit simulation with the same words,
     and the result's rounding, 1.7e-3 for values that spread over a binade; together the root of the sum of squares.  Smaller matrices,
     with both words where it shows, stay within the same bound."""
import pytest
import torch

from paper_2605_01989_b200 import binding as dblp

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
FULL = {F32: 1.2e-5, F16: 1.2e-5 + 2.0 ** -12, BF16: 3e-3}
FEW = {F32: 1.44e-4, F16: 1.44e-4 + 2.0 ** -12, BF16: 3e-3}
ALIKE = {F32: 1.2e-5, F16: 1.2e-5 + 2.0 ** -12, BF16: 3e-3}


def randn(shape, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float64)


def matrix(m, n, kind, seed):
    if kind.startswith("rank"):
        k = int(kind[4:])
        return randn((m, k), seed) @ randn((k, n), seed + 1)
    g = randn((m, n), seed)
    if kind == "strong":
        return randn((m, 3), seed + 1) @ randn((3, n), seed + 2) + 0.1 * g
    if kind == "gradient":
        return 0.5 * randn((m, 8), seed + 1) @ randn((8, n), seed + 2) + g
    if kind == "alike":
        return torch.linalg.qr(g)[0] if m >= n else torch.linalg.qr(g.T)[0].T
    return g


def iteration(x):
    x = x.double()
    x = x / (x.norm() + 1e-7)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    for a, b, c in dblp.MUON_COEFFICIENTS:
        A = x @ x.T
        x = a * x + (b * A + c * A @ A) @ x
    return x.T if tall else x


@pytest.mark.parametrize("out_dtype", [F32, F16, BF16])
@pytest.mark.parametrize("kind", ["noise", "strong", "gradient", "alike", "rank1", "rank2", "rank8"])
@pytest.mark.parametrize("m,n", [(64, 64), (129, 200), (700, 90), (384, 640), (1030, 520), (1600, 1600)])
def test_the_result_is_as_near_as_the_header_says(m, n, kind, out_dtype):
    x = (matrix(m, n, kind, m + n) * 1e-3).float().contiguous()
    out = torch.empty((m, n), dtype=out_dtype, device=DEV)
    dblp.dblp_orthogonalize(x, out, torch.empty(dblp.dblp_orthogonalize_workspace_bytes(x, out), dtype=torch.uint8, device=DEV))
    want = iteration(x)
    off = ((out.double() - want).norm() / want.norm()).item()
    bound = (FEW if kind.startswith("rank") else ALIKE if kind == "alike" else FULL)[out_dtype]
    assert off < bound, (off, bound)


@pytest.mark.parametrize("m,n", [(1, 1), (1, 50), (2, 1), (2, 3), (3, 2), (28, 2), (8, 8), (17, 40), (63, 63), (700, 33), (1, 4000)])
def test_bf16_results_of_small_matrices_are_rounded_once(m, n):
    """Element by element half a step of the result: 2^-8 of it, and what the products of both words are off by, 1.44e-4 of the norm at most."""
    for seed in range(20):
        x = randn((5, m, n), 100 + seed).float()
        out = torch.empty((5, m, n), dtype=BF16, device=DEV)
        dblp.dblp_orthogonalize(x, out, torch.empty(dblp.dblp_orthogonalize_workspace_bytes(x, out), dtype=torch.uint8, device=DEV))
        for j in range(5):
            want = iteration(x[j])
            tol = 2.0 ** -8 * want.abs() + 1.44e-4 * want.norm()
            assert ((out[j].double() - want).abs() <= tol).all(), (seed, j)


@pytest.mark.parametrize("kind", ["noise", "gradient"])
@pytest.mark.parametrize("m,n", [(129, 200), (200, 3000), (384, 640), (1030, 520), (700, 4000), (900, 4096), (1024, 2000), (1300, 4000), (6400, 1600)])
def test_fp32_results_are_as_near_as_the_iteration_in_fp32(m, n, kind):
    """Off by at most half as much again as the same iteration in plain fp32, on the same matrix."""
    x = matrix(m, n, kind, m + n).float() * 1e-2
    out = torch.empty_like(x)
    dblp.dblp_orthogonalize(x, out, torch.empty(dblp.dblp_orthogonalize_workspace_bytes(x, out), dtype=torch.uint8, device=DEV))
    want, plain = iteration(x), x / (x.norm() + 1e-7)
    plain = plain.T if m > n else plain
    assert not torch.backends.cuda.matmul.allow_tf32
    for a, b, c in dblp.MUON_COEFFICIENTS:
        A = plain @ plain.T
        plain = a * plain + (b * A + c * (A @ A)) @ plain
    plain = plain.T if m > n else plain
    off, fp32 = (((t.double() - want).norm() / want.norm()).item() for t in (out, plain))
    assert off <= 1.5 * fp32, (off, fp32)


@pytest.mark.parametrize("kind", ["noise", "gradient"])
@pytest.mark.parametrize("m,n", [(64, 64), (64, 4000), (100, 3000), (129, 200), (300, 300), (383, 900), (384, 640), (384, 4096), (511, 4096), (512, 2048), (512, 4096), (1030, 520), (1600, 1600)])
def test_bf16_results_are_near_their_own_rounding(m, n, kind):
    """Below 512 on the shorter side 1.2 times what rounding the exact result is off by (three last steps of both words), beyond 1.5 times."""
    x = matrix(m, n, kind, m + n).float() * 1e-2
    out = torch.empty((m, n), dtype=BF16, device=DEV)
    dblp.dblp_orthogonalize(x, out, torch.empty(dblp.dblp_orthogonalize_workspace_bytes(x, out), dtype=torch.uint8, device=DEV))
    want = iteration(x)
    off, rounded = ((out.double() - want).norm().item(), (want.bfloat16().double() - want).norm().item())
    assert off <= (1.2 if min(m, n) < 512 else 1.5) * rounded, off / rounded


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 7])
@pytest.mark.parametrize("m,n", [(40, 90), (200, 130), (400, 500), (600, 520)])
def test_other_numbers_of_steps(m, n, steps):
    """The workspace does not depend on the steps; which products read both words does."""
    coefficients = ((1.5, -0.5, 0.0),) * steps
    x = matrix(m, n, "noise", 7).float()
    for out_dtype in (BF16, F32):
        out = torch.empty((m, n), dtype=out_dtype, device=DEV)
        ws = torch.full((dblp.dblp_orthogonalize_workspace_bytes(x, out),), 0xAB, dtype=torch.uint8, device=DEV)
        dblp.dblp_orthogonalize(x, out, ws, coefficients=coefficients)
        want = x.double() / (x.double().norm() + 1e-7)
        for a, b, c in coefficients:
            A = want @ want.T
            want = a * want + (b * A + c * A @ A) @ want
        assert ((out.double() - want).norm() / want.norm()).item() < FULL[out_dtype]
