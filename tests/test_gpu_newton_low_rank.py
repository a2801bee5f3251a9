"""GPU: orthogonalising matrices near low rank (a weight's gradient from fewer rows
than its width) and of strongly graded spectrum.

Five steps enlarge small singular directions about 480 times, and with them what
the storage of X, A and B rounds off. The reference is the definition in 64 bits;
the yardstick is the same formula in 32 bits, whose roundings are enlarged alike.
The kernels' stored values round to 2^-23 at most (fp32: 2^-24) and their sums
run in fp32 as well, so their error is at most twice the 32-bit form's; in bf16
the result's own rounding (1.6e-3) hides both, and 1.1 times is asked.
"""

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TIMES = {"f32": 2.0, "bf16": 1.1}
A, B, C = 3.4445, -4.7750, 2.0315


def ps():
    import paper_1806_01973_amd
    return paper_1806_01973_amd


def newton(g, dtype):
    flip = g.shape[0] > g.shape[1]
    X = (g.t() if flip else g).to(dtype).contiguous()
    X = X / (X.norm() + 1e-7)
    for _ in range(5):
        S = X @ X.t()
        X = A * X + (B * S + C * (S @ S)) @ X
    return X.t() if flip else X


def matrix(rows, cols, rank, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    if rank == "graded":  # singular values from 1 down to 1e-4
        k = min(rows, cols)
        u = torch.linalg.qr(torch.randn(rows, k, generator=gen, dtype=torch.float64))[0]
        v = torch.linalg.qr(torch.randn(cols, k, generator=gen, dtype=torch.float64))[0]
        g = (u * torch.logspace(0, -4, k, dtype=torch.float64)) @ v.t()
    else:
        g = torch.randn(rows, rank, generator=gen) @ torch.randn(rank, cols, generator=gen)
    return (g * 1e-3).to(DT[dtype])


def error(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rank", [1, 4, 16, "graded"])
@pytest.mark.parametrize("rows,cols", [(48, 200), (100, 300), (130, 600), (256, 512), (512, 300)])
def test_low_rank(rows, cols, rank, dtype):
    g = matrix(rows, cols, rank, dtype, rows + cols)
    want = newton(g, torch.float64)
    plain = error(newton(g, torch.float32).to(g.dtype), want)
    got = error(ps().orthogonalize(g.cuda()), want)
    assert got <= TIMES[dtype] * plain, f"{got:.3g} against the 32-bit form's {plain:.3g}"


@pytest.mark.parametrize("rank", [1, 16])
def test_optimiser_step_of_a_low_rank_gradient(rank):
    """bf16 weights: W' = W - lr O, O's rows through the difference of the two."""
    g = matrix(200, 320, rank, "bf16", 7)
    W = torch.zeros(200, 320, dtype=torch.bfloat16)
    m = torch.zeros(200, 320)
    want = -newton(g.double() * 1.95, torch.float64)
    got, _ = ps().muon_step(W.cuda(), g.cuda(), m.cuda(), lr=1.0, scale=1.0)
    plain = error(-newton(g.float() * 1.95, torch.float32).bfloat16(), want)
    assert error(got, want) <= TIMES["bf16"] * plain
