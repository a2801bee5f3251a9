"""GPU: fp32 orthogonalisation of few long rows, whose Gram matrix sums thousands of
products of one sign.

The error's mean over draws is held against the 32-bit formula's: X, A and B are kept
to 2^-23, of the size of fp32's own roundings, and sums round as fp32's do, so
sqrt(2) times it, in quadrature.
"""

import pytest
import torch

pytestmark = pytest.mark.gpu


def newton(g, dtype):
    X = g.to(dtype)
    X = X / (X.norm() + 1e-7)
    for _ in range(5):
        S = torch.mm(X, X.t().contiguous())
        X = 3.4445 * X + torch.mm(-4.7750 * S + 2.0315 * torch.mm(S, S), X)
    return X


@pytest.mark.parametrize("rows,cols", [(16, 2000), (40, 310), (50, 2000), (64, 2048), (128, 2048),
                                       (100, 1900), (200, 2000), (300, 4000), (700, 2048)])
def test_no_less_accurate_than_32_bits(rows, cols):
    import paper_1806_01973_amd as ps
    got = plain = 0.0
    for seed in range(6):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        g = torch.randn(rows, cols, generator=gen, device="cuda") * 1e-3
        want = newton(g, torch.float64)
        got += ((ps.orthogonalize(g).double() - want).norm() / want.norm()).item()
        plain += ((newton(g, torch.float32).double() - want).norm() / want.norm()).item()
    assert got <= 2 ** 0.5 * plain, f"{got / plain:.3g} times"
