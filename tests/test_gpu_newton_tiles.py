"""GPU: every kernel that Newton-Schulz chooses from, against 64 bits, and that the
sizes here still reach it (by the names of the kernels that ran).

The error is held against that of the same formula in 32 bits, rounded once: twice
it in fp32 (values are kept to 2^-23, sums run in fp32 as its own), 1.1 times in bf16.
"""

import pytest
import torch

from test_gpu_dense_tiles import names_of

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TIMES = {"f32": 2.0, "bf16": 1.1}


def newton(g, dtype):
    flip = g.shape[0] > g.shape[1]
    X = (g.t() if flip else g).to(dtype).contiguous()
    X = X / (X.norm() + 1e-7)
    for _ in range(5):
        S = torch.mm(X, X.t().contiguous())
        X = 3.4445 * X + torch.mm(-4.7750 * S + 2.0315 * torch.mm(S, S), X)
    return X.t() if flip else X


def ring(kind, side, k, stages):
    return f"RingCfg<2, {side}, {side}, {k}, 2, 2, {kind}, {kind}, {stages},"


GRAM, REST = "true", "false"  # operands by columns, or by rows
CASES = [  # batch, rows, cols, what has to run
    (3, 60, 300, ["newton_small_kernel"]),
    (2, 64, 400, ["newton_band_kernel<64>", ring(GRAM, 64, 64, 4)]),
    (2, 500, 120, ["newton_band_kernel<128>", ring(GRAM, 64, 64, 4)]),
    (1, 200, 330, [ring(GRAM, 64, 64, 4), ring(REST, 64, 64, 4)]),
    (1, 1410, 1400, [ring(GRAM, 64, 64, 4), ring(REST, 64, 64, 2)]),
    (1, 1900, 2048, [ring(GRAM, 64, 64, 2), ring(REST, 128, 32, 4)]),
    (8, 1000, 1100, [ring(GRAM, 128, 32, 4), ring(REST, 128, 32, 4)]),
    (5, 1100, 1000, [ring(GRAM, 128, 32, 4), ring(REST, 128, 32, 4)]),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,rows,cols,want", CASES)
def test_kernels(batch, rows, cols, want, dtype):
    import paper_1806_01973_amd as ps
    gen = torch.Generator(device="cuda").manual_seed(rows)
    g = (torch.randn(batch, rows, cols, generator=gen, device="cuda") * 1e-3).to(DT[dtype])
    out, names = names_of(lambda: ps.orthogonalize(g))
    for w in want:
        assert not names or any(w in n for n in names), (w, names)
    for i in range(batch):
        exact = newton(g[i], torch.float64)
        plain = (newton(g[i], torch.float32).to(g.dtype).double() - exact).norm()
        err = (out[i].double() - exact).norm()
        assert err <= TIMES[dtype] * plain, f"matrix {i}: {(err / plain).item():.3g} times"
