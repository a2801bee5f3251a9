"""GPU: fp32 dense layers over fp32's whole range, forward and backward.

Bound per element against 64 bits: k products of fp32 operands, each of whose sums
rounds to 2^-24 of the running sum of magnitudes S, and fp32's last place 2^-149
where results are that small: (k + 8) (2^-24 S + 2^-149), as fp32 products
anywhere in the library. Both the kernels of few rows and the tiles are taken.
"""

import pytest
import torch

pytestmark = pytest.mark.gpu


def ps():
    import paper_1806_01973_amd
    return paper_1806_01973_amd


def within(got, a, b, what):
    """got = a @ b."""
    a, b = a.double(), b.double()
    k = a.shape[1]
    want = a @ b
    bound = (k + 8) * (2.0 ** -24 * (a.abs() @ b.abs()) + 2.0 ** -149)
    worst = ((got.double().cpu() - want).abs() / bound).max().item()
    assert worst <= 1.0, f"{what}: {worst:.3g} times the bound"


SCALES = [(1.0, 1.0), (1e-37, 1.0), (1.0, 1e-37), (1e-37, 1e30), (1e30, 1e-37), (1e-34, 2.0 ** 60),
          (1e37, 1e-37), (1e-20, 1e-17), (1e-37, 1e37), (1e36, 1e-2), (1e-42, 1e20)]


@pytest.mark.parametrize("sx,sw", SCALES)
@pytest.mark.parametrize("n,d_in,d_out", [(24, 64, 48), (300, 64, 96), (300, 37, 50),
                                          (40_000, 64, 136), (40_000, 75, 141)])
def test_scaled_operands(n, d_in, d_out, sx, sw):
    g = torch.Generator().manual_seed(n + d_in)
    x = (torch.randn(n, d_in, generator=g) * sx).float()
    W = (torch.randn(d_out, d_in, generator=g) / d_in * sw).float()
    dy = (torch.randn(n, d_out, generator=g) * sx).float()
    y = ps().dense_forward(x.cuda(), W.cuda())
    within(y, x, W.t().contiguous(), "y")
    # dW's sums have n products: of dy at one scale, x at the other.
    xw = (torch.randn(n, d_in, generator=g) * sw / n).float()
    dx, dW, _ = ps().dense_backward(dy.cuda(), xw.cuda(), W.cuda())
    within(dx, dy, W, "dx")
    within(dW, dy.t().contiguous(), xw, "dW")


@pytest.mark.parametrize("groups", [False, True])
def test_tiny_rows_among_ordinary_ones(groups):
    """Rows and columns at the ends of the range beside others of the same tile, whose
    bits they leave alone."""
    n, d_in, d_out = 1500, 96, 160
    g = torch.Generator().manual_seed(3)
    x, W = torch.randn(n, d_in, generator=g), torch.randn(d_out, d_in, generator=g)
    off = torch.tensor([0, 700, 700, n], dtype=torch.int64).cuda() if groups else None
    Ws = W.expand(3, -1, -1).contiguous() if groups else W
    clean = ps().dense_forward(x.cuda(), Ws.cuda(), offsets=off).cpu()
    x[5] *= 1e-38
    x[6, 3] = 1.2345 * 2.0 ** -130
    x[1400] *= 1e37
    y = ps().dense_forward(x.cuda(), Ws.cuda(), offsets=off).cpu()
    within(y, x, W.t().contiguous(), "y")
    kept = [i for i in range(n) if i not in (5, 6, 1400)]
    assert torch.equal(y[kept], clean[kept])
    Ws = Ws.clone()
    Ws[..., 9, :] *= 1e-37
    Ws[..., 9, 0] = 2.0 ** -140
    W = Ws[0] if groups else Ws
    within(ps().dense_forward(x.cuda(), Ws.cuda(), offsets=off), x, W.t().contiguous(), "y")


@pytest.mark.parametrize("n", [40, 4000, 40_000])
def test_a_lone_product_is_rounded_once(n):
    """Diagonal weights: half a unit in the last place of each product, the parts' sums
    below 2^-31."""
    g = torch.Generator().manual_seed(n)
    diag = (1.0 + torch.rand(64, generator=g)) * 2.0 ** torch.randint(-9, 9, (64,), generator=g)
    x = torch.randn(n, 64, generator=g)
    for got in (ps().dense_forward(x.cuda(), torch.diag(diag).cuda()),
                ps().dense_backward(x.cuda(), x.cuda(), torch.diag(diag).cuda())[0]):
        want = x.double() * diag.double()
        assert ((got.double().cpu() - want).abs() / want.abs()).max() <= 2.0 ** -24 * (1 + 2.0 ** -6)
