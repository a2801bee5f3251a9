"""GPU: fp32 layers whose operands are not finite cost little more than others.

Elements that are not finite are formed again with fp32 matrix instructions: twice
the time of the split products' instructions and once more for loads that nothing
hides, so four times a clean call's time in all.
"""

import pytest
import torch

pytestmark = pytest.mark.gpu


def ps():
    import paper_1806_01973_amd
    return paper_1806_01973_amd


def best_us(call):
    call()
    times = []
    for _ in range(7):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    return min(times)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("n,d_in,d_out", [(4096, 512, 512), (20_000, 256, 512), (20_000, 255, 511)])
def test_not_finite_calls_are_not_slow(n, d_in, d_out, bad):
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(n, d_in, generator=g, device="cuda")
    W = torch.randn(d_out, d_in, generator=g, device="cuda")
    dy = torch.randn(n, d_out, generator=g, device="cuda")
    clean = best_us(lambda: ps().dense_forward(x, W))
    clean_back = best_us(lambda: ps().dense_backward(dy, x, W))
    x[n // 2], dy[n // 2] = bad, bad
    W[3] = bad
    forward = best_us(lambda: ps().dense_forward(x, W))
    back = best_us(lambda: ps().dense_backward(dy, x, W))
    assert not torch.isfinite(ps().dense_forward(x, W)[:, 3]).any()
    assert forward <= 4 * clean, f"{forward:.0f} us against {clean:.0f}"
    assert back <= 4 * clean_back, f"{back:.0f} us against {clean_back:.0f}"
