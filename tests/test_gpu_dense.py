"""GPU: dense layers (forward and backward, one weight or one per group of rows)
against a plain implementation in 64 bits.

Tolerances, per element, from the arithmetic (S = the sum of the products'
magnitudes): a sum of k products in fp32 is within (k + 8) 2^-23 S; the
activation's exponential and reciprocal are within 2^-20 (1 + |u|) of its value,
and its slope is at most 1.13; a stored value is within 2^-8 of itself (bf16) or
2^-23 (fp32); dz carries that rounding into dx and dW.
"""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

ACTS = ("none", "relu", "gelu", "silu")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ROUND = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8}


def ps():
    import paper_1806_01973_amd
    return paper_1806_01973_amd


def act64(u, act):
    if act == "relu":
        return torch.relu(u)
    if act == "gelu":
        return 0.5 * u * (1 + torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3)))
    if act == "silu":
        return u / (1 + torch.exp(-u))
    return u


def slope64(u, act):
    v = u.clone().requires_grad_(True)
    with torch.enable_grad():
        act64(v, act).sum().backward()
    return v.grad if v.grad is not None else torch.ones_like(u)


def make(n, d_in, d_out, dtype, groups=0, sizes=None, seed=0):
    g = torch.Generator().manual_seed(seed)
    lead = (groups,) if groups else ()
    x = torch.randn(n, d_in, generator=g).to(DT[dtype])
    W = (torch.randn(*lead, d_out, d_in, generator=g) / math.sqrt(d_in)).to(DT[dtype])
    b = torch.randn(*lead, d_out, generator=g) * 0.1
    r = torch.randn(n, d_out, generator=g).to(DT[dtype])
    off = None
    if groups:
        off = torch.tensor([0] + list(torch.tensor(sizes).cumsum(0)), dtype=torch.int64)
    return x, W, b, r, off


def spans(n, off):
    return [(0, n)] if off is None else list(zip(off[:-1].tolist(), off[1:].tolist()))


def pre64(x, W, b, off):
    """(u, its error bound) in 64 bits; rows of no group stay zero."""
    x, W, b = x.double(), W.double(), b.double()
    if off is None:
        W, b = W[None], b[None]
    u = torch.zeros(x.shape[0], W.shape[1], dtype=torch.float64)
    e = torch.zeros_like(u)
    for g, (lo, hi) in enumerate(spans(x.shape[0], off)):
        u[lo:hi] = x[lo:hi] @ W[g].t() + b[g]
        e[lo:hi] = (x[lo:hi].abs() @ W[g].abs().t() + b[g].abs()) * (x.shape[1] + 8) * 2.0 ** -23
    return u, e


def close(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    worst = ((got - want).abs() / bound.clamp_min(1e-300)).max().item() if got.numel() else 0.0
    assert torch.isfinite(got).all() and worst <= 1.0, f"{what}: worst error / bound {worst:.3g}"


def check_forward(x, W, b, r, off, act, dtype, y, u=None):
    want_u, e = pre64(x, W, b, off)
    if u is not None:
        close(u, want_u, e + ROUND[dtype] * want_u.abs() + 1e-30, "u")
    v = act64(want_u, act)
    live = torch.zeros(x.shape[0], 1, dtype=torch.float64)
    for lo, hi in spans(x.shape[0], off):
        live[lo:hi] = 1
    want = (v + (r.double() if r is not None else 0)) * live
    bound = 1.13 * e + 2.0 ** -20 * (1 + want_u.abs()) * v.abs() + 2.0 ** -22 * v.abs() \
        + ROUND[dtype] * want.abs() + 2.0 ** -23 * (want - v * live).abs() + 1e-30
    close(y, want, bound, "y")


SIZES = [  # n, d_in, d_out
    (1, 1, 1), (1, 1024, 2048), (3, 7, 5), (16, 64, 64), (17, 33, 129), (64, 100, 16),
    (65, 256, 512), (130, 31, 300), (1000, 512, 100), (777, 129, 65), (4596, 256, 256),
    (9000, 72, 521), (33_000, 40, 136),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d_in,d_out", SIZES)
def test_forward(n, d_in, d_out, dtype):
    act = ACTS[(n + d_out) % 4]
    x, W, b, r, _ = make(n, d_in, d_out, dtype)
    y, u = ps().dense_forward(x.cuda(), W.cuda(), b.cuda(), act, residual=r.cuda(),
                              want_preact=True)
    check_forward(x, W, b, r, None, act, dtype, y, u)
    plain = ps().dense_forward(x.cuda(), W.cuda())
    check_forward(x, W, torch.zeros(d_out), None, None, "none", dtype, plain)


GROUPS = [  # sizes, d_in, d_out, rows past the last group
    ([5], 16, 16, 0), ([0, 1, 0, 3, 0], 64, 32, 2), ([17, 0, 40, 1], 100, 77, 0),
    ([300, 0, 1, 129, 64, 0], 128, 200, 3), ([0, 0, 0], 32, 32, 4),
    ([1000, 2000, 70, 0, 5000], 96, 136, 0), ([9] * 70 + [0] * 60 + [130, 1], 48, 33, 1),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,d_in,d_out,past", GROUPS)
def test_grouped_forward(sizes, d_in, d_out, past, dtype):
    n = sum(sizes) + past
    act = ACTS[n % 4]
    x, W, b, r, off = make(n, d_in, d_out, dtype, len(sizes), sizes)
    y, u = ps().dense_forward(x.cuda(), W.cuda(), b.cuda(), act, residual=r.cuda(),
                              offsets=off.cuda(), want_preact=True)
    check_forward(x, W, b, r, off, act, dtype, y, u)
    assert not y[sum(sizes):].any() and not u[sum(sizes):].any()


def check_backward(x, W, u, dy, off, act, dtype, dx, dW, db):
    rnd = ROUND[dtype]
    u64, dy64, x64 = u.double(), dy.double(), x.double()
    dz = dy64 * slope64(u64, act)
    e = 2.0 ** -19 * (1 + u64.abs()) * dy64.abs() if act in ("gelu", "silu") else 0 * dz
    e_stored = e + rnd * dz.abs() if act != "none" else e
    W64 = W.double() if off is not None else W.double()[None]
    want_dx, b_dx = torch.zeros_like(x64), torch.zeros_like(x64)
    for g, (lo, hi) in enumerate(spans(x.shape[0], off)):
        z, zs = dz[lo:hi], e_stored[lo:hi]
        want_dx[lo:hi] = z @ W64[g]
        b_dx[lo:hi] = (zs + (W.shape[-2] + 8) * 2.0 ** -23 * z.abs()) @ W64[g].abs()
        want_dW = z.t() @ x64[lo:hi]
        b_dW = (zs + (hi - lo + 8) * 2.0 ** -23 * z.abs()).t() @ x64[lo:hi].abs()
        got = dW[g] if off is not None else dW
        close(got, want_dW, b_dW + rnd * want_dW.abs() + 1e-30, f"dW {g}")
        got = db[g] if off is not None else db
        close(got, z.sum(0), (e[lo:hi] + (hi - lo + 8) * 2.0 ** -23 * z.abs()).sum(0) + 1e-30,
              f"db {g}")
    close(dx, want_dx, b_dx + rnd * want_dx.abs() + 1e-30, "dx")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d_in,d_out", SIZES)
def test_backward(n, d_in, d_out, dtype):
    act = ACTS[(n + d_in) % 4]
    x, W, b, dy, _ = make(n, d_in, d_out, dtype, seed=1)
    u = pre64(x, W, b, None)[0].to(DT[dtype])
    got = ps().dense_backward(dy.cuda(), x.cuda(), W.cuda(), u.cuda(), act)
    check_backward(x, W, u, dy, None, act, dtype, *got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,d_in,d_out,past", GROUPS)
def test_grouped_backward(sizes, d_in, d_out, past, dtype):
    n = sum(sizes) + past
    act = ACTS[(n + 1) % 4]
    x, W, b, dy, off = make(n, d_in, d_out, dtype, len(sizes), sizes, seed=2)
    u = pre64(x, W, b, off)[0].to(DT[dtype])
    got = ps().dense_backward(dy.cuda(), x.cuda(), W.cuda(), u.cuda(), act, offsets=off.cuda())
    check_backward(x, W, u, dy, off, act, dtype, *got)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_activation_both_ways(act, dtype):
    x, W, b, r, _ = make(70, 48, 90, dtype, seed=3)
    x[0] *= 40  # far out on both sides
    y, u = ps().dense_forward(x.cuda(), W.cuda(), b.cuda(), act, want_preact=True)
    check_forward(x, W, b, None, None, act, dtype, y, u)
    got = ps().dense_backward(r.cuda(), x.cuda(), W.cuda(), u, act)
    check_backward(x, W, u.cpu(), r, None, act, dtype, *got)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("groups", [0, 3])
def test_gradients_against_differences(act, groups):
    """Directional differences of the forward pass itself. L = sum(y dy); with
    a step h the central difference is off by h^2 / 6 times the third
    derivative, and by the rounding of y, 2^-23 sum(|y dy|) / h: h = 2^-6 and
    sums of a few thousand terms leave 1e-2 of the derivative's scale."""
    sizes = [40, 0, 33]
    n, d_in, d_out = 73, 24, 37
    x, W, b, dy, off = make(n, d_in, d_out, "f32", groups, sizes, seed=4)
    if act == "relu":
        W, b = W * 1.0, b + 0.0
        u0, _ = pre64(x, W, b, off)
        dy[(u0.abs() < 0.2)] = 0  # no kink within a step's reach
    dev = [t.cuda() for t in (x, W, b)]
    o = off.cuda() if off is not None else None
    u = ps().dense_forward(*dev, act, offsets=o, want_preact=True)[1]
    grads = ps().dense_backward(dy.cuda(), dev[0], dev[1], u, act, offsets=o)
    h = 2.0 ** -6
    for i, g in enumerate(grads):
        v = torch.randn(dev[i].shape, generator=torch.Generator().manual_seed(i))
        v = (v / v.norm()).cuda()
        ends = []
        for s in (1, -1):
            p = list(dev)
            p[i] = p[i] + s * h * v
            ends.append((ps().dense_forward(*p, act, offsets=o).double() * dy.cuda()).sum())
        want = ((ends[0] - ends[1]) / (2 * h)).item()
        got = (g.double() * v).sum().item()
        assert abs(got - want) <= 1e-2 * (abs(want) + g.double().norm().item() / math.sqrt(v.numel())), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [9, 300, 40_000])
def test_strides_and_offsets_of_rows(n, dtype):
    """Column slices of wider matrices, from odd columns on."""
    d_in, d_out = 50, 70
    x, W, b, r, _ = make(n, d_in, d_out, dtype, seed=5)

    def inside(t, before, after):
        wide = torch.full((t.shape[0], before + t.shape[1] + after), 7.0, dtype=t.dtype,
                          device="cuda")
        wide[:, before:before + t.shape[1]] = t.cuda()
        return wide, wide[:, before:before + t.shape[1]]

    xs, Ws, rs = inside(x, 3, 2)[1], inside(W, 1, 6)[1], inside(r, 5, 0)[1]
    wide, ys = inside(torch.zeros(n, d_out, dtype=DT[dtype]), 1, 3)
    out = ps().dense_forward(xs, Ws, b.cuda(), "gelu", residual=rs, out=ys)
    assert out is ys and (wide[:, :1] == 7).all() and (wide[:, -3:] == 7).all()
    check_forward(x, W, b, r, None, "gelu", dtype, ys)
    u = pre64(x, W, b, None)[0].to(DT[dtype])
    got = ps().dense_backward(rs, xs, Ws, inside(u, 3, 3)[1], "gelu")
    check_backward(x, W, u, r, None, "gelu", dtype, *got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d_in,d_out", [
    (40, 7, 3), (200, 3, 67), (200, 67, 5), (150, 131, 71), (150, 9, 129), (700, 15, 15),
    (300, 64, 65), (300, 65, 64), (9000, 301, 131), (9000, 131, 301), (20_000, 257, 259)])
def test_nothing_around_the_operands_is_used(n, d_in, d_out, dtype):
    """Rows that end inside a 16-byte vector, at odd addresses, with NaN before and
    behind every row and around the whole operand."""
    x, W, b, dy, _ = make(n, d_in, d_out, dtype, seed=12)

    def among_nan(t):
        wide = torch.full((t.shape[0] + 2, t.shape[1] + 9), math.nan, dtype=t.dtype, device="cuda")
        view = wide[1:-1, 3:3 + t.shape[1]]
        view.copy_(t)
        return view

    xs, Ws, dys = among_nan(x), among_nan(W), among_nan(dy)
    out = ps().dense_forward(xs, Ws, b.cuda(), "silu", residual=dys)
    check_forward(x, W, b, dy, None, "silu", dtype, out)
    u = pre64(x, W, b, None)[0].to(DT[dtype])
    got = ps().dense_backward(dys, xs, Ws, among_nan(u), "silu")
    check_backward(x, W, u, dy, None, "silu", dtype, *got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,d_in,d_out", [
    ([150, 0, 3, 700], 37, 69), ([64, 65, 1, 2000], 130, 5), ([3000, 0, 2500], 75, 141)])
def test_grouped_layers_of_odd_widths(sizes, d_in, d_out, dtype):
    n = sum(sizes)
    x, W, b, dy, off = make(n, d_in, d_out, dtype, len(sizes), sizes, seed=13)
    y = ps().dense_forward(x.cuda(), W.cuda(), b.cuda(), "gelu", offsets=off.cuda())
    check_forward(x, W, b, None, off, "gelu", dtype, y)
    u = pre64(x, W, b, off)[0].to(DT[dtype])
    got = ps().dense_backward(dy.cuda(), x.cuda(), W.cuda(), u.cuda(), "gelu", offsets=off.cuda())
    check_backward(x, W, u, dy, off, "gelu", dtype, *got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_residual_in_place(dtype):
    x, W, b, r, _ = make(500, 64, 96, dtype, seed=6)
    y = r.cuda()
    ps().dense_forward(x.cuda(), W.cuda(), b.cuda(), "silu", residual=y, out=y)
    check_forward(x, W, b, r, None, "silu", dtype, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [20, 400])
def test_infinities_and_nan_stay_in_their_rows(n, dtype):
    x, W, b, _, _ = make(n, 200, 150, dtype, seed=7)
    clean = ps().dense_forward(x.cuda(), W.cuda(), b.cuda())
    x[3, 5], x[7, 199], x[11, 0], x[n - 1, 17] = math.inf, -math.inf, math.nan, 3.3e38
    W[9, 17] = 0.0
    y = ps().dense_forward(x.cuda(), W.cuda(), b.cuda()).cpu()
    want = x.double() @ W.double().t() + b.double()
    for row in (3, 7):
        inf = torch.isinf(want[row])
        assert torch.equal(torch.isinf(y[row]), inf) and inf.any()
        assert torch.equal(torch.sign(y[row][inf]).double(), torch.sign(want[row][inf]))
    assert torch.isnan(y[11]).all()
    assert abs(y[n - 1, 9].double() - want[n - 1, 9]) <= 1e-2 * (1 + abs(want[n - 1, 9]))
    kept = [i for i in range(n) if i not in (3, 7, 11, n - 1)]
    cols = [c for c in range(150) if c != 9]
    assert torch.equal(y[kept][:, cols], clean.cpu()[kept][:, cols])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_of_a_group_stays_in_it(dtype):
    sizes = [100, 0, 30, 200]
    x, W, b, dy, off = make(330, 80, 60, dtype, 4, sizes, seed=8)
    x[100:130] = math.nan
    dy[100:130] = math.inf
    u = torch.ones(330, 60, dtype=DT[dtype])
    y = ps().dense_forward(x.cuda(), W.cuda(), b.cuda(), offsets=off.cuda())
    assert torch.isnan(y[100:130]).all()
    assert torch.isfinite(y[:100]).all() and torch.isfinite(y[130:]).all()
    dx, dW, db = ps().dense_backward(dy.cuda(), x.cuda(), W.cuda(), u.cuda(), "silu",
                                     offsets=off.cuda())
    for t in (dW, db):
        assert torch.isfinite(t[0]).all() and torch.isfinite(t[3]).all() and not t[1].any()
    assert torch.isfinite(dx[:100]).all() and torch.isfinite(dx[130:]).all()


def test_wide_range_fp32():
    """Rows and columns of very different scale keep fp32's relative accuracy."""
    x, W, b, _, _ = make(300, 96, 140, "f32", seed=9)
    x *= torch.logspace(-12, 12, 300)[:, None]
    W *= torch.logspace(8, -8, 140)[:, None]
    b *= 0
    y = ps().dense_forward(x.cuda(), W.cuda(), b.cuda())
    check_forward(x, W, b, None, None, "none", "f32", y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_of_the_gradient_alone(dtype):
    x, W, b, dy, _ = make(600, 64, 48, dtype, seed=10)
    u = pre64(x, W, b, None)[0].to(DT[dtype])
    args = [t.cuda() for t in (dy, x, W, u)]
    full = ps().dense_backward(*args, "gelu")
    for i in range(3):
        need = [j == i for j in range(3)]
        got = ps().dense_backward(*args, "gelu", None, *need)
        assert [g is not None for g in got] == need
        assert torch.equal(got[i], full[i])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows(dtype):
    x, W, b, _, _ = make(0, 32, 48, dtype)
    assert ps().dense_forward(x.cuda(), W.cuda(), b.cuda()).shape == (0, 48)
    dx, dW, db = ps().dense_backward(torch.zeros(0, 48, dtype=DT[dtype]).cuda(), x.cuda(),
                                     W.cuda(), torch.zeros(0, 48, dtype=DT[dtype]).cuda(), "relu")
    assert dx.shape == (0, 32) and not dW.any() and not db.any()
    off = torch.zeros(4, dtype=torch.int64).cuda()
    W3 = W.expand(3, 48, 32).contiguous().cuda()
    dx, dW, db = ps().dense_backward(torch.zeros(0, 48, dtype=DT[dtype]).cuda(), x.cuda(), W3,
                                     offsets=off)
    assert dW.shape == (3, 48, 32) and not dW.any() and not db.any()


def test_offsets_out_of_order_touch_nothing_outside():
    """Malformed offsets are clamped: results are unspecified, accesses are not."""
    x, W, b, _, _ = make(200, 32, 48, "bf16", 3, [1, 1, 1])
    guard = torch.full((202, 48), 7.0, dtype=torch.bfloat16, device="cuda")
    for off in ([0, 500, -3, 200], [-(2 ** 40), 2 ** 40, 2 ** 62, 5], [200, 150, 100, 0]):
        o = torch.tensor(off, dtype=torch.int64).cuda()
        ps().dense_forward(x.cuda(), W.cuda(), b.cuda(), offsets=o, out=guard[1:201])
        ps().dense_backward(guard[1:201], x.cuda(), W.cuda(), offsets=o)
        torch.cuda.synchronize()
        assert (guard[0] == 7).all() and (guard[201] == 7).all()


def test_overlapping_groups_keep_to_the_workspace():
    """Offsets that give every other group all rows count far more partial sums than the
    workspace holds; the bytes after it stay."""
    n, groups = 6000, 40
    x, W, b, _, _ = make(n, 64, 48, "bf16", groups, [0] * groups)
    off = torch.tensor([0, n] * (groups // 2) + [n], dtype=torch.int64).cuda()
    dy = torch.ones(n, 48, dtype=torch.bfloat16, device="cuda")
    need = ps().dense_backward_workspace_size(W.cuda(), n, "none", off)
    whole = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    ps().dense_backward(dy, x.cuda(), W.cuda(), offsets=off, workspace=whole[:need])
    torch.cuda.synchronize()
    assert (whole[need:] == 77).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_again_and_on_another_stream(dtype):
    sizes = [700, 0, 1300, 90]
    x, W, b, dy, off = make(2090, 128, 160, dtype, 4, sizes, seed=11)
    dev = [t.cuda() for t in (x, W, b, dy, off)]

    def all_of_it():
        y, u = ps().dense_forward(dev[0], dev[1], dev[2], "gelu", offsets=dev[4], want_preact=True)
        return (y, u) + ps().dense_backward(dev[3], dev[0], dev[1], u, "gelu", offsets=dev[4])

    first = all_of_it()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = all_of_it()
    s.synchronize()
    for p, q in zip(first, second):
        assert torch.equal(p, q)


def test_captured_in_a_graph():
    x, W, b, dy, _ = make(3000, 96, 128, "bf16", seed=12)
    dev = [t.cuda() for t in (x, W, b, dy)]
    y = torch.empty(3000, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(ps().dense_backward_workspace_size(dev[1], 3000, "silu"), dtype=torch.uint8,
                     device="cuda")
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        ps().dense_forward(dev[0], dev[1], dev[2], "silu", out=y)
    s.synchronize()
    with torch.cuda.graph(graph, stream=s):
        _, u = ps().dense_forward(dev[0], dev[1], dev[2], "silu", out=y, want_preact=True)
        grads = ps().dense_backward(dev[3], dev[0], dev[1], u, "silu", workspace=ws)
    for k in range(3):
        dev[0].copy_((x * (k + 1)).cuda())
        graph.replay()
        torch.cuda.synchronize()
        want_y, want_u = ps().dense_forward(dev[0], dev[1], dev[2], "silu", want_preact=True)
        want = ps().dense_backward(dev[3], dev[0], dev[1], want_u, "silu")
        assert torch.equal(y, want_y) and torch.equal(u, want_u)
        for p, q in zip(grads, want):
            assert torch.equal(p, q)


@pytest.mark.parametrize("dtype,d_in", [("bf16", 2048), ("bf16", 2047), ("f32", 2048)])
def test_rows_past_32_bits_of_elements(dtype, d_in):
    """1.1M rows of 2,048: element offsets pass 2^31 (and bytes 2^32). Only the last rows
    are not zero, so the sums are theirs."""
    n, d_out, last = 1_100_000, 24, 300
    _, W, b, _, _ = make(1, d_in, d_out, dtype, seed=13)
    tail, _, _, dy, _ = make(last, d_in, d_out, dtype, seed=14)
    x = torch.zeros(n, d_in, dtype=DT[dtype], device="cuda")
    x[-last:] = tail.cuda()
    y, u = ps().dense_forward(x, W.cuda(), b.cuda(), "silu", want_preact=True)
    check_forward(tail, W, b, None, None, "silu", dtype, y[-last:], u[-last:])
    assert (u[:-last] == b.cuda().to(DT[dtype])).all()
    g = torch.zeros(n, d_out, dtype=DT[dtype], device="cuda")
    g[-last:] = dy.cuda()
    dx, dW, db = ps().dense_backward(g, x, W.cuda(), u, "silu")
    assert not dx[:-last].any()
    check_backward(tail, W, u[-last:].cpu(), dy, None, "silu", dtype, dx[-last:], dW, db)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[500] + [0] * 63, [0] * 63 + [500], [3000] + [1] * 40,
                                   [2100, 0, 0, 4000, 7, 1900]])
def test_groups_that_hold_nearly_all_rows(sizes, dtype):
    n = sum(sizes)
    x, W, b, dy, off = make(n, 72, 56, dtype, len(sizes), sizes, seed=15)
    y, u = ps().dense_forward(x.cuda(), W.cuda(), b.cuda(), "gelu", offsets=off.cuda(),
                              want_preact=True)
    check_forward(x, W, b, None, off, "gelu", dtype, y, u)
    got = ps().dense_backward(dy.cuda(), x.cuda(), W.cuda(), u, "gelu", offsets=off.cuda())
    check_backward(x, W, u.cpu(), dy, off, "gelu", dtype, *got)


def test_refusals():
    P = ps()
    x, W, b, r, off = make(10, 32, 48, "bf16", 2, [4, 6])
    x, W, b, r, off = (t.cuda() for t in (x, W, b, r, off))
    bad = [
        lambda: P.dense_forward(x, W, b, "tanh", offsets=off),
        lambda: P.dense_forward(x, W, b),                       # groups without offsets
        lambda: P.dense_forward(x, W[0], b[0], offsets=off),
        lambda: P.dense_forward(x.float(), W, b, offsets=off),
        lambda: P.dense_forward(x, W, b.bfloat16(), offsets=off),
        lambda: P.dense_forward(x, W, b, offsets=off.int()),
        lambda: P.dense_forward(x, W, b[:1], offsets=off),
        lambda: P.dense_forward(x[:, :31], W, b, offsets=off),
        lambda: P.dense_forward(x.t().contiguous().t(), W, b, offsets=off),
        lambda: P.dense_forward(x, W, b, offsets=off, residual=r[:9]),
        lambda: P.dense_forward(x, W, b, offsets=off, out=r.float()),
        lambda: P.dense_forward(x.cpu(), W, b, offsets=off),
        lambda: P.dense_backward(r, x, W, None, "relu", offsets=off),
        lambda: P.dense_backward(r, x, W, r[:, :47], "relu", offsets=off),
        lambda: P.dense_backward(r[:1].expand(10, 48), x[:, :1].expand(10, 32), W, offsets=off),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(P.PinsageError):
        P.dense_backward(r, x, W, offsets=off, workspace=torch.empty(16, dtype=torch.uint8,
                                                                     device="cuda"))
