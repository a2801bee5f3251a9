"""GPU: every tile that the dense layers choose from, with several chunks of k and rows
and columns that end inside a tile, against 64 bits; and that the sizes here still
reach the tiles they are here for (by the names of the kernels that ran).

Bounds per element: k roundings of 2^-23 of the sum of magnitudes, the result's own
rounding (2^-8 bf16, 2^-23 fp32); through SiLU the slope's 2^-19 (1 + |u|) and, in
bf16, dz's 2^-16.
"""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
ROUND = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8}
# mode, rows x columns x k, waves, operands by columns, stages, ...
BF16, BF16_TWO, F32 = 0, 1, 3


def ps():
    import paper_1806_01973_amd
    return paper_1806_01973_amd


def names_of(call):
    from torch.profiler import ProfilerActivity, profile
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        out = call()
        torch.cuda.synchronize()
    return out, [e.key for e in p.key_averages() if "pinsage" in e.key]


def ran(names, kernel, mode, side, k, stages=None, regs=False):
    """Whether `kernel` ran on tiles of that kind (nothing recorded: nothing to say)."""
    if not names:
        return True
    for n in names:
        if kernel not in n:
            continue
        for c in n.split("RingCfg<")[1:]:
            f = [v.strip() for v in c.split(">")[0].split(",")]
            if (int(f[0]), int(f[1]), int(f[2]), int(f[3])) == (mode, side, side, k) \
                    and (f[11] == "true") == regs and (stages is None or int(f[8]) == stages):
                return True
    return False


def make(n, d_in, d_out, dtype, sizes, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    G = len(sizes) if sizes else 1
    x = torch.randn(n, d_in, generator=g, device="cuda").to(DT[dtype])
    W = (torch.randn(G, d_out, d_in, generator=g, device="cuda") / math.sqrt(d_in)).to(DT[dtype])
    b = torch.randn(G, d_out, generator=g, device="cuda") * 0.1
    t = torch.randn(n, d_out, generator=g, device="cuda").to(DT[dtype])
    off = torch.tensor([0] + list(torch.tensor(sizes).cumsum(0)), device="cuda") if sizes else None
    ends = off.tolist() if sizes else [0, n]
    return x, W, b, t, off, list(zip(ends[:-1], ends[1:]))


def within(got, want, bound, what):
    worst = ((got.double() - want).abs() / bound).max().item()
    assert worst <= 1.0, f"{what}: {worst:.3g} times the bound"


FORWARD = [  # dtype, n, d_in, d_out, sizes, (mode, side, k, stages, regs)
    ("bf16", 300, 200, 72, None, (BF16, 64, 64, 4, False)),
    ("bf16", 4600, 328, 520, None, (BF16, 64, 64, 2, False)),
    ("bf16", 9001, 328, 520, None, (BF16, 128, 64, 2, False)),
    ("bf16", 40_003, 200, 520, None, (BF16, 256, 64, 2, False)),
    ("bf16", 40_003, 520, 520, None, (BF16, 256, 64, 2, False)),
    ("bf16", 300, 201, 73, None, (BF16, 64, 64, 2, True)),
    ("bf16", 9001, 203, 517, None, (BF16, 128, 64, 2, True)),
    ("bf16", 20_000, 328, 520, [2000, 0, 7] + [600] * 29 + [593], (BF16, 128, 64, 2, False)),
    ("bf16", 60_001, 264, 520, [30_000, 0, 5, 29_990], (BF16, 256, 64, 2, False)),
    ("bf16", 20_000, 203, 517, [9000, 0, 5, 10_990], (BF16, 128, 64, 2, True)),
    ("f32", 300, 100, 72, None, (F32, 64, 16, 4, False)),
    ("f32", 9001, 132, 520, None, (F32, 128, 16, 4, False)),
    ("f32", 9001, 133, 517, None, (F32, 64, 32, 2, True)),
    ("f32", 20_000, 132, 520, [9000, 0, 5, 10_990], (F32, 128, 16, 4, False)),
]


@pytest.mark.parametrize("dtype,n,d_in,d_out,sizes,tile", FORWARD)
def test_forward(dtype, n, d_in, d_out, sizes, tile):
    x, W, b, r, off, ends = make(n, d_in, d_out, dtype, sizes)
    (y, u), names = names_of(lambda: ps().dense_forward(
        x, W if sizes else W[0], b if sizes else b[0], residual=r, offsets=off, want_preact=True))
    mode, side, k, stages, regs = tile
    assert ran(names, "dense_rows_kernel", mode, side, k, stages, regs), names
    for g, (lo, hi) in enumerate(ends):
        xg, Wt = x[lo:hi].double(), W[g].double().t().contiguous()
        if hi == lo:
            continue
        want = xg @ Wt + b[g].double()
        e = (d_in + 8) * 2.0 ** -23 * (xg.abs() @ Wt.abs() + b[g].double().abs())
        within(u[lo:hi], want, e + ROUND[dtype] * want.abs(), f"u {g}")
        res = r[lo:hi].double()
        within(y[lo:hi], want + res, e + 2.0 ** -23 * res.abs() + ROUND[dtype] * (want + res).abs(),
               f"y {g}")
    assert not y[ends[-1][1]:].any()


def check_gradients(x, W, dy, u, ends, act, dtype, dx, dW, grouped):
    dz, slack = dy.double(), torch.zeros_like(dy, dtype=torch.float64)
    if act == "silu":
        p = torch.sigmoid(u.double())
        dz = dz * p * (1 + u.double() * (1 - p))
        slack = 2.0 ** -19 * (1 + u.double().abs()) * dy.double().abs()
        if dtype == "bf16":
            slack = slack + 2.0 ** -16 * dz.abs()
    for g, (lo, hi) in enumerate(ends):
        if hi == lo:
            continue
        z, e, Wg, xg = dz[lo:hi], slack[lo:hi], W[g].double(), x[lo:hi].double()
        if dx is not None:
            want = z @ Wg
            bound = ((z.shape[1] + 8) * 2.0 ** -23 * z.abs() + e) @ Wg.abs()
            within(dx[lo:hi], want, bound + ROUND[dtype] * want.abs() + 1e-30, f"dx {g}")
        if dW is not None:
            zt, et = z.t().contiguous(), e.t().contiguous()
            want = zt @ xg
            bound = ((hi - lo + 8) * 2.0 ** -23 * zt.abs() + et) @ xg.abs()
            within(dW[g] if grouped else dW, want, bound + ROUND[dtype] * want.abs() + 1e-30,
                   f"dW {g}")
    if dx is not None:
        assert not dx[ends[-1][1]:].any()


def backward(dtype, act, n, d_in, d_out, sizes, need):
    x, W, _, dy, off, ends = make(n, d_in, d_out, dtype, sizes, seed=1)
    u = torch.randn(n, d_out, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    u = u.to(DT[dtype])
    (dx, dW, _), names = names_of(lambda: ps().dense_backward(
        dy, x, W if sizes else W[0], u, act, offsets=off, need_dx=need[0], need_dW=need[1]))
    check_gradients(x, W, dy, u, ends, act, dtype, dx, dW, bool(sizes))
    return names


# One part, two parts, fp32.
KINDS = [("bf16", "none", BF16), ("bf16", "silu", BF16_TWO), ("f32", "silu", F32)]
K_OF = {BF16: {64: 64, 128: 64, 256: 64}, BF16_TWO: {64: 64, 128: 32, 256: 32}, F32: {64: 16, 128: 16}}


DX = [  # n, d_in, d_out, sizes, side, regs
    (300, 72, 200, None, 64, False), (4600, 520, 328, None, 64, False),
    (9001, 520, 328, None, 128, False), (40_003, 520, 328, None, 256, False),
    (300, 73, 201, None, 64, True), (9001, 517, 203, None, 128, True),
    (20_000, 520, 328, [2000, 0, 7] + [600] * 29 + [593], 128, False),
    (60_001, 520, 264, [30_000, 0, 5, 29_990], 256, False),
]


@pytest.mark.parametrize("dtype,act,mode", KINDS)
@pytest.mark.parametrize("n,d_in,d_out,sizes,side,regs", DX)
def test_dx(n, d_in, d_out, sizes, side, regs, dtype, act, mode):
    names = backward(dtype, act, n, d_in, d_out, sizes, (True, False))
    if mode == F32:
        side, k = (64, 32) if regs else (min(side, 128), 16)
    else:
        k = K_OF[mode][side]
    assert ran(names, "dense_rows_kernel", mode, side, k, None, regs), names


DW = [  # n, d_in, d_out, sizes, side, regs
    (1000, 72, 200, None, 64, False), (5000, 520, 520, None, 64, False),
    (9001, 520, 520, None, 128, False), (44_001, 520, 520, None, 256, False),
    (1000, 73, 201, None, 64, True), (9001, 517, 519, None, 128, True),
    (20_000, 264, 520, [9000, 0, 5, 700, 10_295], 128, False),
    (60_001, 520, 520, [30_000, 0, 5, 29_990], 256, False),
]


@pytest.mark.parametrize("dtype,act,mode", KINDS)
@pytest.mark.parametrize("n,d_in,d_out,sizes,side,regs", DW)
def test_dw(n, d_in, d_out, sizes, side, regs, dtype, act, mode):
    names = backward(dtype, act, n, d_in, d_out, sizes, (False, True))
    if mode == F32:
        side, k = (64, 32) if regs else (min(side, 128), 16)
    else:
        k = K_OF[mode][side]
    assert ran(names, "dense_dw_kernel", mode, side, k, None, regs), names


TOGETHER = [  # n, d_in, d_out, dx's side, dW's side
    (300, 72, 200, 64, 64), (4596, 264, 520, 64, 64), (8300, 72, 2048, 64, 128),
    (9001, 520, 40, 128, 64), (9001, 520, 520, 128, 128),
]


@pytest.mark.parametrize("dtype,act,mode", KINDS)
@pytest.mark.parametrize("n,d_in,d_out,side_x,side_w", TOGETHER)
def test_both_in_one_launch(n, d_in, d_out, side_x, side_w, dtype, act, mode):
    names = backward(dtype, act, n, d_in, d_out, None, (True, True))
    for side in (side_x, side_w):
        assert ran(names, "dense_grads_kernel", mode, side, K_OF[mode][side]), names


@pytest.mark.parametrize("dtype,act,mode", KINDS)
def test_both_in_one_launch_by_groups(dtype, act, mode):
    names = backward(dtype, act, 12_000, 520, 264, [5000, 0, 5, 700, 6290], (True, True))
    assert not names or any("dense_grads_kernel" in n for n in names), names
