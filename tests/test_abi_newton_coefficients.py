"""Newton-Schulz coefficients whose steps leave the range of what the kernels keep are
refused on the host, for the worst matrix (one singular value anywhere in [0, 1])."""

import ctypes
import os

import numpy as np
import pytest


@pytest.fixture(scope="module")
def L():
    from paper_1806_01973_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libpinsage.so not built (run __graft_entry__.build())")
    _lib.lib()
    return _lib


def status(L, a, b, c, steps):
    p = L.NewtonSchulz(1, 100, 300, L.PINSAGE_F32, steps, a, b, c, 1e-7)
    need = ctypes.c_size_t(0)
    return L.lib().pinsage_newton_schulz_workspace_size(ctypes.byref(p), ctypes.byref(need))


def worst(a, b, c, steps):
    """The largest of what the steps keep, over a grid of first singular values."""
    x = np.linspace(0.0, 1.0, 200_001)
    most = 0.0
    with np.errstate(all="ignore"):
        for _ in range(steps):
            s = x * x
            most = max(most, s.max(), np.abs(b * s + c * s * s).max(), (np.abs(x) * s).max())
            x = np.abs(x * (a + b * s + c * s * s))
            most = max(most, x.max())
    return most


@pytest.mark.parametrize("a,b,c,steps", [
    (3.4445, -4.7750, 2.0315, 64), (1.5, -0.5, 0.0, 64), (2.0, -1.5, 0.5, 64),
    (1.875, -1.25, 0.375, 64), (0.0, 0.0, 0.0, 3), (1.0, 1.0, 1.0, 1), (1.5, 0.0, 0.0, 3)])
def test_accepted(L, a, b, c, steps):
    assert worst(a, b, c, steps) < 15.5
    assert status(L, a, b, c, steps) == 0


@pytest.mark.parametrize("a,b,c,steps", [
    (3.4445, -4.7750, 6.0, 3), (16.0, 0.0, 0.0, 1), (1.5, 0.0, 0.0, 4), (1.0, 1.0, 1.0, 2),
    (0.0, 16.0, 0.0, 1), (0.0, -70.0, 70.0, 1), (1e30, 1e30, -1e30, 64), (-20.0, 0.0, 0.0, 1)])
def test_refused(L, a, b, c, steps):
    assert not worst(a, b, c, steps) < 15.5
    assert status(L, a, b, c, steps) == L.PINSAGE_EUNSUPPORTED


def test_against_the_grid(L):
    rng = np.random.default_rng(0)
    for _ in range(300):
        a, b, c = (float(np.float32(v)) for v in rng.normal(size=3) * (2.0, 3.0, 2.0))
        steps = int(rng.integers(1, 7))
        w = worst(a, b, c, steps)
        if not w < 15.6:
            assert status(L, a, b, c, steps) == L.PINSAGE_EUNSUPPORTED, (a, b, c, steps, w)
