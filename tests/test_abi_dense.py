"""C-ABI checks of the dense layers and the orthogonalisation that need no GPU:
malformed arguments are refused on the host before any HIP call (the pointers
passed here are never dereferenced), and the workspace queries."""

import ctypes
import os

import pytest

FAKE = 0x10000


@pytest.fixture(scope="module")
def L():
    from paper_1806_01973_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libpinsage.so not built (run __graft_entry__.build())")
    _lib.lib()
    return _lib


def _dense(L, **kw):
    d = dict(d_in=64, d_out=48, num_groups=0, dtype=L.PINSAGE_BF16, activation=1, W=FAKE, ldw=64,
             b=FAKE, offsets=None)
    d.update(kw)
    return L.Dense(**d)


def _forward(L, d, x=FAKE, n=10, ldx=64, r=None, ldr=0, u=None, ldu=0, y=FAKE, ldy=48):
    return L.lib().pinsage_dense_forward(ctypes.byref(d) if d is not None else None, x, n, ldx, r,
                                         ldr, u, ldu, y, ldy, None)


def test_dense_forward_validation(L):
    inval, unsup = L.PINSAGE_EINVAL, L.PINSAGE_EUNSUPPORTED
    assert _forward(L, None) == inval
    for kw, want in ((dict(dtype=7), inval), (dict(activation=4), inval), (dict(activation=-1), inval),
                     (dict(d_in=0), inval), (dict(d_out=-3), inval), (dict(d_in=16385), unsup),
                     (dict(d_out=16385), unsup), (dict(num_groups=-1), inval),
                     (dict(num_groups=4097, offsets=FAKE), unsup), (dict(num_groups=2), inval),
                     (dict(offsets=FAKE), inval), (dict(W=None), inval), (dict(ldw=63), inval),
                     (dict(ldw=(1 << 20) + 1), unsup)):
        assert _forward(L, _dense(L, **kw)) == want, kw
        assert L.lib().pinsage_last_error()
    for kw, want in ((dict(x=None), inval), (dict(y=None), inval), (dict(n=-1), inval),
                     (dict(n=1 << 31), unsup), (dict(ldx=63), inval), (dict(ldy=47), inval),
                     (dict(r=FAKE, ldr=47), inval), (dict(u=FAKE, ldu=47), inval),
                     (dict(ldx=1 << 21), unsup)):
        assert _forward(L, _dense(L), **kw) == want, kw
    big = _dense(L, d_out=16384)
    assert _forward(L, big, n=(1 << 31) - 1, ldy=16384) == unsup  # more tiles than a launch has
    assert _forward(L, _dense(L), x=None, n=0) == L.PINSAGE_OK


def test_dense_backward_validation(L):
    lib = L.lib()
    need = ctypes.c_size_t(0)

    def call(d, dy=FAKE, lddy=48, x=FAKE, ldx=64, u=FAKE, ldu=48, n=1000, dx=FAKE, lddx=64, dW=FAKE,
             db=FAKE, ws=FAKE, wsb=None):
        return lib.pinsage_dense_backward(ctypes.byref(d), dy, lddy, x, ldx, u, ldu, n, dx, lddx, dW,
                                          db, ws, need.value if wsb is None else wsb, None)

    d = _dense(L)
    assert lib.pinsage_dense_backward_workspace_size(ctypes.byref(d), 1000, None) == L.PINSAGE_EINVAL
    assert lib.pinsage_dense_backward_workspace_size(ctypes.byref(d), -1, ctypes.byref(need)) == \
        L.PINSAGE_EINVAL
    assert lib.pinsage_dense_backward_workspace_size(ctypes.byref(d), 1000, ctypes.byref(need)) == 0
    assert need.value >= 1000 * 48 * 2  # dz
    for kw in (dict(dy=None), dict(x=None), dict(u=None), dict(lddy=47), dict(ldx=63), dict(ldu=47),
               dict(lddx=63), dict(n=-1)):
        assert call(d, **kw) == L.PINSAGE_EINVAL, kw
    assert call(_dense(L, W=None)) == L.PINSAGE_EINVAL
    assert call(d, wsb=need.value - 1) == L.PINSAGE_EWORKSPACE
    assert call(d, ws=None) == L.PINSAGE_EWORKSPACE
    assert call(d, ws=FAKE + 8) == L.PINSAGE_EINVAL
    none = _dense(L, activation=0)
    assert lib.pinsage_dense_backward_workspace_size(ctypes.byref(none), 1000,
                                                     ctypes.byref(need)) == 0
    assert need.value < 1000 * 48 * 2  # no dz without an activation


def test_newton_schulz_validation(L):
    lib = L.lib()
    need = ctypes.c_size_t(0)

    def params(**kw):
        p = dict(batch=2, rows=100, cols=60, dtype=L.PINSAGE_F32, steps=5, a=3.4445, b=-4.775,
                 c=2.0315, eps=1e-7)
        p.update(kw)
        return L.NewtonSchulz(**p)

    assert lib.pinsage_newton_schulz_workspace_size(None, ctypes.byref(need)) == L.PINSAGE_EINVAL
    assert lib.pinsage_newton_schulz_workspace_size(ctypes.byref(params()), None) == L.PINSAGE_EINVAL
    inval, unsup = L.PINSAGE_EINVAL, L.PINSAGE_EUNSUPPORTED
    for kw, want in ((dict(dtype=3), inval), (dict(batch=-1), inval), (dict(rows=0), inval),
                     (dict(cols=0), inval), (dict(steps=0), inval), (dict(steps=65), unsup),
                     (dict(rows=16385), unsup), (dict(batch=65536), unsup),
                     (dict(eps=-1.0), inval), (dict(eps=float("nan")), inval),
                     (dict(a=float("inf")), inval)):
        assert lib.pinsage_newton_schulz_workspace_size(ctypes.byref(params(**kw)),
                                                        ctypes.byref(need)) == want, kw
        assert need.value == 0
    assert lib.pinsage_newton_schulz_workspace_size(ctypes.byref(params()), ctypes.byref(need)) == 0
    size = need.value
    assert size > 2 * 100 * 60 * 4
    ortho = lambda i, o, ws, b: lib.pinsage_orthogonalize(ctypes.byref(params()), i, o, ws, b, None)
    assert ortho(None, FAKE, FAKE, size) == inval
    assert ortho(FAKE, None, FAKE, size) == inval
    assert ortho(FAKE, FAKE, FAKE, size - 1) == L.PINSAGE_EWORKSPACE
    assert ortho(FAKE, FAKE, None, size) == L.PINSAGE_EWORKSPACE
    assert ortho(FAKE, FAKE, FAKE + 1, size) == inval
    muon = lambda m, W=FAKE, g=FAKE, mom=FAKE, Wo=FAKE, mo=FAKE: lib.pinsage_muon_step(
        ctypes.byref(params()), ctypes.byref(m) if m is not None else None, W, g, mom, Wo, mo, FAKE,
        size - 1, None)
    ok = L.Muon(0.02, 0.95, 0.0, 1.0, 1)
    assert muon(None) == inval
    assert muon(L.Muon(float("nan"), 0.95, 0.0, 1.0, 1)) == inval
    for k in ("W", "g", "mom", "Wo", "mo"):
        assert muon(ok, **{k: None}) == inval
    assert muon(ok) == L.PINSAGE_EWORKSPACE
