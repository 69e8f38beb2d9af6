"""What the microscaled 4-bit entry points refuse, before anything is launched (CPU: addresses are never dereferenced)."""
import ctypes as C
import os

import pytest

from paper_2505_20932_amd import binding


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2505_20932_amd import build
        build.build_library(verbose=False)
    return binding.lib()


A, ODD4, ODD8, NULL = C.c_void_p(4096), C.c_void_p(4100), C.c_void_p(4104), None
F32, INT8, INT32, F16, BF16 = 1, 0, 2, 3, 4


def test_scale_bytes(lib):
    size = lib.cwac_mx4_scale_bytes
    assert size(1, 32) == 8 and size(5, 256) == 40 and size(5, 288) == 80 and size(16384, 11008) == 16384 * 43 * 8
    assert size(1 << 31, 1 << 18) == (1 << 31) * 8192
    assert size(0, 32) == 0 and size(4, 0) == 0 and size(4, (1 << 18) + 32) == 0


def test_quantize_and_dequantize(lib):
    q = lib.cwac_mx4_quantize
    #        x  type ldx rows k  codes ldc scales
    assert q(NULL, F32, 64, 4, 64, A, 32, A, NULL) == -1
    assert q(A, F32, 64, 4, 64, NULL, 32, A, NULL) == -1
    assert q(A, F32, 64, 4, 64, A, 32, NULL, NULL) == -1
    assert q(A, INT8, 64, 4, 64, A, 32, A, NULL) == -4
    assert q(A, F32, 64, 4, 48, A, 32, A, NULL) == -2         # k % 32
    assert q(A, F32, 64, 4, 0, A, 32, A, NULL) == -2
    assert q(A, F32, 64, -1, 64, A, 32, A, NULL) == -2
    assert q(A, F32, 32, 4, 64, A, 32, A, NULL) == -2         # ldx < k
    assert q(A, F32, 64, 4, 64, A, 16, A, NULL) == -2         # ldc < k / 2
    assert q(A, F32, 66, 4, 64, A, 32, A, NULL) == -3         # rows off the 16-byte grid
    assert q(A, F16, 68, 4, 64, A, 32, A, NULL) == -3
    assert q(ODD8, F32, 64, 4, 64, A, 32, A, NULL) == -3
    assert q(A, F32, 64, 4, 64, ODD8, 32, A, NULL) == -3
    assert q(A, F32, 64, 4, 64, A, 40, A, NULL) == -3
    assert q(A, F32, 64, 4, 64, A, 32, ODD4, NULL) == -3
    assert q(A, F32, 64, 0, 64, A, 32, A, NULL) == 0          # no rows: nothing to do
    d = lib.cwac_mx4_dequantize
    #        codes ldc scales rows k out type ldo
    assert d(NULL, 32, A, 4, 64, A, F32, 64, NULL) == -1
    assert d(A, 32, A, 4, 64, A, INT32, 64, NULL) == -4
    assert d(A, 32, A, 4, 80, A, F32, 80, NULL) == -2
    assert d(A, 32, A, 4, 64, A, BF16, 68, NULL) == -3
    assert d(A, 32, A, 0, 64, A, BF16, 64, NULL) == 0


def test_layer(lib):
    f = lib.qlinear_mx4_cwac_forward
    ok = dict(x=A, ldx=64, xs=A, w=A, ldw=64, ws=A, m=4, n=4, k=128, mult=NULL, fb=NULL, kind=F32, out=A, ldo=4)

    def call(**kw):
        a = {**ok, **kw}
        return f(*a.values(), NULL)
    for name in ("x", "xs", "w", "ws", "out"):
        assert call(**{name: NULL}) == -1
    for bad in (dict(m=0), dict(n=0), dict(k=0), dict(k=144), dict(k=(1 << 18) + 32), dict(ldx=48), dict(ldw=48), dict(ldo=3),
                dict(ldx=(1 << 24) + 16), dict(ldw=(1 << 24) + 16), dict(m=1 << 31)):
        assert call(**bad) == -2, bad
    for kind in (INT8, INT32, 5, -1):
        assert call(kind=kind) == -4
    for bad in (dict(x=ODD8), dict(w=ODD8), dict(ldx=72), dict(ldw=72), dict(xs=ODD4), dict(ws=ODD4), dict(out=C.c_void_p(4098))):
        assert call(**bad) == -3, bad
    assert call(kind=F16, out=C.c_void_p(4097)) == -3


def test_tuning(lib):
    f = lib.qlinear_mx4_cwac_forward_ex
    for bad in (binding.make_tuning(kernel=7), binding.make_tuning(shape=9), binding.make_tuning(persist_loaders=3)):
        assert f(A, 64, A, A, 64, A, 4, 4, 128, NULL, NULL, F32, A, 4, C.byref(bad), NULL) == -4
    assert f(A, 64, A, A, 64, A, 4, 4, 144, NULL, NULL, F32, A, 4, C.byref(binding.make_tuning()), NULL) == -2
