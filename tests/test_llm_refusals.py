"""What the paged cache's entry points refuse, before anything is launched (CPU: addresses are never dereferenced), and the
rule that splits a length."""
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


def P(n):
    return C.c_void_p(n << 20)          # addresses a MiB apart


NULL = None
FP32, INT8, F16, BF16 = 1, 0, 3, 4


def _caller(f, ok):
    def call(**kw):
        assert set(kw) <= set(ok)
        return f(*{**ok, **kw}.values(), NULL)
    return call


def test_assign_pages(lib):
    call = _caller(lib.llm_kv_assign_pages,
                   dict(old=P(1), new=P(2), batch=4, page=16, free=P(3), cap=64, n_free=P(4), table=P(5), ldt=8, cols=8,
                        slots=P(6), slot_cap=32, start=P(7), lens=P(8), left=P(9)))
    for name in ("old", "new", "free", "n_free", "table", "slots", "start", "lens", "left"):
        assert call(**{name: NULL}) == -1, name
    for bad in (dict(batch=0), dict(batch=8193), dict(page=8), dict(page=24), dict(page=2048), dict(page=0), dict(cap=-1),
                dict(cols=0, ldt=0), dict(ldt=7), dict(slot_cap=-1), dict(cols=1 << 27, ldt=1 << 27)):
        assert call(**bad) == -2, bad
    for name in ("old", "new", "free", "n_free", "table", "start", "lens", "left"):
        assert call(**{name: C.c_void_p((20 << 20) + 2)}) == -3, name
    assert call(slots=C.c_void_p((20 << 20) + 4)) == -3
    # what is written is not what is read
    for bad in (dict(lens=P(1)), dict(lens=P(2)), dict(left=P(4)), dict(start=P(1)), dict(left=C.c_void_p((3 << 20) + 63 * 4)),
                dict(table=C.c_void_p((3 << 20) - 31 * 4)), dict(slots=P(3)), dict(start=C.c_void_p((1 << 20) - 16))):
        assert call(**bad) == -4, bad


def test_append(lib):
    call = _caller(lib.llm_kv_append,
                   dict(k=P(1), ldk=256, v=P(2), ldv=256, type=F16, slots=P(3), tokens=5, heads=2, d=128, kc=P(4), vc=P(5),
                        kind=F16, ks=NULL, vs=NULL, pages=9, page=16))
    for name in ("k", "v", "slots", "kc", "vc"):
        assert call(**{name: NULL}) == -1, name
    assert call(kind=INT8) == -1 and call(kind=INT8, ks=P(6)) == -1          # an 8-bit cache has scales
    for bad in (dict(tokens=-1), dict(heads=0), dict(heads=1025), dict(d=96), dict(pages=0), dict(page=8), dict(page=48), dict(ldk=248),
                dict(ldv=248)):
        assert call(**bad) == -2, bad
    for bad in (dict(type=FP32), dict(type=INT8), dict(kind=BF16), dict(kind=FP32), dict(type=BF16)):
        assert call(**bad) == -4, bad
    for bad in (dict(k=C.c_void_p(4104)), dict(v=C.c_void_p(4104)), dict(ldk=260), dict(ldv=260), dict(slots=C.c_void_p(4100)),
                dict(kc=C.c_void_p(4104)), dict(vc=C.c_void_p(4104)), dict(kind=INT8, ks=C.c_void_p(4098), vs=P(7))):
        assert call(**bad) == -3, bad
    assert call(tokens=0) == 0


def test_attention(lib):
    call = _caller(lib.llm_paged_attention,
                   dict(q=P(1), ldq=512, type=F16, kc=P(2), vc=P(3), kind=F16, ks=NULL, vs=NULL, pages=9, page=16, table=P(4),
                        ldt=64, cols=64, lens=P(5), batch=3, heads=4, kv=2, d=128, scale=1.0, window=0, out=P(6), ldo=512,
                        ws=P(7), bytes=1 << 30))
    for name in ("q", "kc", "vc", "table", "lens", "out"):
        assert call(**{name: NULL}) == -1, name
    assert call(kind=INT8) == -1 and call(kind=INT8, vs=P(8)) == -1
    for bad in (dict(batch=0), dict(batch=65536), dict(heads=0), dict(heads=5), dict(kv=0), dict(heads=2050, kv=1025), dict(d=80),
                dict(cols=0), dict(ldt=63), dict(page=20), dict(pages=0), dict(window=-1), dict(ldq=511), dict(ldo=508),
                dict(cols=1 << 27, ldt=1 << 27)):
        assert call(**bad) == -2, bad
    for bad in (dict(type=FP32), dict(type=INT8), dict(kind=BF16), dict(kind=FP32)):
        assert call(**bad) == -4, bad
    for bad in (dict(q=C.c_void_p(4104)), dict(ldq=516), dict(kc=C.c_void_p(4104)), dict(vc=C.c_void_p(4104)), dict(table=C.c_void_p(4098)),
                dict(lens=C.c_void_p(4098)), dict(out=C.c_void_p(4100)), dict(ldo=514), dict(ws=C.c_void_p(4104))):
        assert call(**bad) == -3, bad
    need = lib.llm_paged_attention_workspace(3, 4, 2, 128, 64, 16)
    assert need > 16                                                           # 1024 tokens of six rows are split
    assert call(ws=NULL) == -5 and call(bytes=need - 1) == -5


def test_workspace_sizes(lib):
    size = lib.llm_paged_attention_workspace
    assert size(0, 4, 2, 128, 64, 16) == 0 and size(3, 4, 3, 128, 64, 16) == 0 and size(3, 4, 2, 96, 64, 16) == 0
    assert size(4096, 32, 8, 128, 512, 16) == 16                               # enough rows: nothing is split
    # no more splits than turns of 128 tokens, and never more than 128
    for batch, kv, cols in ((1, 1, 8), (1, 8, 512), (7, 2, 8192), (64, 8, 512), (1, 1, 1 << 20)):
        got = size(batch, 4 * kv, kv, 128, cols, 16)
        splits = got // (batch * 4 * kv * 130 * 4)
        assert got in (16, splits * batch * 4 * kv * 130 * 4)
        assert splits <= min(128, -(-cols * 16 // 128))
