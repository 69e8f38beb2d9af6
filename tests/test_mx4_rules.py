"""The rule that picks a kernel for a layer on microscaled 4-bit operands, at measured sizes (CPU)."""
import os
import subprocess

import pytest

_ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SPLIT16, SPLIT32X16, SPLIT32, SPLIT64, DEEP, PAIR, T256 = range(1, 8)


@pytest.fixture(scope="module")
def form(tmp_path_factory):
    import ctypes as C
    d = tmp_path_factory.mktemp("mx4")
    src, so = d / "r.cpp", d / "r.so"
    src.write_text('#include "mx4_rules.h"\nextern "C" int form(long long m, int n, int k) { return cwac::mx4_form(m, n, k); }\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                    os.path.join(_ROOT, "paper_2505_20932_amd", "csrc"), "-I", os.path.join(_ROOT, "include"), str(src), "-o", str(so)], check=True)
    f = C.CDLL(str(so)).form
    f.argtypes = [C.c_longlong, C.c_int, C.c_int]
    return f


@pytest.mark.parametrize("m,n,k,want", [
    (1, 4096, 4096, SPLIT16), (16, 4096, 11008, SPLIT16), (1, 11008, 4096, SPLIT32X16), (24, 4096, 11008, SPLIT32X16),
    (64, 4096, 4096, SPLIT32), (128, 4096, 4096, SPLIT32), (1024, 768, 2880, SPLIT32), (256, 4096, 11008, SPLIT64), (200, 4096, 4096, SPLIT64),
    (601, 4096, 4096, DEEP), (601, 2304, 768, DEEP), (601, 2049, 5504, DEEP), (4096, 1024, 1024, DEEP), (2048, 4096, 4096, PAIR),
    (1500, 11008, 4096, PAIR), (8192, 2304, 768, PAIR), (8192, 2049, 5504, PAIR), (4096, 4096, 4096, T256), (16384, 4096, 11008, T256),
    (8192, 11008, 4096, T256), (1, 1, 32, SPLIT16), (100000, 17, 64, SPLIT32), (50, 100000, 64, SPLIT32)])
def test_measured_sizes(form, m, n, k, want):
    assert form(m, n, k) == want


def test_every_tile_fits_its_layer(form):
    for m in (1, 16, 17, 127, 128, 255, 256, 3000, 1 << 20):
        for n in (1, 127, 128, 255, 256, 5000, 1 << 20):
            for k in (32, 800, 4096, 1 << 18):
                f = form(m, n, k)
                assert f in range(1, 8)
                if f in (DEEP, PAIR):
                    assert m >= 128 and n >= 128
                if f == T256:
                    assert m >= 256 and n >= 256
