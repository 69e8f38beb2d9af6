"""How the attention over a paged cache is split (CPU): what the launcher plans fits the workspace that was asked for."""
import ctypes as C
import os
import subprocess

import pytest

_ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TILE, TURN = 32, 128


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("llm")
    src, so = d / "r.cpp", d / "r.so"
    src.write_text('''#include "llm_rules.h"
extern "C" {
int splits(long long batch, int heads, int kv, long long tokens) { return cwac::paged_splits(batch, heads, kv, tokens); }
long long chunk(long long tokens, int splits) { return cwac::paged_chunk(tokens, splits); }
int wide(long long batch, int heads, int kv, int d, long long tokens) { return cwac::paged_wide(batch, heads, kv, d, tokens); }
int waves(long long tokens) { return cwac::paged_waves(tokens); }
long long span(long long cap, int window) { return cwac::paged_span(cap, window); }
}
''')
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                    os.path.join(_ROOT, "paper_2505_20932_amd", "csrc"), str(src), "-o", str(so)], check=True)
    lib, ll, i = C.CDLL(str(so)), C.c_longlong, C.c_int
    lib.wide.argtypes = [ll, i, i, i, ll]
    lib.splits.argtypes, lib.chunk.argtypes, lib.span.argtypes = [ll, i, i, ll], [ll, i], [ll, i]
    lib.chunk.restype = lib.span.restype = ll
    return lib


def test_a_window_of_any_size(rules):
    cap = 64 * 1024
    assert rules.span(cap, 0) == cap and rules.span(cap, 1) == TILE and rules.span(cap, 1000) == 1031
    for window in (cap - 31, cap, cap + 1, 2**31 - 32, 2**31 - 31, 2**31 - 1):
        assert rules.span(cap, window) == cap
    for window in (1, 2, 31, 32, 33, 500):                            # enough for every place that a window can have
        for end in range(window, window + 2 * TILE):
            tiles = (end - 1) // TILE - (end - window) // TILE + 1
            assert -(-rules.span(cap, window) // TILE) >= tiles


def test_splits_cover_the_tokens_and_fit_the_workspace(rules):
    for batch in (1, 3, 61, 700, 65535):
        for heads, kv in ((1, 1), (8, 8), (32, 8), (34, 2), (1024, 1024)):
            for cap in (16, 1000, 4096, 131072, 2**31 - 65):
                most = rules.splits(batch, heads, kv, cap)
                assert 1 <= most <= 128
                for window in (0, 1, 100, 5000, 2**31 - 1):
                    n = rules.span(cap, window)
                    s = rules.splits(batch, heads, kv, n)
                    c = rules.chunk(n, s)
                    used = -(-n // c)
                    assert c % TURN == 0 and used * c >= n and 1 <= used <= s <= most


def test_short_lengths_go_to_one_workgroup(rules):
    # what was measured on both sides of the rule: rows (requests x key heads), head width, tokens
    for batch, kv, d, tokens, want in [(1, 32, 128, 256, 1), (1, 32, 128, 400, 1), (1, 32, 128, 700, 0), (1, 8, 128, 1000, 0), (8, 8, 128, 700, 1),
                                       (8, 8, 128, 1000, 0), (16, 8, 128, 1500, 1), (32, 8, 128, 2000, 1), (32, 8, 128, 3500, 0),
                                       (64, 8, 128, 2000, 1), (2, 8, 256, 256, 1), (2, 8, 256, 400, 0), (16, 8, 256, 1500, 1),
                                       (1, 1, 64, 128, 0), (4096, 8, 128, 512, 0)]:
        assert rules.wide(batch, 4 * kv, kv, d, tokens) == want, (batch, kv, d, tokens)


def test_no_more_wavefronts_than_tiles(rules):
    rules.waves.argtypes = [C.c_longlong]
    assert [rules.waves(n) for n in (1, 16, 32, 33, 64, 65, 128, 5000)] == [1, 1, 1, 2, 2, 4, 4, 4]
