"""Attention over short paged lengths, where one workgroup takes a request's whole length: sizes on both sides of its turns, against the
plain 64-bit form, and the same request alone and in a batch of the same shape."""
import pytest
import torch

import paper_2505_20932_amd as P
from test_gpu_llm import DEV, I4, _case, _check, _run

pytestmark = pytest.mark.gpu

SHAPES = [
    # lens, page, q heads, kv heads, d, window, columns
    ([129], 16, 1, 1, 64, 0, None), ([255, 256, 257, 0, 1], 16, 8, 2, 128, 0, 32), ([512, 511, 224, 225], 32, 33, 1, 64, 0, 16),
    ([1, 2, 3, 500], 16, 20, 4, 128, 100, None), ([480, 33] * 16, 16, 16, 8, 128, 0, None), ([1600, 1, 0, 999] * 6, 64, 12, 6, 64, 0, None),
    ([256, 17], 16, 8, 4, 256, 0, 16), ([2048, 5, 300] * 20, 128, 6, 3, 64, 700, 16), ([300] * 9, 16, 16, 16, 256, 0, None),
]


@pytest.mark.parametrize("lens,page,heads,kv,d,window,cols", SHAPES)
@pytest.mark.parametrize("t,cache", [("f16", "f16"), ("bf16", "bf16"), ("f16", "i8"), ("bf16", "i8")])
def test_short_lengths(lens, page, heads, kv, d, window, cols, t, cache):
    case = _case(lens, page, heads, kv, d, t, cache, 11 + len(lens) + d, cols)
    scale = -0.7 * d ** -0.5 if heads == 20 else d ** -0.5
    out = _run(*case, scale, window, page)
    assert torch.equal(out, _run(*case, scale, window, page))
    _check(out, *case, scale, window, t)


@pytest.mark.parametrize("cache", ["f16", "i8"])
def test_missing_pages(cache):
    q, k, v, ks, vs, table, lens = _case([400, 390, 70], 16, 8, 2, 128, "f16", cache, 3)
    table[0, 3:9], table[1, 0], table[2, :] = -1, k.shape[0], -5
    _check(_run(q, k, v, ks, vs, table, lens, 0.1, 0, 16), q, k, v, ks, vs, table, lens, 0.1, 0, "f16")


def test_no_workspace_is_needed():
    q, k, v, ks, vs, table, lens = _case([250, 3], 16, 8, 2, 128, "f16", "f16", 5)
    want = _run(q, k, v, ks, vs, table, lens, 0.1, 0, 16)
    out = torch.zeros_like(q)
    P.llm_paged_attention(q, k, v, ks, vs, table, lens, 0.1, 0, out, None)
    assert torch.equal(out, want)
    lens.copy_(torch.tensor([0, -4], dtype=I4, device=DEV))
    P.llm_paged_attention(q, k, v, ks, vs, table, lens, 0.1, 0, out, None)
    assert not out.any()
