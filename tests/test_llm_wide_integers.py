"""Whole numbers beyond 32 bits in the 4-bit and paged-cache calls (CPU: nothing is launched): refused, not taken modulo 2^32."""
import ctypes as C

import pytest
import torch

from paper_2505_20932_amd import binding as B

A = C.c_void_p(1 << 20)


def test_a_window_or_page_beyond_32_bits():
    f = B.lib().llm_paged_attention
    odd = C.c_void_p((1 << 20) + 2)                                    # (an address that the call refuses by itself)
    call = [odd, 512, B.CWAC_OUT_FP16, A, A, B.CWAC_OUT_FP16, None, None, 9, 16, A, 64, 64, A, 3, 4, 2, 128, 1.0, 0, A, 512, A, 1 << 30, None]
    assert f(*call) == -3
    for at, value in ((19, 2 ** 32 + 5), (19, 2 ** 31), (19, -2 ** 32), (9, 2 ** 32 + 16), (8, 2 ** 32 + 9), (12, 2 ** 32 + 64), (14, 2 ** 32 + 3)):
        with pytest.raises(C.ArgumentError):
            f(*call[:at], value, *call[at + 1:])


def test_a_page_of_the_assignment():
    f = B.lib().llm_kv_assign_pages
    call = [A, A, 4, 16, A, 64, A, A, 8, 8, A, 32, A, A, A, None]       # (outputs over inputs: refused by itself)
    assert f(*call) == -4
    with pytest.raises(C.ArgumentError):
        f(*call[:3], 2 ** 32 + 16, *call[4:])


def test_a_row_of_codes_of_2_to_the_32_values():
    q = B.lib().cwac_mx4_quantize
    assert q(C.c_void_p(4), B.CWAC_OUT_FP32, 64, 4, 64, A, 32, A, None) == -3
    with pytest.raises(C.ArgumentError):
        q(C.c_void_p(4), B.CWAC_OUT_FP32, 1 << 40, 4, 2 ** 32 + 64, A, 1 << 40, A, None)
    f = B.lib().qlinear_mx4_cwac_forward
    with pytest.raises(C.ArgumentError):
        f(C.c_void_p(4), 1 << 24, A, A, 1 << 24, A, 4, 4, 2 ** 32 + 64, None, None, B.CWAC_OUT_FP32, A, 4, None)


def test_queries():
    assert B.cwac_mx4_scale_bytes(1, 32) == 8 and B.cwac_mx4_scale_bytes(1, 2 ** 32 + 32) == 0
    ok = (3, 32, 8, 128, 4096, 16)
    assert B.llm_paged_attention_workspace(*ok) > 16
    for i in range(6):
        assert B.llm_paged_attention_workspace(*ok[:i], ok[i] + 2 ** 32, *ok[i + 1:]) == 0
    with pytest.raises(C.ArgumentError):
        B.cwac_mx4_scale_bytes(1, 32.0)


@pytest.mark.gpu
@pytest.mark.parametrize("window", [2 ** 32, 2 ** 32 + 5, 2 ** 31])
def test_the_call_itself(window):
    z = lambda *s, dtype=torch.float16: torch.zeros(s, dtype=dtype, device="cuda:0")  # noqa: E731
    q, kc, vc, out = z(1, 2, 64), z(2, 1, 16, 64), z(2, 1, 16, 64) + 1, z(1, 2, 64)
    table, lens = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda:0"), z(1, dtype=torch.int32) + 32
    with pytest.raises(C.ArgumentError):
        B.llm_paged_attention(q, kc, vc, None, None, table, lens, 0.1, window, out, None)
    assert not out.any()
