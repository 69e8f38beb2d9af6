"""The 4-bit and paged-cache calls through the binding: the native form and the ctypes form give the same bytes and refuse the same
calls; other streams, threads, and captured steps that share a workspace."""
import ctypes
import threading

import numpy as np
import pytest
import torch

import paper_2505_20932_amd as P
from paper_2505_20932_amd import binding as B

DEV = "cuda:0"
U1, I4, I8, F2 = torch.uint8, torch.int32, torch.int64, torch.float16
NATIVE = {"mx4_quantize": 4, "mx4_dequantize": 4, "mx4_forward": 8, "kv_assign": 11, "kv_append": 8, "paged_attention": 12}


def mx4(rows, k, dev=DEV):
    return torch.zeros(rows, k // 2, dtype=U1, device=dev), torch.zeros(-(-k // 256), rows, 8, dtype=U1, device=dev)


def everything(dev):
    """One call of each kind: {native name: (entry point, arguments, what it writes)}."""
    g = torch.Generator(device=dev).manual_seed(3)
    x = torch.randn(5, 320, device=dev, generator=g)
    w = torch.randn(48, 320, device=dev, generator=g)
    f, y = torch.zeros(5, 320, device=dev), torch.zeros(5, 48, dtype=F2, device=dev)
    xc, wc = mx4(5, 320, dev), mx4(48, 320, dev)
    mult = torch.rand(48, device=dev, generator=g)
    old, new = torch.tensor([0, 3, 16], dtype=I4, device=dev), torch.tensor([1, 20, 1], dtype=I4, device=dev)
    free, n_free = torch.arange(8, dtype=I4, device=dev), torch.tensor([8], dtype=I4, device=dev)
    table = torch.full((3, 4), -1, dtype=I4, device=dev)
    table[1, 0], table[2, 0] = 8, 9
    slots = torch.zeros(22, dtype=I8, device=dev)
    start, lens, left = (torch.zeros(n, dtype=I4, device=dev) for n in (4, 3, 1))
    kv = torch.randn(22, 2, 2, 64, device=dev, generator=g).to(F2)
    kc, vc = (torch.zeros(10, 2, 16, 64, dtype=torch.int8, device=dev) for _ in range(2))
    ks, vs = (torch.zeros(10, 2, 16, device=dev) for _ in range(2))
    q, o = torch.randn(3, 4, 64, device=dev, generator=g).to(F2), torch.zeros(3, 4, 64, dtype=F2, device=dev)
    ws = torch.zeros(B.llm_paged_attention_workspace(3, 4, 2, 64, 4, 16), dtype=U1, device=dev)
    return {
        "mx4_quantize": (P.cwac_mx4_quantize, [x, *xc], xc),
        "mx4_quantize w": (P.cwac_mx4_quantize, [w, *wc], wc),
        "mx4_dequantize": (P.cwac_mx4_dequantize, [*xc, f], [f]),
        "mx4_forward": (P.qlinear_mx4_cwac_forward, [*xc, *wc, mult, None, y], [y]),
        "kv_assign": (P.llm_kv_assign_pages, [old, new, 16, free, n_free, table, slots, start, lens, left], [table, slots, start, lens, left]),
        "kv_append": (P.llm_kv_append, [kv[:, 0], kv[:, 1], slots, kc, vc, ks, vs], [kc, vc, ks, vs]),
        "paged_attention": (P.llm_paged_attention, [q, kc, vc, ks, vs, table, lens, 0.125, 0, o, ws], [o]),
    }


def test_native_forms_decline_what_is_not_on_a_device():
    calls = B._fast_calls()
    for name, (entry, args, _) in everything("cpu").items():
        native = getattr(calls, name.split()[0])
        assert native(*args, None) is False and native(*args) is False and native() is False
        assert native(*["x"] * NATIVE[name.split()[0]]) is False
        with pytest.raises(AssertionError):
            entry(*args)


def test_more_tokens_than_can_be_counted():
    assert B.lib().llm_kv_append(16, 64, 16, 64, B.CWAC_OUT_FP16, 16, 1 << 31, 1, 64, 16, 16, B.CWAC_OUT_FP16, None, None, 4, 16,
                                 None) == -2


@pytest.mark.gpu
def test_native_and_ctypes_forms_agree(monkeypatch):
    calls, a = B._fast_calls(), everything(DEV)
    for name, (_, args, _) in a.items():
        assert getattr(calls, name.split()[0])(*args, None) is True, name
    b = everything(DEV)
    monkeypatch.setattr(B, "_calls", B._NoFastCalls())
    for entry, args, _ in b.values():
        entry(*args)
    for name in a:
        for s, t in zip(a[name][2], b[name][2]):
            assert torch.equal(s.view(U1), t.view(U1)) and s.any(), name


def misfits():
    """{native name: calls of it that must be refused, as changes of one argument}"""
    c = everything(DEV)
    z = lambda *s, dtype=F2: torch.zeros(s, dtype=dtype, device=DEV)  # noqa: E731
    return c, {
        "mx4_quantize": [(0, z(5, 320, dtype=torch.float64)), (0, z(4, 320, dtype=torch.float32)), (0, z(320, 5, dtype=torch.float32).t()), (1, z(5, 160)),
                         (1, z(5, 152, dtype=U1)), (2, z(1, 5, 8, dtype=U1)), (2, z(2, 5, 16, dtype=U1)[..., ::2]), (2, z(80, dtype=U1))],
        "mx4_dequantize": [(2, z(5, 320, dtype=I4)), (2, z(5, 288)), (0, z(5, 160, dtype=torch.int8)), (2, z(1600))],
        "mx4_forward": [(0, z(5, 144, dtype=U1)), (2, z(47, 160, dtype=U1)), (4, z(47, dtype=torch.float32)), (4, z(48)), (5, z(96, dtype=torch.float32)[::2]),
                        (6, z(48, 5).t()), (6, z(6, 48)), (6, z(5, 48, dtype=torch.float64)), (3, z(2, 47, 8, dtype=U1))],
        "kv_assign": [(0, z(3, dtype=I8)), (1, z(4, dtype=I4)), (2, 17), (2, 2.0), (3, z(8, dtype=I8)), (4, z(2, dtype=I4)), (5, z(2, 4, dtype=I4)),
                      (5, z(4, 3, dtype=I4).t()), (6, z(22, dtype=I4)), (7, z(3, dtype=I4)), (8, z(6, dtype=I4)[::2]), (8, c["kv_assign"][1][0])],
        "kv_append": [(0, z(22, 2, 64, dtype=torch.bfloat16)), (0, z(22, 3, 64)), (0, z(22, 2, 128)[:, :, ::2]), (1, z(21, 2, 64)), (2, z(21, dtype=I8)),
                      (2, z(22, dtype=I4)), (3, z(10, 2, 16, 64)), (4, z(9, 2, 16, 64, dtype=torch.int8)), (5, z(10, 2, 16)), (6, None), (0, z(22, 128)),
                      (0, z(22, 4, 64)[:, ::2])],
        "paged_attention": [(0, z(3, 3, 64)), (0, z(3, 4, 128)), (9, z(3, 4, 64, dtype=torch.bfloat16)), (9, z(2, 4, 64)), (5, z(2, 4, dtype=I4)),
                            (5, z(3, 4, dtype=I8)), (6, z(4, dtype=I4)), (6, z(3, dtype=I8)), (7, "1"), (8, -1),
                            (3, None), (1, z(10, 2, 16, 64))],
    }


@pytest.mark.gpu
def test_misfits_are_refused():
    calls, (c, bad) = B._fast_calls(), misfits()
    for name, changes in bad.items():
        entry, args, outs = c[name]
        before = [t.clone() for t in outs]
        for at, value in changes:
            call = list(args)
            call[at] = value
            assert getattr(calls, name)(*call, None) is False, (name, at)
            with pytest.raises((AssertionError, B.CwacError, KeyError, ValueError, AttributeError, ctypes.ArgumentError)):
                entry(*call)
        for s, t in zip(before, outs):
            assert torch.equal(s.view(U1), t.view(U1)), name
    entry, args, outs = c["paged_attention"]
    # a length that is not split needs no workspace (16 bytes are asked for, so that it is never an empty one) ...
    assert args[10].numel() == 16
    assert calls.paged_attention(*args[:10], None, None) is True
    wide = torch.full((3, 4096), -1, dtype=I4, device=DEV)            # ... one that is does
    for ws in (None, torch.zeros(16, dtype=U1, device=DEV)):
        call = args[:5] + [wide] + args[6:10] + [ws]
        assert calls.paged_attention(*call, None) is False
        with pytest.raises(B.CwacError):
            entry(*call)
    P.llm_kv_assign_pages(*c["kv_assign"][1])
    P.llm_kv_append(*c["kv_append"][1])
    for scale in (np.float64(0.125), 0.125):                          # numbers of other types are the ctypes form's
        outs[0].zero_()
        entry(*args[:7], scale, np.int64(0), *args[9:])
        assert outs[0].any()


@pytest.mark.gpu
def test_another_stream_and_threads():
    want = everything(DEV)
    for entry, args, _ in want.values():
        entry(*args)
    given = everything(DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for entry, args, _ in given.values():                              # a stream given
        entry(*args, stream=s)
    s.synchronize()
    sets = [everything(DEV) for _ in range(4)]
    torch.cuda.synchronize()

    def work(calls):
        with torch.cuda.stream(torch.cuda.Stream()):                  # the thread's current stream
            for _ in range(20):
                for entry, args, _ in calls.values():
                    entry(*args)
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(c,)) for c in sets]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for calls in [given] + sets:
        for name in want:
            for a, b in zip(want[name][2], calls[name][2]):
                assert torch.equal(a.view(U1), b.view(U1)), name


@pytest.mark.gpu
def test_two_captured_attentions_share_a_workspace():
    """Two graphs of the same shapes and one workspace, replayed in turn on one stream with other calls between them."""
    g = torch.Generator(device=DEV).manual_seed(8)
    page, cols, heads, kv, d = 16, 256, 8, 2, 128
    kc, vc = (torch.randn(cols, kv, page, d, device=DEV, generator=g).to(F2) for _ in range(2))
    table = torch.randperm(cols, device=DEV, generator=g).to(I4)[None].contiguous()
    ws = torch.empty(B.llm_paged_attention_workspace(1, heads, kv, d, cols, page), dtype=U1, device=DEV)
    assert ws.numel() > 0
    runs = []
    for n in (4000, 1201):
        q = torch.randn(1, heads, d, device=DEV, generator=g).to(F2)
        lens, out = torch.tensor([n], dtype=I4, device=DEV), torch.zeros(1, heads, d, dtype=F2, device=DEV)
        args = (q, kc, vc, None, None, table, lens, d ** -0.5, 0, out, ws)
        P.llm_paged_attention(*args)
        want = out.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            P.llm_paged_attention(*args)
        runs.append((graph, args, out, want))
    for i in range(6):
        for graph, args, out, want in (runs if i % 2 else runs[::-1]):
            out.zero_()
            if i % 3 == 0:
                P.llm_paged_attention(*runs[0][1])
                runs[0][2].zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


@pytest.mark.gpu
@pytest.mark.parametrize("window", [4096, 2**31 - 32, 2**31 - 1])
def test_a_window_that_sees_everything(window):
    g = torch.Generator(device=DEV).manual_seed(9)
    kc, vc = (torch.randn(256, 2, 16, 64, device=DEV, generator=g).to(F2) for _ in range(2))
    q, out = torch.randn(3, 4, 64, device=DEV, generator=g).to(F2), torch.zeros(3, 4, 64, dtype=F2, device=DEV)
    table, lens = torch.arange(256, dtype=I4, device=DEV).repeat(3, 1), torch.tensor([4096, 1, 300], dtype=I4, device=DEV)
    ws = torch.zeros(B.llm_paged_attention_workspace(3, 4, 2, 64, 256, 16), dtype=U1, device=DEV)
    P.llm_paged_attention(q, kc, vc, None, None, table, lens, 0.125, 0, out, ws)
    want = out.clone()
    P.llm_paged_attention(q, kc, vc, None, None, table, lens, 0.125, window, out.zero_(), ws)
    assert torch.equal(out, want)
