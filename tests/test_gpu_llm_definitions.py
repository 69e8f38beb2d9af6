"""The 8-bit append against the definition in 64 bits and against the library's own row quantizer; one request's attention alone and beside others."""
import numpy as np
import pytest
import torch

import paper_2505_20932_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("t", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_codes_and_scales_of_the_append(t, d):
    """s = max |x| / 127 to 2^-23 of itself (1 / 127 and the product, half a step each), a code within half a step and what that moves it by
    (127 * 2^-23 and the quotient's rounding); the row quantizer's differ by a last place and at midpoints only."""
    tokens, heads, page = 4000, 3, 16
    g = torch.Generator(device=DEV).manual_seed(d)
    x = (torch.randn(tokens, 2, heads, d, generator=g, device=DEV) * torch.exp2(torch.randint(-20, 12, (tokens, 2, heads, 1), device=DEV, generator=g).float())).to(t)
    pages = tokens // page
    kc, vc = (torch.zeros(pages, heads, page, d, dtype=torch.int8, device=DEV) for _ in range(2))
    ks, vs = (torch.zeros(pages, heads, page, device=DEV) for _ in range(2))
    slots = torch.randperm(tokens, generator=g, device=DEV)
    P.llm_kv_append(x[:, 0].contiguous(), x[:, 1].contiguous(), slots, kc, vc, ks, vs)
    for i, (c, s) in enumerate(((kc, ks), (vc, vs))):
        code = c.transpose(1, 2).reshape(tokens, heads, d)[slots].double()
        scale = s.transpose(1, 2).reshape(tokens, heads)[slots].double()
        v = x[:, i].double()
        want = (v.abs().amax(2) / 127).clamp(min=2.0 ** -118)
        assert ((scale - want).abs() <= 2.0 ** -23 * want).all()
        assert ((v / want[..., None] - code).abs() <= 0.5 + 127 * 2.0 ** -22).all()
        q, qs = torch.empty(tokens * heads, d, dtype=torch.int8, device=DEV), torch.empty(tokens * heads, device=DEV)
        P.cwac_quantize_rows_sym(x[:, i].float().reshape(-1, d).contiguous(), qs, q)
        assert ((qs.double() - scale.reshape(-1)).abs() <= 2.0 ** -23 * scale.reshape(-1)).all()
        other = q.view(tokens, heads, d).double() != code
        mid = ((v / want[..., None]).abs().frac() - 0.5).abs() <= 127 * 2.0 ** -22
        assert (mid | ~other).all()


@pytest.mark.parametrize("cache", ["f16", "i8"])
@pytest.mark.parametrize("cols", [2, 16, 32, 300])
def test_a_request_alone_and_beside_others(cache, cols):
    """For one batch size and table width a request's result is the same bits whatever the others are: one workgroup of one, four and eight
    wavefronts, split lengths."""
    batch, page, heads, kv, d = 4, 16, 8, 2, 128
    g = torch.Generator(device=DEV).manual_seed(cols)
    pages = batch * cols
    if cache == "i8":
        kc, vc = (torch.randint(-127, 128, (pages, kv, page, d), dtype=torch.int8, device=DEV, generator=g) for _ in range(2))
        ks, vs = (torch.rand(pages, kv, page, device=DEV, generator=g) * 0.02 for _ in range(2))
    else:
        kc, vc = (torch.randn(pages, kv, page, d, device=DEV, generator=g).half() for _ in range(2))
        ks = vs = None
    q = torch.randn(batch, heads, d, device=DEV, generator=g).half()
    table = torch.randperm(pages, device=DEV, generator=g).to(torch.int32).view(batch, cols)
    cap = cols * page
    ws = torch.empty(P.llm_paged_attention_workspace(batch, heads, kv, d, cols, page), dtype=torch.uint8, device=DEV)

    def run(lens, who=q):
        out = torch.full_like(q, 9.0)
        P.llm_paged_attention(who, kc, vc, ks, vs, table, torch.tensor(lens, dtype=torch.int32, device=DEV), d ** -0.5, 0, out, ws)
        return out
    lens = [cap, cap - 3, cap // 2 + 1, 1]
    base = run(lens)
    for i in range(batch):
        others = torch.randn(batch, heads, d, device=DEV, generator=g).half()
        others[i] = q[i]
        for rest in (0, cap, 7):
            mixed = [lens[i] if j == i else rest for j in range(batch)]
            assert torch.equal(run(mixed, others)[i], base[i])
