"""Attention over a paged cache whose tokens count very unevenly: one that takes nearly all of the weight and brings nothing, one whose values are
far larger and whose weight is next to none, early, late and in the middle of a length, against the 64-bit form."""
import numpy as np
import pytest
import torch

import paper_2505_20932_amd as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}
EPS = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
# (length, columns of the table, q heads, kv heads, head size): one, two, four and eight wavefronts, splits, heads of 256
SHAPES = [(30, 2, 4, 2, 64), (61, 4, 3, 1, 128), (300, 20, 64, 32, 64), (250, 16, 8, 4, 128), (700, 64, 8, 2, 64), (3000, 200, 4, 2, 128), (900, 60, 2, 1, 256)]
SCALE = 0.25
SPECIAL = 4.0                                    # dim 0 of every query; of the keys only a special token's is not zero: its logit is exact


def _cache(n, cols, heads, kv, d, t, cache, special, seed):
    """One request of n tokens in order.  special: {token: (its logit, the factor of its values)}; the others' logits are about N(0, 1), their
    values between 32 and 64."""
    page = 16
    rng = np.random.default_rng(seed)
    k = rng.standard_normal((n, kv, d)) / np.sqrt(d - 1)
    q = rng.standard_normal((1, heads, d)) / SCALE
    v = 32.0 + 32.0 * rng.random((n, kv, d))
    k[:, :, 0], q[:, :, 0] = 0.0, SPECIAL
    for at, (logit, factor) in special.items():
        k[at], k[at, :, 0] = 0.0, logit / (SCALE * SPECIAL)
        v[at] *= factor
    pages = -(-n // page)
    store = []
    for x in (k, v):
        full = np.zeros((pages * page, kv, d))
        full[:n] = x
        full = torch.from_numpy(full).view(pages, page, kv, d).transpose(1, 2).contiguous()
        if cache == "i8":
            s = (full.abs().amax(-1) / 127).clamp(min=2.0 ** -118).float()
            store.append((torch.round(full / s.double()[..., None]).clamp(-127, 127).to(torch.int8).to(DEV), s.to(DEV)))
        else:
            store.append((full.to(TYPES[cache]).to(DEV), None))
    table = torch.full((1, cols), -1, dtype=torch.int32)
    table[0, :pages] = torch.arange(pages)
    (kc, ks), (vc, vs) = store
    return torch.from_numpy(q).to(TYPES[t]).to(DEV), kc, vc, ks, vs, table.to(DEV), torch.tensor([n], dtype=torch.int32, device=DEV)


def _reference(q, kc, vc, ks, vs, n):
    """Per head: the output, sum w |v|, the largest sum of |q k|, the largest |v| (8-bit cache: the largest w * s over the
    values' scales s)."""
    def rows(c, s):
        x = c.double() if s is None else c.double() * s.double()[..., None]
        return x.transpose(1, 2).reshape(-1, c.shape[1], c.shape[3])[:n].cpu().numpy()
    k, v, qn = rows(kc, ks), rows(vc, vs), q[0].double().cpu().numpy()
    heads, d = qn.shape
    group = heads // k.shape[1]
    out, mag, qk, peak = np.zeros((heads, d)), np.zeros((heads, d)), np.zeros(heads), np.zeros(heads)
    for h in range(heads):
        g = h // group
        s = SCALE * (k[:, g] @ qn[h])
        w = np.exp(s - s.max())
        w /= w.sum()
        out[h], mag[h] = w @ v[:, g], w @ np.abs(v[:, g])
        qk[h] = SCALE * (np.abs(k[:, g]) @ np.abs(qn[h])).max()
        unit = np.abs(v[:, g]).max(axis=1) if vs is None else vs.double().transpose(1, 2).reshape(-1, kc.shape[1])[:n, g].cpu().numpy()
        peak[h] = unit.max() if vs is None else (w * unit).max()
    return out, mag, qk, peak


def _run(n, cols, heads, kv, d, t, cache, special, seed=0):
    c = _cache(n, cols, heads, kv, d, t, cache, special, seed)
    q, kc, vc, ks, vs, table, lens = c
    out = torch.full_like(q, 9.0)
    ws = torch.empty(P.llm_paged_attention_workspace(1, heads, kv, d, cols, 16), dtype=torch.uint8, device=DEV)
    P.llm_paged_attention(q, kc, vc, ks, vs, table, lens, SCALE, 0, out, ws)
    want, mag, qk, peak = _reference(q, kc, vc, ks, vs, n)
    # Relative to sum w |v|: the two terms of a weight (2^-20 cut off binary16, 2^-16 bfloat16); the logits' fp32 sums, products and
    # exponential, which enter a weight relatively and both sums; the fp32 sums over the tokens.  bfloat16 queries over 8 bits are binary16 relative
    # to 2^e <= 2 max |q|, each off by at most half its smallest step: 2^-25 * 2^e.
    half = t == "f16" or cache == "i8"
    logit = (d / 16 + 8) * 2.0 ** -23 * (qk + 1.0)
    if t == "bf16" and half:
        top = float(kc.abs().amax()) if ks is None else float((kc.abs().amax(-1).float() * ks).amax())
        logit = logit + d * 2.0 ** -24 * float(q.abs().max()) * top * SCALE
    rel = (2.0 ** -20 if half else 2.0 ** -16) + 2 * logit + 2.0 ** -23 * (n + 16)
    # Absolute, per token: binary16's smallest step, 2^-24.  16 bit: the largest weight is 2^15 (and their sum no less), so 2^-39 of the largest value.
    # 8 bit: where a weight times its scale is largest it is 2^10 or more, so 2^-34 of it next to codes of at most 127.
    step = 0.0 if not half else n * (2.0 ** -39 * peak if cache != "i8" else 2.0 ** -34 * 127 * peak)
    tol = EPS[t] * np.abs(want) + (rel[:, None] * mag + np.reshape(step, (-1, 1))) * 1.01 + (2.0 ** -25 if t == "f16" else 2.0 ** -134)
    got = out[0].double().cpu().numpy()
    assert np.isfinite(got).all()
    err = np.abs(got - want)
    print(f"{t} {cache} {n} {d} {special}: error {(err / np.maximum(np.abs(want), 1e-300)).max():.2e} of the output, {(err / tol).max():.2f} of the bound",
          flush=True)
    assert (err <= tol).all()


@pytest.mark.parametrize("gap", [8, 12, 14, 16])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("t,cache", [("f16", "f16"), ("bf16", "bf16"), ("f16", "i8"), ("bf16", "i8")])
def test_a_token_of_nearly_all_the_weight_and_no_values(shape, t, cache, gap):
    """The output is what the others' small weights bring."""
    for at in (0, shape[0] - 1):
        _run(*shape, t, cache, {at: (float(gap), 0.0)})


UNEVEN = [("bf16", "bf16"), ("f16", "i8"), ("bf16", "i8")]


@pytest.mark.parametrize("factor", [6, 10, 13, 16, 20, 40])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("t,cache", UNEVEN)
def test_a_token_of_large_values_and_no_weight(shape, t, cache, factor):
    """Values 2^factor times the others' at e^-50 of their weight: the others' output."""
    for at in (0, shape[0] // 2, shape[0] - 1):
        _run(*shape, t, cache, {at: (-50.0, 2.0 ** factor)})


@pytest.mark.parametrize("factor", [-20, 4, 16, 24])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("t,cache", UNEVEN)
def test_large_values_lose_their_weight(shape, t, cache, factor):
    """Tokens of other values lead for a while; then come logits that leave them e^-40.  And the other way round."""
    n = shape[0]
    early, late = range(0, max(1, n // 4)), range(n - max(1, n // 4), n)
    for low, high in ((early, late), (late, early)):
        special = {i: (3.0 + 0.01 * (i % 7), 2.0 ** factor) for i in low}
        special.update({i: (43.0 + 0.1 * (i % 11), 1.0) for i in high})
        _run(*shape, t, cache, special)


@pytest.mark.parametrize("scale", [1.0, -1.0, 8.0, 2.0 ** -3])
@pytest.mark.parametrize("d,n", [(64, 40), (128, 900), (256, 300)])
def test_the_largest_bfloat16_queries_over_8_bits(d, n, scale):
    """Queries of 2^127 over key scales of 2^-125: logits of 64 at most."""
    g = torch.Generator(device=DEV).manual_seed(n)
    pages = -(-n // 16)
    kc = torch.zeros(pages, 1, 16, d, dtype=torch.int8, device=DEV)
    kc[..., 3] = torch.randint(0, 3, kc.shape[:3], device=DEV, generator=g).to(torch.int8)
    ks = torch.full(kc.shape[:3], 2.0 ** -125, device=DEV)
    vc = torch.randint(1, 128, kc.shape, device=DEV, generator=g).to(torch.int8)
    vs = torch.full(kc.shape[:3], 0.01, device=DEV)
    q = torch.zeros(1, 2, d, dtype=torch.bfloat16, device=DEV)
    q[0, 0, 3], q[0, 1, 3] = 2.0 ** 127, -2.0 ** 127
    q[0, :, 5] = 2.0 ** 120                                            # meets zeros
    table, lens = torch.arange(pages, dtype=torch.int32, device=DEV)[None].contiguous(), torch.tensor([n], dtype=torch.int32, device=DEV)
    out = torch.full_like(q, 9.0)
    ws = torch.empty(max(1, P.llm_paged_attention_workspace(1, 2, 1, d, pages, 16)), dtype=torch.uint8, device=DEV)
    P.llm_paged_attention(q, kc, vc, ks, vs, table, lens, scale, 0, out, ws)
    code = kc.transpose(1, 2).reshape(-1, d)[:n, 3].double()
    v = vc.transpose(1, 2).reshape(-1, d)[:n].double() * vs[0, 0, 0].double()
    for h, sign in ((0, 1.0), (1, -1.0)):
        w = torch.softmax(sign * scale * 4.0 * code, dim=0)
        want = w @ v
        # the output's rounding; logits of at most 64 in fp32 (two products of 2^-24 each), fp32 sums over n tokens, the two terms of a weight
        rel = 2.0 ** -8 + 4 * 64 * 2.0 ** -24 + 2.0 ** -23 * (n + 16) + 2.0 ** -20
        assert ((out[0, h].double() - want).abs() <= want.abs() * rel + n * 2.0 ** -34 * 127 * 0.01).all()
