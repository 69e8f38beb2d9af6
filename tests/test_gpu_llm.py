"""The paged key-value cache and the attention that reads it, on the GPU against the plain 64-bit forms."""
import numpy as np
import pytest
import torch

import paper_2505_20932_amd as P
from oracle import llm_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8}
I4, I8 = torch.int32, torch.int64


def _dev(a, dtype):
    return torch.tensor(np.asarray(a), dtype=dtype, device=DEV)


# ------------------------------------------------------------------------------------------ pages and slots
def _assign(old, new, page, free, n_free, table, cap):
    t = _dev(table, I4)
    outs = [torch.full((n,), -77, dtype=dt, device=DEV) for n, dt in ((cap, I8), (len(old) + 1, I4), (len(old), I4), (1, I4))]
    slots, start, lens, left = outs
    args = (_dev(old, I4), _dev(new, I4), page, _dev(free, I4), _dev([n_free], I4), t, slots, start, lens, left)
    P.llm_kv_assign_pages(*args)
    first = [x.cpu().numpy() for x in (t, slots, start, lens, left)]
    P.llm_kv_assign_pages(*args)                                  # again on the same inputs: the same
    for a, b in zip(first, (t, slots, start, lens, left)):
        assert np.array_equal(a, b.cpu().numpy())
    return first


def _compare(old, new, page, free, n_free, table, cap):
    got = _assign(old, new, page, free, n_free, table, cap)
    want = orc.assign_pages(old, new, page, free, n_free, table, cap)
    for name, g, w in zip(("table", "slots", "token_start", "seq_lens", "n_left"), got, want):
        assert np.array_equal(g.reshape(-1), np.asarray(w).reshape(-1)), name
    return want


@pytest.mark.parametrize("batch,page,longest,new", [(1, 16, 0, 1), (1, 16, 15, 1), (1, 1024, 5000, 3000), (7, 32, 100, 40), (64, 16, 900, 1),
                                                    (65, 64, 500, 257), (1000, 16, 300, 20), (1025, 128, 2000, 5), (8192, 16, 60, 3)])
@pytest.mark.parametrize("supply", ["plenty", "short", "none"])
def test_pages_and_slots(batch, page, longest, new, supply):
    rng = np.random.default_rng(batch + page + new)
    old, w = rng.integers(0, longest + 1, batch), rng.integers(0, new + 1, batch)
    cols = -(-(longest + new) // page) + 1
    have = -(-old // page)
    ids = rng.permutation(int(have.sum()) + batch * 2 * (new // page + 2)).astype(np.int32)
    table = np.full((batch, cols), -1, np.int32)
    at = 0
    for b in range(batch):
        table[b, :have[b]] = ids[at:at + have[b]]
        at += have[b]
    free = ids[at:]
    need = int((-(-(old + w) // page) - have).sum())
    n_free = {"plenty": len(free), "short": min(need // 2, len(free)), "none": 0}[supply]
    _compare(old, w, page, free, n_free, table, int(w.sum()) + 9)
    _compare(old, w, page, free, n_free, table, int(w.sum()) // 2)   # a token batch that is cut


def test_pages_hostile_lengths():
    """Negative and huge lengths, table rows that are too short, entries that are not pages, a stack counter out of range."""
    old = [-5, 2 ** 31 - 1, 40, 0, 33, 16, 2 ** 31 - 1, 5]
    new = [3, 2 ** 31 - 1, 8, -7, 2 ** 31 - 1, 16, 0, 4]
    table = np.arange(8 * 4).reshape(8, 4) + 100
    table[7, 0] = -3
    free = np.arange(20)
    for n_free in (20, 3, 1, 0, -4, 2 ** 31 - 1):
        want = _compare(old, new, 16, free, n_free, table, 50)
        assert want[2][-1] == 2 ** 31 - 1
    _compare([0] * 3, [0] * 3, 16, free, 20, table[:3], 0)           # nothing new, no slots at all


# ------------------------------------------------------------------------------------------ append
def _pool(pages, heads, page, d, cache, fill):
    shape = (pages, heads, page, d)
    if cache == "i8":
        return [torch.full(shape, fill, dtype=torch.int8, device=DEV) for _ in range(2)] + \
               [torch.full(shape[:3], float(fill), device=DEV) for _ in range(2)]
    return [torch.full(shape, float(fill), dtype=TYPES[cache], device=DEV) for _ in range(2)] + [None, None]


@pytest.mark.parametrize("tokens,heads,d,page", [(1, 1, 64, 16), (3, 8, 128, 16), (37, 5, 64, 32), (100, 3, 256, 128), (513, 8, 128, 64),
                                                 (5000, 2, 128, 16), (2049, 40, 128, 16)])
@pytest.mark.parametrize("t,cache", [("f16", "f16"), ("bf16", "bf16"), ("f16", "i8"), ("bf16", "i8")])
def test_append(tokens, heads, d, page, t, cache):
    g = torch.Generator(device=DEV).manual_seed(tokens + d)
    qkv = torch.randn(tokens, 3 * heads * d, generator=g, device=DEV)
    qkv[:, ::7] *= 30
    qkv[tokens // 2, heads * d:] = 0.0                               # a token of zeros
    if tokens > 3 and cache == "i8":
        qkv[1, heads * d + 5] = float("nan")
        qkv[2, 2 * heads * d + 1] = float("inf")
    qkv = qkv.to(TYPES[t])
    k, v = (qkv[:, i * heads * d:(i + 1) * heads * d].unflatten(1, (heads, d)) for i in (1, 2))
    pages = -(-tokens // page) + 2
    slots = torch.randperm(pages * page, generator=g, device=DEV)[:tokens]
    slots[::5] = -1
    if tokens > 7:
        slots[6] = pages * page                                      # behind the pool
        slots[7] = -2 ** 62
    kc, vc, ks, vs = _pool(pages, heads, page, d, cache, 3)
    P.llm_kv_append(k, v, slots, kc, vc, ks, vs)
    s = slots.cpu().numpy()
    live = np.flatnonzero((s >= 0) & (s < pages * page))
    pg, at = s[live] // page, s[live] % page
    for x, c, sc in ((k, kc, ks), (v, vc, vs)):
        x = x.float().cpu().numpy()[live]
        want = np.full(c.shape, 3, dtype=np.float32)
        if cache == "i8":
            codes, scale = orc.rows_sym(x)
            want_s = np.full(sc.shape, 3, dtype=np.float32)
            want[pg, :, at], want_s[pg, :, at] = codes, scale
            assert np.array_equal(sc.cpu().numpy(), want_s, equal_nan=True)
        else:
            want[pg, :, at] = x
        assert np.array_equal(c.float().cpu().numpy(), want)


# ------------------------------------------------------------------------------------------ attention
EPS = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _case(lens, page, heads, kv, d, t, cache, seed, cols=None, dirt=True):
    """A cache in which every place that is not a request's token holds NaN (8-bit: scale NaN)."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    counts = [-(-n // page) for n in lens]
    pages = sum(counts) + 2
    ids = rng.permutation(pages)[:sum(counts)]
    cols = cols or max(1, max(counts))
    table = np.full((len(lens), cols), -1, np.int32)
    live = torch.zeros(pages, page, dtype=torch.bool, device=DEV)
    at = 0
    for b, n in enumerate(lens):
        table[b, :counts[b]] = ids[at:at + counts[b]]
        for i, p in enumerate(ids[at:at + counts[b]]):
            live[p, :min(page, n - i * page)] = True
        at += counts[b]
    shape = (pages, kv, page, d)
    dead = ~live[:, None, :].expand(pages, kv, page)
    out = []
    for _ in range(2):
        if cache == "i8":
            c = torch.randint(-127, 128, shape, dtype=torch.int8, device=DEV, generator=g)
            s = torch.exp2(torch.randint(-12, 3, shape[:3], device=DEV, generator=g).float()) * (1 + torch.rand(shape[:3], device=DEV, generator=g))
            s = s * (0.02 if len(out) == 0 else 1.0)
            out.append((c, torch.where(dead, float("nan") if dirt else 1.0, s)))
        else:
            c = torch.randn(shape, device=DEV, generator=g)
            out.append((torch.where(dead[..., None], float("nan") if dirt else 1.0, c).to(TYPES[cache]), None))
    q = torch.randn(len(lens), heads, d, device=DEV, generator=g).to(TYPES[t])
    return q, out[0][0], out[1][0], out[0][1], out[1][1], _dev(table, I4), _dev(lens, I4)


def _numbers(c, s):
    x = c.double() if s is None else c.double() * s.double()[..., None]
    return x.cpu().numpy()


def _run(q, k, v, ks, vs, table, lens, scale, window, page):
    batch, heads, d = q.shape
    out = torch.full_like(q, 9.0)
    ws = torch.full((P.llm_paged_attention_workspace(batch, heads, k.shape[1], d, table.shape[1], page),), 0xff,
                    dtype=torch.uint8, device=DEV)
    P.llm_paged_attention(q, k, v, ks, vs, table, lens, scale, window, out, ws)
    return out


def _check(out, q, k, v, ks, vs, table, lens, scale, window, t):
    """Bound of the error: the output's rounding; a weight's (two binary16 terms that are cut off: 2^-10 of 2^-10, and binary16's smallest
    step next to the largest weight 1; two bfloat16 terms: 2^-16); the logits' fp32 sums, products and exponential, which enter a weight
    relatively and both sums; fp32 sums over the tokens.  All of them times sum w |v|, the smallest step times max |v|.
    8-bit caches: weights are binary16 for either type, and bfloat16 queries become binary16 relative to 2^e <= 2 max |q|, each off by
    at most half its smallest step, 2^-25 * 2^e."""
    kn, vn = _numbers(k, ks), _numbers(v, vs)
    d = q.shape[2]
    want, mag, seen, qk = orc.attention(q.double().cpu().numpy(), kn, vn, table.cpu().numpy(), lens.cpu().numpy(), scale, window,
                                        q.shape[1] // k.shape[1])
    weight = 2.0 ** -20 if t == "f16" or k.dtype == torch.int8 else 2.0 ** -16
    logit = (d / 16 + 8) * 2.0 ** -23 * (qk + 1.0)
    half = t == "f16" or k.dtype == torch.int8
    if t == "bf16" and half:
        logit = logit + d * 2.0 ** -24 * float(q.abs().max()) * np.nan_to_num(np.abs(kn)).max() * abs(scale)
    rel = weight + 2 * logit + 2.0 ** -23 * (seen[:, None] + 16)
    vmax = np.nan_to_num(np.abs(vn)).max()
    tol = EPS[t] * np.abs(want) + rel[..., None] * mag * 1.01 + (seen[:, None, None] * 2.0 ** -24 * vmax if half else 0.0) + \
        (2.0 ** -25 if t == "f16" else 0.0)
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    err = np.abs(got - want)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())
    assert (got[seen == 0] == 0).all()


SHAPES = [
    # lens, page, q heads, kv heads, d, window
    ([1], 16, 1, 1, 64, 0), ([0], 16, 4, 2, 128, 0), ([17], 16, 8, 8, 128, 0), ([31, 32, 33, 0, 1], 32, 6, 2, 64, 0),
    ([700], 16, 32, 32, 128, 0), ([129, 5, 1000], 128, 28, 4, 128, 0), ([513, 2, 64], 64, 16, 1, 256, 0),
    ([300, 77], 16, 34, 2, 64, 0), ([40, 0, 255, 256, 257], 256, 48, 1, 128, 0), ([3000, 1, 1777], 16, 32, 8, 128, 0),
    ([5000], 1024, 8, 1, 256, 0), ([9000, 8999], 16, 4, 4, 64, 0),
    ([100, 1000, 7], 16, 8, 2, 128, 1), ([100, 1000, 7, 33, 64], 32, 8, 2, 128, 33), ([2500, 4097], 16, 7, 1, 128, 1000),
    ([65, 66, 67], 64, 4, 2, 256, 64), ([20000], 16, 2, 1, 128, 5),
]


@pytest.mark.parametrize("lens,page,heads,kv,d,window", SHAPES)
@pytest.mark.parametrize("t,cache", [("f16", "f16"), ("bf16", "bf16"), ("f16", "i8"), ("bf16", "i8")])
def test_attention(lens, page, heads, kv, d, window, t, cache):
    c = _case(lens, page, heads, kv, d, t, cache, sum(lens) + heads)
    scale = d ** -0.5
    out = _run(*c, scale, window, page)
    _check(out, *c, scale, window, t)
    assert torch.equal(out, _run(*c, scale, window, page))            # bit for bit the same again


@pytest.mark.parametrize("t,cache", [("f16", "f16"), ("bf16", "i8")])
def test_attention_sees_nothing_else(t, cache):
    """A wider table, lengths beyond it, entries that are no pages: left out; a request's result does not depend on the
    other requests."""
    lens = [200, 1, 90, 0, 333]
    q, k, v, ks, vs, table, n = _case(lens, 16, 8, 2, 128, t, cache, 3, cols=40)
    scale = 0.09
    base = _run(q, k, v, ks, vs, table, n, scale, 0, 16)
    _check(base, q, k, v, ks, vs, table, n, scale, 0, t)
    bad = table.clone()
    bad[0, 3], bad[0, 7], bad[2, 0], bad[4, 20] = -1, k.shape[0], 2 ** 31 - 1, -2 ** 31
    out = _run(q, k, v, ks, vs, bad, n, scale, 0, 16)
    _check(out, q, k, v, ks, vs, bad, n, scale, 0, t)
    assert torch.equal(out[1], base[1]) and (out[3] == 0).all()
    none = torch.full_like(table, -9)
    assert (_run(q, k, v, ks, vs, none, n, scale, 0, 16) == 0).all()
    # lengths beyond the table are cut, negative ones are none
    long = n.clone()
    long[1], long[3] = -5, 0
    cut = table[:, :5].contiguous()
    out = _run(q, k, v, ks, vs, cut, long, scale, 0, 16)
    _check(out, q, k, v, ks, vs, cut, long, scale, 0, t)
    # the requests alone, with the same table width and batch: other lengths elsewhere do not matter
    alone = n.clone()
    alone[:4] = 0
    assert torch.equal(_run(q, k, v, ks, vs, table, alone, scale, 0, 16)[4], base[4])


@pytest.mark.parametrize("t,cache", [("f16", "f16"), ("bf16", "bf16"), ("f16", "i8")])
def test_attention_of_hard_logits(t, cache):
    """Maxima that arrive late and early, equal logits, a scale of zero and a negative one; strided queries and outputs."""
    lens = [1500, 700]
    q, k, v, ks, vs, table, n = _case(lens, 32, 8, 2, 64, t, cache, 11)
    if cache != "i8":
        for b, at in ((0, 1499), (1, 0)):
            k[int(table[b, at // 32]), :, at % 32] = 6 * q[b, 0]
    for scale in (1.0, 0.0, -0.3):
        wide = torch.full((2, 8 * 64 * 3), 5.0, dtype=q.dtype, device=DEV)
        qs = wide[:, 512:1024].unflatten(1, (8, 64))
        qs.copy_(q)
        os = wide[:, 1024:].unflatten(1, (8, 64))
        ws = torch.empty(P.llm_paged_attention_workspace(2, 8, 2, 64, table.shape[1], 32), dtype=torch.uint8, device=DEV)
        P.llm_paged_attention(qs, k, v, ks, vs, table, n, scale, 0, os, ws)
        _check(os, q, k, v, ks, vs, table, n, scale, 0, t)
        assert (wide[:, :512] == 5.0).all()


def test_cache_beyond_32_bit_offsets():
    """Pages whose values and scales lie more than 2^32 bytes into the pool."""
    page, kv, d = 1024, 32, 256                       # 16 MiB of binary16 per page
    pages = 270
    k = torch.zeros(pages, kv, page, d, dtype=torch.float16, device=DEV)
    v = torch.zeros_like(k)
    n = 5
    g = torch.Generator(device=DEV).manual_seed(1)
    rows = torch.randn(n, 2, kv, d, generator=g, device=DEV).half()
    last = pages - 1
    slots = torch.arange(n, device=DEV, dtype=I8) + last * page + 7
    P.llm_kv_append(rows[:, 0].contiguous(), rows[:, 1].contiguous(), slots, k, v)
    assert torch.equal(k[last, :, 7:7 + n].transpose(0, 1), rows[:, 0]) and int(k.count_nonzero()) == int(rows[:, 0].count_nonzero())
    q = torch.randn(1, kv, d, generator=g, device=DEV).half()
    table = _dev([[last]], I4)
    lens = _dev([7 + n], I4)
    out = _run(q, k, v, None, None, table, lens, 0.05, n, page)
    sub_k, sub_v = k[last:].contiguous(), v[last:].contiguous()
    _check(out, q, sub_k, sub_v, None, None, _dev([[0]], I4), lens, 0.05, n, "f16")


def test_decoding_steps_run_together():
    """Steps of an attention sub-layer as a program runs them: 4-bit qkv layer, pages, append, attention, 4-bit output layer; the
    captured step replayed while the requests grow, against the plain forms on the same codes."""
    torch.manual_seed(5)
    batch, heads, kv, d, page, width = 5, 8, 2, 64, 16, 512
    steps = 21
    g = torch.Generator(device=DEV).manual_seed(2)
    wq = torch.randn((heads + 2 * kv) * d, width, generator=g, device=DEV) * width ** -0.5
    wo = torch.randn(width, heads * d, generator=g, device=DEV) * (heads * d) ** -0.5

    def mx4(rows, k):
        return (torch.empty(rows, k // 2, dtype=torch.uint8, device=DEV), torch.empty(-(-k // 256), rows, 8, dtype=torch.uint8, device=DEV))
    qc, oc = mx4(*wq.shape), mx4(*wo.shape)
    P.cwac_mx4_quantize(wq, *qc)
    P.cwac_mx4_quantize(wo, *oc)
    x = torch.empty(batch, width, dtype=torch.float16, device=DEV)
    xc, ac = mx4(batch, width), mx4(batch, heads * d)
    qkv = torch.empty(batch, wq.shape[0], dtype=torch.float16, device=DEV)
    attn = torch.empty(batch, heads, d, dtype=torch.float16, device=DEV)
    y = torch.empty(batch, width, dtype=torch.float16, device=DEV)
    cols = 4
    kc, vc, _, _ = _pool(batch * cols, kv, page, d, "f16", 0)
    kc.fill_(float("nan"))
    vc.fill_(float("nan"))
    old, lens = torch.tensor([0, 3, 15, 16, 40], dtype=I4, device=DEV), torch.empty(batch, dtype=I4, device=DEV)
    new = torch.ones(batch, dtype=I4, device=DEV)
    table = torch.full((batch, cols), -1, dtype=I4, device=DEV)
    free = torch.randperm(batch * cols, generator=g, device=DEV).to(I4)
    n_free, left = _dev([batch * cols], I4), torch.empty(1, dtype=I4, device=DEV)
    start, slots = torch.empty(batch + 1, dtype=I4, device=DEV), torch.empty(64, dtype=I8, device=DEV)
    # the tokens that are there already
    past = old.clone()
    P.llm_kv_assign_pages(torch.zeros_like(old), past, page, free, n_free, table, slots.new_empty(200), start, lens, left)
    n_free.copy_(left)
    hist = {b: [] for b in range(batch)}
    first = torch.randn(int(past.sum()), 2, kv, d, generator=g, device=DEV).half()
    s200 = torch.empty(200, dtype=I8, device=DEV)
    P.llm_kv_assign_pages(torch.zeros_like(old), past, page, free, _dev([batch * cols], I4), table, s200, start, lens, left)
    P.llm_kv_append(first[:, 0].contiguous(), first[:, 1].contiguous(), s200[:first.shape[0]].contiguous(), kc, vc)
    at = 0
    for b, c in enumerate(past.tolist()):
        hist[b] = [first[at + i] for i in range(c)]
        at += c
    ws = torch.empty(P.llm_paged_attention_workspace(batch, heads, kv, d, cols, page), dtype=torch.uint8, device=DEV)

    def step():
        P.cwac_mx4_quantize(x, *xc)
        P.qlinear_mx4_cwac_forward(*xc, *qc, None, None, qkv)
        P.llm_kv_assign_pages(old, new, page, free, n_free, table, slots, start, lens, left)
        k = qkv[:, heads * d:(heads + kv) * d].unflatten(1, (kv, d))
        v = qkv[:, (heads + kv) * d:].unflatten(1, (kv, d))
        P.llm_kv_append(k, v, slots[:batch], kc, vc)
        P.llm_paged_attention(qkv[:, :heads * d].unflatten(1, (heads, d)), kc, vc, None, None, table, lens, d ** -0.5, 0, attn, ws)
        P.cwac_mx4_quantize(attn.view(batch, heads * d), *ac)
        P.qlinear_mx4_cwac_forward(*ac, *oc, None, None, y)
        old.copy_(lens)
        n_free.copy_(left)

    def check(i):
        want = np.zeros((batch, heads, d))
        q64 = qkv.double().cpu().numpy()
        for b in range(batch):
            row = qkv[b, heads * d:].view(2, kv, d).clone()
            if len(hist[b]) < cols * page:
                hist[b].append(row)
            kk = torch.stack([h[0] for h in hist[b]]).double().cpu().numpy()
            vv = torch.stack([h[1] for h in hist[b]]).double().cpu().numpy()
            for h in range(heads):
                s = kk[:, h // (heads // kv)] @ q64[b, h * d:(h + 1) * d] * d ** -0.5
                w = np.exp(s - s.max())
                want[b, h] = (w / w.sum()) @ vv[:, h // (heads // kv)]
        # rounding of the output and of the weights, values below 8: 2^-11 each, next to it fp32 arithmetic
        assert np.abs(attn.double().cpu().numpy() - want).max() <= 2 * 2.0 ** -11 * 8 + 1e-4, i
        assert lens.tolist() == [len(hist[b]) for b in range(batch)]
        v = torch.empty(batch, heads * d, dtype=torch.float64, device=DEV)
        f = torch.empty(batch, heads * d, device=DEV)
        P.cwac_mx4_dequantize(*ac, f)
        wv = torch.empty(wo.shape, device=DEV)
        P.cwac_mx4_dequantize(*oc, wv)
        ref = f.double() @ wv.double().t()
        bound = f.double().abs() @ wv.double().abs().t()
        assert ((y.double() - ref).abs() <= 2.0 ** -11 * ref.abs() + 20 * 2.0 ** -23 * bound + 2.0 ** -25).all()

    for i in range(3):
        x.copy_(torch.randn(batch, width, generator=g, device=DEV))
        step()
        check(i)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    for i in range(3, steps):
        x.copy_(torch.randn(batch, width, generator=g, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        check(i)
