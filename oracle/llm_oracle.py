"""Plain forms of the paged cache's operators (numpy, requests one by one, 64 bits)."""
import numpy as np

TINY = np.float32(2.0 ** -118)                      # FLT_MIN * 256: the smallest scale of an 8-bit row


def assign_pages(old, new, page, free, n_free, table, slot_capacity):
    """-> (table, slots, token_start, seq_lens, n_left): requests in order, pages from the top of the free stack; one
    whose rows do not all have a slot is not served (slot_capacity 0: no slots are asked for)."""
    table = np.array(table, dtype=np.int32)
    slots = np.full(slot_capacity, -1, dtype=np.int64)
    n_free = min(max(int(n_free), 0), len(free))
    start, lens, asked, left, row = [], [], 0, n_free, 0
    for b, (o, w) in enumerate(zip(old, new)):
        o, w = max(int(o), 0), max(int(w), 0)
        have, end = -(-o // page), -(-(o + w) // page)
        fits = end <= table.shape[1]
        need = end - have if fits else 0
        rows = w == 0 or slot_capacity == 0 or row + w <= min(slot_capacity, 2 ** 31 - 1)
        served = fits and rows and (need == 0 or asked + need <= n_free)
        start.append(min(row, 2 ** 31 - 1))
        if served:
            for i in range(need):
                table[b, have + i] = free[n_free - 1 - asked - i]
            left = min(left, n_free - asked - need) if need else left
            for i in range(w):
                if row + i < slot_capacity:
                    p = int(table[b, (o + i) // page])
                    slots[row + i] = p * page + (o + i) % page if p >= 0 else -1
        asked += need
        row += w
        lens.append(o + w if served else o)
    return table, slots, np.array(start + [min(row, 2 ** 31 - 1)], np.int32), np.array(lens, np.int32), left


def rows_sym(x):
    """8-bit codes and scales of rows (last axis) as the fp32 arithmetic of the definition gives them."""
    x = np.asarray(x, dtype=np.float32)
    top = np.abs(x).max(axis=-1)
    ok = np.isfinite(top) & np.isfinite(x).all(axis=-1)
    s = np.where(ok, np.maximum(np.where(ok, top, 0).astype(np.float32) * np.float32(1 / 127), TINY), np.float32(np.nan)).astype(np.float32)
    with np.errstate(invalid="ignore"):
        c = np.clip(np.rint(x / s[..., None]), -127, 127)
    return np.where(ok[..., None], c, 0).astype(np.int8), s


def attention(q, k, v, table, lens, scale, window, group):
    """q [batch, heads, d]; k, v [pages, kv_heads, page, d] as numbers.  -> (output, sum of weight * |v|, visible tokens,
    largest sum of |q k|): the last three for error bounds."""
    batch, heads, d = q.shape
    pages, _, page, _ = k.shape
    out, mag, seen = np.zeros((batch, heads, d)), np.zeros((batch, heads, d)), np.zeros(batch, dtype=int)
    qk = np.zeros((batch, heads))
    cap = table.shape[1] * page
    for b in range(batch):
        n = min(max(int(lens[b]), 0), cap)
        t = np.arange(max(0, n - window) if window else 0, n)
        ids = table[b][t // page] if len(t) else np.zeros(0, int)
        good = (ids >= 0) & (ids < pages)
        t, ids = t[good], ids[good]
        seen[b] = len(t)
        if not len(t):
            continue
        for h in range(heads):
            kk, vv = k[ids, h // group, t % page], v[ids, h // group, t % page]
            s = scale * (kk @ q[b, h])
            w = np.exp(s - s.max())
            w /= w.sum()
            out[b, h], mag[b, h] = w @ vv, w @ np.abs(vv)
            qk[b, h] = abs(scale) * (np.abs(kk) @ np.abs(q[b, h])).max()
    return out, mag, seen, qk
