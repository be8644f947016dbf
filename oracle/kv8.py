"""The 8-bit KV pool and the page operations, written out plainly (test infrastructure only).

Format (this library's own, restated here independently): a (layer, page) is a run of bytes,
[K, V][kv head][16 * D] e4m3 codes, then [K, V][kv head] float32 scales.  Inside a block (token t of the
page, feature d) the code's byte is
    K:  ((d // 16) * 16 + t) * 16 + d % 16
    V:  (((d // 64) * 4 + t // 4) * 16 + d % 16) * 16 + ((d // 16) % 4) * 4 + t % 4
and the value is code * scale.  Pools here are numpy uint8 [layers][pages][page stride].

e4m3: 1 sign, 4 exponent (bias 7), 3 mantissa bits, no infinities; 0x7f and 0xff are not numbers.
"""
import numpy as np

PAGE = 16
LEAST = -100              # exponent of the smallest scale
MOST_CODE = 448.0
MOST_HALF = 61440.0       # largest multiple of an e4m3 value that half precision holds
MOST_BF16 = 240 * 2.0 ** 120      # and bf16


def _table():
    v = np.empty(256)
    for c in range(128):
        e, m = c >> 3, c & 7
        v[c] = np.nan if c == 127 else (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    v[128:] = -v[:128]
    return v


VALUES = _table()


def encode(x):
    """Codes (uint8) of float64 values: nearest, ties to the even mantissa; beyond 448 the largest code."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), MOST_CODE)
    pos = VALUES[:127]
    hi = np.clip(np.searchsorted(pos, np.where(np.isnan(a), 0.0, a)), 1, 126)      # pos[hi - 1] < a <= pos[hi]
    lo = hi - 1
    down, up = a - pos[lo], pos[hi] - a
    c = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    c = np.where(np.isnan(x), 127, c)
    return (c | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def k_index(t, d):
    t, d = np.asarray(t), np.asarray(d)
    return ((d // 16) * 16 + t) * 16 + d % 16


def v_index(t, d):
    t, d = np.asarray(t), np.asarray(d)
    return (((d // 64) * 4 + t // 4) * 16 + d % 16) * 16 + ((d // 16) % 4) * 4 + t % 4


def page_bytes(Hkv, D):
    return -(-2 * Hkv * (PAGE * D + 4) // 16) * 16


def block(pool, layer, page, kv, h, Hkv, D):
    """(codes of one block, its scale as an array of one): views."""
    row = pool[layer, page]
    o = (kv * Hkv + h) * PAGE * D
    s = 2 * Hkv * PAGE * D + (kv * Hkv + h) * 4
    return row[o:o + PAGE * D], row[s:s + 4].view(np.float32)


def exponent_for(top):
    """Least e >= LEAST with top <= 448 * 2**e."""
    e = LEAST
    if top > 0:
        e = max(LEAST, int(np.floor(np.log2(top))) - 10)
        while top > MOST_CODE * 2.0 ** e:
            e += 1
    return e


def ref_append(pool, layer, tables, ctx_lens, cu_q_lens, k_new, v_new, Hkv, D, half=False):
    """The append, page by page: k_new, v_new float [T, Hkv, D].  In place.  Pages outside the pool are skipped."""
    d = np.arange(D)
    for s in range(len(ctx_lens)):
        c, q, t0 = int(ctx_lens[s]), int(cu_q_lens[s + 1] - cu_q_lens[s]), int(cu_q_lens[s])
        for j in range(c // PAGE, -(-(c + q) // PAGE) if q else 0):
            page = int(tables[s][j])
            if not 0 <= page < pool.shape[1]:
                continue
            lo, hi = max(c, j * PAGE), min(c + q, j * PAGE + PAGE)
            held = max(0, min(c - j * PAGE, PAGE))
            for kv, (rows, index) in enumerate(((k_new, k_index), (v_new, v_index))):
                for h in range(Hkv):
                    codes, scale = block(pool, layer, page, kv, h, Hkv, D)
                    x = np.asarray(rows[t0 + lo - c:t0 + hi - c, h], np.float64)
                    if half:
                        x = np.clip(x, -MOST_HALF, MOST_HALF)
                    else:                                             # (infinities do not count, and end at the largest value in reach)
                        x = np.where(np.isinf(x), x, np.clip(x, -MOST_BF16, MOST_BF16))
                    size = np.abs(x[np.isfinite(x)])
                    e = exponent_for(size.max() if size.size else 0.0)
                    if held:
                        before = int(np.log2(scale[0]))
                        if e > before:
                            at = index(np.arange(held)[:, None], d)
                            codes[at] = encode(VALUES[codes[at]] * 2.0 ** (before - e))
                        e = max(e, before)
                    if not half:
                        x = np.clip(x, -MOST_BF16, MOST_BF16)
                    codes[index(np.arange(lo, hi)[:, None] - j * PAGE, d)] = encode(x * 2.0 ** -e)
                    scale[0] = 2.0 ** e
    return pool


def read_logical(pool, layer, table_row, n, Hkv, D):
    """K, V (float64 [n, Hkv, D]) of a sequence of n tokens."""
    out = np.empty((2, -(-n // PAGE) * PAGE, Hkv, D))
    t, d = np.arange(PAGE)[:, None], np.arange(D)
    for b in range(-(-n // PAGE)):
        for kv, index in enumerate((k_index, v_index)):
            for h in range(Hkv):
                codes, scale = block(pool, layer, int(table_row[b]), kv, h, Hkv, D)
                out[kv, b * PAGE:(b + 1) * PAGE, h] = VALUES[codes[index(t, d)]] * np.float64(scale[0])
    return out[0, :n], out[1, :n]


def attention(q, K, V, ctx, scale):
    """fp64 softmax attention of q [n, Hq, D] at positions ctx .. ctx + n - 1 over K, V [ctx + n, Hkv, D]: (out, spread), spread
    [n, Hq, D] = sum_j w_j |V_j - out| -- what a relative error of the weights is multiplied by -- and reach [n, Hq] =
    scale * max_j sum_d |q_d K_jd|, the size of what a score is summed from."""
    n, Hq, D = q.shape
    G = Hq // K.shape[1]
    out, spread, reach = np.empty((n, Hq, D)), np.empty((n, Hq, D)), np.empty((n, Hq))
    for h in range(Hq):
        k, v = K[:, h // G], V[:, h // G]
        for i in range(n):
            m = ctx + i + 1
            s = scale * (k[:m] @ q[i, h])
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ v[:m]
            spread[i, h] = w @ np.abs(v[:m] - out[i, h])
            reach[i, h] = scale * (np.abs(k[:m]) @ np.abs(q[i, h])).max()
    return out, spread, reach


def ref_fork(pool, l0, l1, tables, lens, counts, parents, children, fresh, page_size=PAGE):
    """In place; pool [layers][pages][bytes]."""
    for p, c, f in zip(parents, children, fresh):
        n = int(lens[p])
        full = n // page_size
        row = np.full(tables.shape[1], -1, np.int32)
        row[:full] = tables[p, :full]
        counts[row[:full]] += 1                                       # (a row holds a page once)
        if n % page_size:
            row[full] = f
            counts[f] = 1
            pool[l0:l1, f] = pool[l0:l1, tables[p, full]]
        tables[c] = row
        lens[c] = n


def ref_free(tables, lens, counts, rows, page_size=PAGE):
    """In place; returns the freed pages, ascending."""
    gone = set()
    for r in rows:
        for e in range(-(-int(lens[r]) // page_size)):
            p = int(tables[r, e])
            counts[p] -= 1
            if counts[p] == 0:
                gone.add(p)
            tables[r, e] = -1
        lens[r] = 0
    return sorted(gone)


def ref_compact(pool, l0, l1, tables, lens, counts, page_size=PAGE):
    """(new tables, new counts, new ids, pages used); the pool in place."""
    used = np.flatnonzero(counts > 0)
    n = len(used)
    ids = np.full(len(counts), -1, np.int32)
    ids[used] = used
    holes = [p for p in range(n) if counts[p] <= 0]
    movers = [int(p) for p in used if p >= n]
    for a, b in zip(movers, holes):
        ids[a] = b
        pool[l0:l1, b] = pool[l0:l1, a]
    new_counts = np.zeros_like(counts)
    new_counts[ids[used]] = counts[used]
    new_tables = np.full_like(tables, -1)
    for r in range(len(lens)):
        for e in range(-(-int(lens[r]) // page_size)):
            p = int(tables[r, e])
            new_tables[r, e] = ids[p] if 0 <= p < len(counts) else -1
    return new_tables, new_counts, ids, n
