"""CPU float64 oracle of the operators in front of a Test-Time Control block: rotary positions, the cache of 4-bit codes, attention
over it.  Plain numpy from the definitions; shares no code with the GPU path.

A cache is handed over as the bytes that the library keeps (pages, heads, page * (d + d / 16)); `tokens` reads them by the layout
that the C header documents.
"""
import numpy as np

BLOCK = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rope_table(rows, freqs, scale=1.0):
    """(rows, pairs, 2) float64"""
    angle = np.arange(rows, dtype=np.float64)[:, None] * np.asarray(freqs, dtype=np.float64)
    return scale * np.stack([np.cos(angle), np.sin(angle)], -1)


def rope(x, positions, table, layout="half", backward=False):
    """Rotation of the first 2 * table.shape[1] entries of each head of x (tokens, heads, d) by its matrix, pair by pair."""
    y = np.array(x, dtype=np.float64)
    half = table.shape[1]
    for t, p in enumerate(positions):
        for i in range(half):
            a, b = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
            if not 0 <= p < table.shape[0]:
                y[t, :, [a, b]] = np.nan
                continue
            c, s = (float(v) for v in table[p, i])
            m = np.array([[c, -s], [s, c]])
            m = m.T if backward else m
            y[t][:, [a, b]] = np.asarray(x, dtype=np.float64)[t][:, [a, b]] @ m.T
    return y


def quantise(x):
    """(codes, exponents) of the blocks of 32 of the last axis: codes 0 .. 15, exponent bytes 0 .. 255."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    top = np.abs(b).max(-1)
    f, k = np.frexp(np.where(np.isfinite(top), top, 1.0))   # top = f * 2^k, 1/2 <= f < 1
    e = np.where(f >= 0.875, k, k - 1) - 2 + 127
    e = np.where(top == 0, 0, np.clip(e, 0, 252))
    e = np.where(np.isfinite(top), e, 255)
    y = np.where((e == 255)[..., None], 0.0, b / np.exp2(e - 127.0)[..., None])
    gap = np.abs(np.abs(y)[..., None] - MAGNITUDES)
    best = gap.min(-1, keepdims=True)
    near = gap == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = code | (np.signbit(b) << 3)
    return code.reshape(x.shape).astype(np.uint8), e.astype(np.uint8)


def numbers(codes, exponents):
    """float64 numbers of codes (.., d) and exponent bytes (.., d / 32)"""
    v = MAGNITUDES[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    scale = np.where(exponents > 252, np.nan, np.exp2(exponents.astype(np.float64) - 127.0))
    return v * np.repeat(scale, BLOCK, -1)


def parts(cache, d):
    """(key codes, value codes, key exponents, value exponents) of a cache's bytes, each (pages, heads, page, ..) in token order"""
    pages, heads, n = cache.shape
    page = n // (d + d // 16)
    c, e = page * d // 2, page * d // BLOCK

    def codes(b):
        return np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], -1)

    keys = cache[..., :c].reshape(pages, heads, page, d // 2)
    values = cache[..., c:2 * c].reshape(pages, heads, page // 4, 16, 4, d // 32).transpose(0, 1, 2, 4, 3, 5).reshape(pages, heads, page, d // 2)
    ke = cache[..., 2 * c:2 * c + e].reshape(pages, heads, page, d // BLOCK)
    ve = cache[..., 2 * c + e:].reshape(pages, heads, page // 4, d // BLOCK, 4).transpose(0, 1, 2, 4, 3).reshape(pages, heads, page, d // BLOCK)
    return codes(keys), codes(values), ke, ve


def tokens(cache, d):
    """(keys, values) of every slot, (pages * page, heads, d) float64"""
    kc, vc, ke, ve = parts(cache, d)
    k, v = numbers(kc, ke), numbers(vc, ve)
    return (x.transpose(0, 2, 1, 3).reshape(-1, cache.shape[1], d) for x in (k, v))


def attention(q, k, v, block_table, kv_len, cu_q, page, pages, scale, causal=True, window=0):
    """out, lse, and how much the rounding of a weight can move each entry of out: sum of weight * |value|.  k, v by slot."""
    n, heads_q, d = q.shape
    heads = k.shape[1]
    group = heads_q // heads
    out, size = np.zeros((n, heads_q, d)), np.zeros((n, heads_q, d))
    lse = np.full((n, heads_q), -np.inf)
    for s, length in enumerate(kv_len):
        new = cu_q[s + 1] - cu_q[s]
        j = np.arange(length)
        at = block_table[s][j // page].astype(np.int64)
        there = (at >= 0) & (at < pages)
        slot = np.where(there, at, 0) * page + j % page
        for i in range(new):
            p = length - new + i
            seen = there & (j <= p) if causal else there
            if window:
                seen = seen & (j > p - window)
            rows = slot[seen]
            if not len(rows):
                continue
            for h in range(heads_q):
                z = scale * (k[rows, h // group] @ q[cu_q[s] + i, h])
                top = z.max()
                w = np.exp(z - top)
                total = w.sum()
                lse[cu_q[s] + i, h] = top + np.log(total)
                out[cu_q[s] + i, h] = (w / total) @ v[rows, h // group]
                size[cu_q[s] + i, h] = (w / total) @ np.abs(v[rows, h // group])
    return out, lse, size
