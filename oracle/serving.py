"""Float64 oracle of the serving path: packed sequences, a paged cache, rows of 8-bit floats (test infrastructure only)."""
import numpy as np


def round_e4m3(x: np.ndarray) -> np.ndarray:
    """Nearest value, ties to even, of 1 sign, 4 exponent (bias 7) and 3 mantissa bits; |x| <= 448; values that are not finite give NaN."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x)
    y = np.where(fine, x, 0.0)
    _, e = np.frexp(y)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.where(fine, np.rint(y / step) * step, np.nan)


def quantise_rows(x: np.ndarray):
    """Rows (last axis) -> (values of the codes, biased exponents): the smallest power of two from 2^-127 on that brings the finite
    elements into ±448."""
    x = np.asarray(x, dtype=np.float64)
    top = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    e = np.full(top.shape, -127)
    while True:
        over = top > 448.0 * np.exp2(e.astype(np.float64))
        if not over.any():
            break
        e = e + over
    return round_e4m3(np.where(np.isfinite(x), x, np.nan) / np.exp2(e.astype(np.float64))[..., None]), e + 127


def dequantise_rows(codes: np.ndarray, scale: np.ndarray) -> np.ndarray:
    return codes * np.exp2(np.asarray(scale, dtype=np.float64) - 127.0)[..., None]


def bounds(offsets, tokens):
    """(first token, number of tokens) of every sequence."""
    o = np.clip(np.asarray(offsets, dtype=np.int64), 0, tokens)
    return [(int(a), int(max(b - a, 0))) for a, b in zip(o[:-1], o[1:])]


def place(table_row, position, page_size, n_pages):
    """(page, slot) of a position, or None."""
    if position < 0 or position >= len(table_row) * page_size:
        return None
    page = int(table_row[position // page_size])
    return (page, position % page_size) if 0 <= page < n_pages else None


def new_places(table, length, offsets, tokens, page_size, n_pages):
    """[(token, page, slot)] of every new token that has a place."""
    got = []
    for s, (first, n) in enumerate(bounds(offsets, tokens)):
        for i in range(n):
            p = place(table[s], max(int(length[s]), 0) - n + i, page_size, n_pages)
            if p is not None:
                got.append((first + i, *p))
    return got


def attend(q, k, v, seen, scale):
    """One head: q [n, d], k, v [m, d], seen [n, m] -> (O, Σ p·|v|, largest Σ |q·k|, largest |score|); a row that sees nothing is zero.
    Keys that no query sees may hold anything."""
    n, m = seen.shape
    O, A = np.zeros((n, q.shape[1])), np.zeros((n, q.shape[1]))
    reach, top = np.zeros(n), np.zeros(n)
    for i in range(n):
        j = np.nonzero(seen[i])[0]
        if not len(j):
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            s = (k[j] @ q[i]) * scale
            big = s.max()
            if big == -np.inf:
                continue
            p = np.exp(s - big)
            p = p / p.sum()
            O[i], A[i] = p @ v[j], p @ np.abs(v[j])
            reach[i], top[i] = (np.abs(k[j]) @ np.abs(q[i])).max() * abs(scale), np.abs(s).max()
    return O, A, reach, top


def attention(Q, keys, values, offsets, length, causal, scale, present=None):
    """Q [tokens, heads, d]; keys[s], values[s] [m_s, kv_heads, d]; length[s] positions of sequence s (its new tokens are the last);
    present[s] [m_s] bool.  -> (O, A, reach, top) as in attend, None rows (outside every sequence) as NaN in O."""
    tokens, heads, d = Q.shape
    O = np.full((tokens, heads, d), np.nan)
    A, reach, top = np.zeros_like(O), np.zeros((tokens, heads)), np.zeros((tokens, heads))
    scale = scale if scale > 0 else 1.0 / np.sqrt(d)
    for s, (first, n) in enumerate(bounds(offsets, tokens)):
        if not n:
            continue
        m, hk = keys[s].shape[:2]
        g = heads // hk
        pos = length[s] - n + np.arange(n)
        seen = np.ones((n, m), dtype=bool) if present is None else np.broadcast_to(present[s], (n, m)).copy()
        if causal:
            seen &= np.arange(m)[None] <= pos[:, None]
        for h in range(heads):
            r = attend(Q[first:first + n, h], keys[s][:, h // g], values[s][:, h // g], seen, scale)
            O[first:first + n, h], A[first:first + n, h], reach[first:first + n, h], top[first:first + n, h] = r
    return O, A, reach, top


def gather(pages, scale, table_row, length):
    """What one sequence sees: ([m, kv_heads, d], present [m])."""
    n_pages, hk, ps, d = pages.shape
    m = int(min(max(int(length), 0), len(table_row) * ps))
    rows, present = np.zeros((m, hk, d)), np.zeros(m, dtype=bool)
    for j in range(m):
        p = place(table_row, j, ps, n_pages)
        if p is not None:
            rows[j] = pages[p[0], :, p[1]] if scale is None else dequantise_rows(pages[p[0], :, p[1]], scale[p[0], :, p[1]])
            present[j] = True
    return rows, present
