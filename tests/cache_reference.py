"""The operators of a paged cache of keys and values in 64 bits, from their definition (numpy; the oracle compresses)."""
import numpy as np

import oracle


def normed_and_turned(x, weight, eps, table, positions, interleaved):
    """x float64 [tokens, heads, dim] -> float64: norm per row, then the rotation of the first 2 * half elements."""
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight.astype(np.float64)
    if table is None:
        return x
    half = table.shape[2]
    inside = (positions >= 0) & (positions < table.shape[0])
    rows = table[np.where(inside, positions, 0)].astype(np.float64)
    c, s = rows[:, 0][:, None], rows[:, 1][:, None]
    y = x.copy()
    ia, ib = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if interleaved else (np.arange(half), np.arange(half, 2 * half))
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    y[~inside] = np.nan
    return y


def append(kind, cache, k, v, slots, q=None, q_weight=None, k_weight=None, eps=1e-6, table=None, positions=None, interleaved=False):
    """cache = (codes uint8 [2, pages, heads, page, dim], scales) is changed; returns the queries in float64."""
    codes, scales = cache
    page, dim = codes.shape[3], codes.shape[4]
    turned = normed_and_turned(k.astype(np.float64), k_weight, eps, table, positions, interleaved).astype(np.float32)
    for t, slot in enumerate(slots):
        if not 0 <= slot < codes.shape[1] * page or (table is not None and not 0 <= positions[t] < table.shape[0]):
            continue
        for part, rows in enumerate((turned[t], v[t].astype(np.float32))):
            for h in range(codes.shape[2]):
                at = (part, slot // page, h, slot % page)
                if np.isfinite(rows[h]).all():
                    c, s = oracle.encode(kind, np.ascontiguousarray(rows[h]), dim)
                    codes[at], scales[at] = c, s[0]
                else:
                    scales[at] = np.nan  # whatever the codes are, the row stands for NaN
    return None if q is None else normed_and_turned(q.astype(np.float64), q_weight, eps, table, positions, interleaved)


def attention(kind, cache, q, pages, lens, starts, softmax_scale, window=0):
    """(out, tolerance) float64 [tokens, heads, dim]; rows of no sequence are NaN in both.  The tolerance, without the rounding of the
    output, is what the operator's documentation allows.  With u = 2^-11, half a step of binary16, relative:
      an element of a key is off by u at most (a query of 11 bits or fewer not at all), so a score by u scale sum |q_d k_jd| <= E, E the largest of
      the row, and sums in binary32 add less than (dim + 8) 2^-24 of the same;
      a weight over the sum of weights is off by 2 E' relative, E' = E and those sums, to first order, and by u for its rounding;
      a value by u: |out - exact| <= sum_j w_j |v_j| (2 u + 2 E' + (8 + len) 2^-24) (1 + 2^-5), the last factor for second orders (E' < 2^-6 in these tests);
      a weight times a value scale under the normal range of binary16 by 2^-25, where the largest scale is 2^6 at least and the sum
      of weights 1 at least: len 2^-31 max |v|."""
    codes, scales = cache
    cb = oracle.codebook(kind).astype(np.float64)
    page, dim, kv = codes.shape[3], codes.shape[4], codes.shape[2]
    group = q.shape[1] // kv
    out, tol = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    u = 2.0 ** -11
    for b in range(len(lens)):
        first, end = int(starts[b]), int(starts[b + 1])
        n, length = end - first, max(0, min(int(lens[b]), pages.shape[1] * page))
        j = np.arange(length)
        number = pages[b, j // page] if length else np.zeros(0, np.int64)
        there = (number >= 0) & (number < codes.shape[1])
        number = np.where(there, number, 0)
        for i in range(n):
            p = length - n + i
            seen = there & (j <= p) & ((j > p - window) if window else True)
            for h in range(kv):
                kk, vv = (cb[codes[part, number[seen], h, (j % page)[seen]]] * scales[part, number[seen], h, (j % page)[seen]].astype(np.float64)[:, None] for part in (0, 1))
                for x in range(h * group, (h + 1) * group):
                    row = q[first + i, x].astype(np.float64)
                    if not seen.any():
                        out[first + i, x] = tol[first + i, x] = 0.0
                        continue
                    s = kk @ row * softmax_scale
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    out[first + i, x] = w @ vv
                    e = (np.abs(kk) @ np.abs(row)).max() * abs(softmax_scale) * (u + (dim + 8) * 2.0 ** -24)
                    tol[first + i, x] = w @ np.abs(vv) * (2 * u + 2 * e + (8 + length) * 2.0 ** -24) * (1 + 2.0 ** -5) + length * 2.0 ** -31 * np.abs(vv).max()
                    assert not e >= 2.0 ** -6, "inputs outside the derivation"
    return out, tol
