"""Weights in 4 bits, their products, the plan of a step and the verification of drafts from their definitions (numpy, 64 bits, one at a time)."""
import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TOP = 170 * 2.0 ** 118


def bf16(x):
    """Nearest bfloat16 number of finite non-negative float32 numbers, ties to even, as float64."""
    bits = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    bits = (bits + 0x7FFF + ((bits >> np.uint64(16)) & np.uint64(1))) >> np.uint64(16) << np.uint64(16)
    return bits.astype(np.uint32).view(np.float32).astype(np.float64)


def encode(w, group):
    """w float32 [rows, cols] -> (codes uint8 [row tiles, column tiles, 1024], scales float64 [row tiles, column tiles, 16, 128 / group])."""
    rows, cols = w.shape
    nt, kt = -(-rows // 16), -(-cols // 128)
    full = np.zeros((16 * nt, 128 * kt), np.float32)
    full[:rows, :cols] = w
    x = full.reshape(16 * nt, -1, group)
    a = np.abs(x).astype(np.float64)
    bad = ~np.isfinite(x).all(-1)
    most = np.where(bad, 0, a.max(-1)).astype(np.float32)
    s = np.minimum(bf16(most / np.float32(6)), TOP)
    with np.errstate(invalid="ignore"):
        far = np.abs(a[..., None] - MAGNITUDES * s[..., None, None])
    code = np.where((s[..., None] == 0) | bad[..., None], 0, np.where(np.isnan(far), np.inf, far).argmin(-1))  # the first of two as near: the smaller
    code = code + 8 * (np.signbit(x) & ~bad[..., None])
    s = np.where(bad, np.nan, s)
    codes = np.zeros((nt, kt, 1024), np.uint8)
    code = code.reshape(nt, 16, kt, 128)
    for g in range(4):
        for n in range(16):
            for word in range(4):
                for byte in range(4):
                    k = 32 * word + 8 * g + 2 * byte
                    codes[:, :, 16 * (16 * g + n) + 4 * word + byte] = code[:, n, :, k] | code[:, n, :, k + 1] << 4
    return codes, np.ascontiguousarray(s.reshape(nt, 16, kt, 128 // group).transpose(0, 2, 1, 3))


def decode(codes, scales, rows, cols):
    """The values in float64."""
    nt, kt = codes.shape[:2]
    got = np.zeros((nt, 16, kt, 128))
    for g in range(4):
        for n in range(16):
            for word in range(4):
                for byte in range(4):
                    c, k = codes[:, :, 16 * (16 * g + n) + 4 * word + byte], 32 * word + 8 * g + 2 * byte
                    for half, nibble in ((0, c & 15), (1, c >> 4)):
                        got[:, n, :, k + half] = MAGNITUDES[nibble & 7] * np.where(nibble & 8, -1.0, 1.0)
    s = np.asarray(scales, np.float64).transpose(0, 2, 1, 3)
    return (got.reshape(nt, 16, kt, s.shape[3], -1) * s[..., None]).reshape(16 * nt, 128 * kt)[:rows, :cols]


def plan(lens, new, pages, free, n_free, page, tokens, drop=None):
    """pages and free are changed; returns (slots, positions, starts, lens_out, granted, n_free_out)."""
    batch, wide = pages.shape
    count = lambda n: -(-n // page)
    n_free = min(max(int(n_free), 0), len(free))
    want, start = [], 0
    starts = [0]
    for b in range(batch):
        length, more, less = min(max(int(lens[b]), 0), wide * page), max(int(new[b]), 0), 0 if drop is None else max(int(drop[b]), 0)
        kept = max(length - less, 0)
        start += more
        starts.append(min(start, tokens))
        want.append([length, kept, more, kept + more <= wide * page and start <= tokens])
    stack = list(free[:n_free])
    for b, (length, kept, more, fits) in enumerate(want):
        for i in range(count(kept + more), count(length)) if fits else ():
            if len(stack) < len(free):
                stack.append(pages[b, i])
    free[: len(stack)] = stack
    slots, positions = np.full(tokens, -1, np.int64), np.full(tokens, -1, np.int64)
    lens_out, granted = np.zeros(batch, np.int32), np.zeros(batch, np.int32)
    asked, had = 0, len(stack)
    for b, (length, kept, more, fits) in enumerate(want):
        needs = max(0, count(kept + more) - count(length)) if fits else 0
        asked += needs
        if not fits or (needs and asked > had):
            lens_out[b], granted[b] = length, -1
            continue
        for i in range(count(length), count(length) + needs):
            pages[b, i] = stack.pop()
        lens_out[b], granted[b] = kept + more, more
        for i in range(more):
            p = kept + i
            positions[starts[b] + i] = p
            slots[starts[b] + i] = int(pages[b, p // page]) * page + p % page
    return slots, positions, np.array(starts, np.int32), lens_out, granted, len(stack)


def probability(x):
    x = np.asarray(x, np.float64)
    return np.where(np.isfinite(x) & (x > 0), x, 0.0)


def verify(target, ids, uniform, sample, starts, draft=None, out=None):
    """target, draft float [tokens, vocab]; returns (out, accepted, rejected)."""
    tokens, vocab = target.shape
    out = np.full(tokens, -1, np.int64) if out is None else out.copy()
    accepted, rejected = [], []
    for b in range(len(sample)):
        s0, s1 = min(max(int(starts[b]), 0), tokens), min(max(int(starts[b + 1]), 0), tokens)
        if s1 <= s0:
            accepted.append(-1)
            rejected.append(0)
            continue
        i, refused = s0, False
        while i + 1 < s1:
            d = int(ids[i + 1])
            p = float(probability(target[i, d])) if 0 <= d < vocab else 0.0
            q = 1.0 if draft is None else float(probability(draft[i, d])) if 0 <= d < vocab else 0.0
            if not float(uniform[i]) * q < p:
                refused = True
                break
            out[i] = d
            i += 1
        p = probability(target[i])
        w = p
        if refused:
            if draft is None:
                w = p.copy()
                if 0 <= int(ids[i + 1]) < vocab:
                    w[int(ids[i + 1])] = 0
            else:
                w = np.maximum(p - probability(draft[i]), 0)
            if not w.sum() > 0:
                w = p
        r = float(sample[b])
        r = r if r > 0 else 0.0
        over = np.nonzero((np.cumsum(w) > r * w.sum()) & (w > 0))[0]
        some = np.nonzero(w > 0)[0]
        out[i] = over[0] if len(over) else some[-1] if len(some) else -1
        out[i + 1 : s1] = -1
        accepted.append(i - s0)
        rejected.append(s1 - 1 - i)
    return out, np.array(accepted, np.int32), np.array(rejected, np.int32)
