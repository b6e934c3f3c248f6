"""The 8-bit key/value cache and its operators in 64 bits, on the CPU, from their definitions (include/macko.h)."""
import numpy as np

BLOCK = 16


def numbers():
    """What the 256 codes stand for."""
    code = np.arange(256)
    e, f = code >> 3 & 15, code & 7
    x = np.where(e > 0, (8 + f) * np.exp2(e - 10.0), f * 2.0 ** -9)
    return np.where(code & 127 == 127, np.nan, x) * np.where(code & 128, -1.0, 1.0)


NUMBERS = numbers()
STEPS = NUMBERS[:127]                              # magnitudes, in order


def nearest(y):
    """The number nearest to y, of two equally near ones that of the even code; 448 at most; NaN for what is not finite."""
    a = np.where(np.isfinite(y), np.minimum(np.abs(y), 448.0), 0.0)
    up = np.clip(np.searchsorted(STEPS, a), 1, 126)
    low, high = a - STEPS[up - 1], STEPS[up] - a
    code = np.where((low < high) | ((low == high) & (up % 2 == 1)), up - 1, up)
    return np.where(np.isfinite(y), STEPS[code] * np.sign(y), np.nan)


def byte_of(x):
    """The byte of a block with these values."""
    most = np.abs(np.where(np.isfinite(x), x, 0.0)).max()
    b = 1
    while b < 246 and most > 448.0 * 2.0 ** (b - 127):
        b += 1
    return b


def locate(page, dim, t, d):
    """Of channel d of the token at t of a page: its block in the page, and its place among the block's key codes and value codes."""
    at = t % BLOCK
    return t // BLOCK, at * dim + d, (at // 4 * dim + d) * 4 + at % 4


def read(data, scales, page, slots):
    """Keys and values [slots, heads, dim] of data [pages, heads, blocks, 2, 16 dim] and scales [pages, heads, blocks, 2] (numpy); zeros outside the pool."""
    slots = np.asarray(slots, dtype=np.int64)
    dim = data.shape[4] // BLOCK
    there = (slots >= 0) & (slots < data.shape[0] * page)
    at = np.where(there, slots, 0)
    block, key, value = locate(page, dim, (at % page)[:, None], np.arange(dim)[None])
    out = []
    for j, where in ((0, key), (1, value)):
        rows = data[at // page, :, block[:, 0], j]                                # [slots, heads, 16 dim]
        codes = np.take_along_axis(rows, np.broadcast_to(where[:, None], rows.shape[:2] + (dim,)), 2)
        with np.errstate(over="ignore"):
            x = NUMBERS[codes] * np.exp2(scales[at // page, :, block[:, 0], j].astype(np.float64) - 127.0)[..., None]
        x[~there] = 0.0
        out.append(x)
    return out


def append(held, k, v, page, tables, lengths, start, pages):
    """`held`: (keys, values, bytes) as read() and scales give them for every slot, changed in place: what the pool stands for after the call.
    k and v [tokens, heads, dim] as they are stored.  Returns the slots that were written."""
    written = []
    for b, length in enumerate(lengths):
        length, rows = max(0, int(length)), start[b + 1] - start[b]
        place, row = length - rows, start[b]
        if place < 0:
            place, row = 0, row - place
        while place < length:
            end = min(length, place // BLOCK * BLOCK + BLOCK)
            first, index = place % BLOCK, place // page
            if index < tables.shape[1] and 0 <= tables[b, index] < pages:
                p, block = int(tables[b, index]), place % page // BLOCK
                base = p * page + block * BLOCK
                written += range(base + first, base + first + end - place)
                for j, x in enumerate((k, v)):
                    for h in range(k.shape[1]):
                        new = x[row:row + end - place, h]
                        had = int(held[2][p, h, block, j])
                        byte = byte_of(new) if first == 0 else max(byte_of(new), had)
                        pool = held[j]
                        unit = 2.0 ** (byte - 127)
                        if byte != had:
                            pool[base:base + first, h] = nearest(pool[base:base + first, h] / unit) * unit
                            pool[base + first + end - place:base + BLOCK, h] *= 2.0 ** (byte - had)       # codes stay
                        pool[base + first:base + first + end - place, h] = nearest(new / unit) * unit
                        held[2][p, h, block, j] = byte
            row += end - place
            place = end
    return written


def attend(q, k, v, first=0, scale=None, window=0):
    """Rows q [n, heads, dim] at the places first, first + 1, ... over k and v [tokens, kv heads, dim]: results, sums and, for bounds, the largest sum of
    |q k| scale and the largest |v| of each row."""
    n, heads, dim = q.shape
    scale = dim ** -0.5 if scale is None else scale
    out, sums = np.zeros(q.shape), np.full((n, heads), -np.inf)
    reach, far = np.zeros((n, heads)), np.zeros((n, heads))
    for i in range(n):
        p = first + i
        lo = max(0, p - window + 1) if window else 0
        if p < lo:
            continue
        for h in range(heads):
            g = h * k.shape[1] // heads
            kh, vh = k[lo:p + 1, g], v[lo:p + 1, g]
            with np.errstate(invalid="ignore", over="ignore"):
                x = kh @ q[i, h] * scale
                m = x.max()
                w = np.exp(x - m)
                out[i, h] = w @ vh / w.sum()
                sums[i, h] = m + np.log(w.sum())
                reach[i, h] = (np.abs(kh) @ np.abs(q[i, h])).max() * abs(scale)
                far[i, h] = np.abs(vh).max()
    return out, sums, reach, far


def attend_cached(q, data, scales, page, tables, lengths, start=None, scale=None, window=0):
    """attend over the pool; NaN for rows that need a page which is not there."""
    tokens, heads, dim = q.shape
    start = list(range(tokens + 1)) if start is None else list(start)
    parts = [np.zeros(q.shape), np.full((tokens, heads), -np.inf), np.zeros((tokens, heads)), np.zeros((tokens, heads))]
    for b, length in enumerate(lengths):
        length, n = max(0, int(length)), start[b + 1] - start[b]
        t = np.arange(length)
        index = t // page
        pages = tables[b, np.minimum(index, tables.shape[1] - 1)].astype(np.int64) if tables.shape[1] else np.full(length, -1)
        fine = (index < tables.shape[1]) & (pages >= 0) & (pages < len(data))
        k, v = read(data, scales, page, np.where(fine, pages * page + t % page, -1))
        got = attend(q[start[b]:start[b + 1]], k, v, length - n, scale, window)
        for i in range(n):
            p = length - n + i
            lo = max(0, p - window + 1) if window else 0
            if p >= lo and not fine[lo:p + 1].all():
                got[0][i], got[1][i] = np.nan, np.nan
        for whole, part in zip(parts, got):
            whole[start[b]:start[b + 1]] = part
    return parts
