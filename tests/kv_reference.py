"""The 4-bit key/value cache and its operators in 64 bits, on the CPU, from their definitions (include/macko.h)."""
import math

import numpy as np
import torch

STEPS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def piece_bytes(page, dim):
    return page * (dim + dim // 16)


def addresses(page, dim, t, d):
    """Where channel d of the token at t of a page lies in a head's piece: (byte, shift) of its key code, of its value code, and the bytes of their groups."""
    n = dim // 32
    key = t * (dim // 2) + d // 2
    value = page * dim // 2 + ((t // 4 * 16 + d % 16) * 4 + t % 4) * n + d // 32
    return (key, 4 * (d % 2)), (value, 4 * (d // 16 % 2)), page * dim + t * n + d // 32, page * dim + page * n + t * n + d // 32


def unit_of(byte):
    return np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127.0))


def read(data, page, dim, slots):
    """Keys and values [len(slots), heads, dim] as they stand in data [pages, heads, bytes] (numpy); zeros for slots outside the pool."""
    slots = np.asarray(slots, dtype=np.int64)
    there = (slots >= 0) & (slots < data.shape[0] * page)
    at = np.where(there, slots, 0)
    rows = data[at // page]                                    # [slots, heads, bytes]
    d = np.arange(dim)
    (kb, ks), (vb, vs), kg, vg = addresses(page, dim, (at % page)[:, None], d[None])
    out = []
    for byte, shift, group in ((kb, ks, kg), (vb, vs, vg)):
        take = lambda i: np.take_along_axis(rows, np.broadcast_to(i[:, None, :], (len(at), rows.shape[1], dim)), axis=2)  # noqa: E731
        code = (take(byte) >> np.broadcast_to(shift, byte.shape)[:, None, :].astype(np.uint8)) & 15
        value = STEPS[code & 7] * np.where(code & 8, -1.0, 1.0) * unit_of(take(group))
        value[~there] = 0.0
        out.append(value)
    return out


def nearest(x):
    """x [..., dim] (numpy, 64 bits) as the values that the cache holds for it."""
    g = x.reshape(x.shape[:-1] + (-1, 32))
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        most = np.abs(g).max(-1, keepdims=True)                # NaN stays
        b = np.zeros(most.shape)
        fine = np.isfinite(most) & (most > 0)
        e = np.ceil(np.log2(np.where(fine, most, 1.0) / 7.0))
        e = np.where(most > 7.0 * np.exp2(e), e + 1, e)
        e = np.where(most <= 7.0 * np.exp2(e - 1), e - 1, e)
        b = np.where(fine, np.clip(e + 127, 0, 254), 0)
        unit = np.exp2(b - 127)
        y = np.abs(g) / unit
        # the nearest step; of two equally near ones that of the even code
        gap = np.abs(y[..., None] - STEPS)
        code = np.argmin(np.where(np.arange(8) % 2 == 0, gap, np.nextafter(gap, np.inf)), axis=-1)
        code = np.where(np.isnan(y), 0, code)
        out = STEPS[code] * unit * np.sign(g)
        out = np.where(np.isfinite(most), out, np.nan)
    return out.reshape(x.shape)


def table(length, rot, base=10000.0, first=0, factor=1.0, trained=0, low=1.0, high=32.0, amplitude=1.0):
    f = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if factor != 1.0:
        turns = trained * f / (2 * math.pi)
        keep = np.clip((turns - low) / (high - low), 0, 1) if high > low else np.zeros_like(f)
        f = f * keep + f / factor * (1 - keep)
    angle = (first + np.arange(length))[:, None] * f
    return np.stack([np.cos(angle) * amplitude, np.sin(angle) * amplitude], 1)


def rotate(x, positions, tab, weight=None, eps=1e-6, interleaved=False):
    """x [tokens, heads, dim] in 64 bits; positions outside the table give NaN."""
    x = x.astype(np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    if tab is None:
        return x
    r = tab.shape[2]
    out = x.copy()
    positions = np.asarray(positions, dtype=np.int64)
    there = (positions >= 0) & (positions < len(tab))
    t = tab[np.where(there, positions, 0)].astype(np.float64)
    c, s = t[:, 0][:, None], t[:, 1][:, None]
    one, two = (np.arange(r) * 2, np.arange(r) * 2 + 1) if interleaved else (np.arange(r), np.arange(r) + r)
    a, b = x[..., one], x[..., two]
    out[..., one], out[..., two] = a * c - b * s, a * s + b * c
    out[~there] = np.nan
    return out


def attend(q, data, page, tables, lengths, start=None, scale=None, window=0):
    """out [tokens, heads, dim], sums [tokens, heads] and, for bounds, the largest sum of |q k| scale and the largest |v| of each row."""
    tokens, heads, dim = q.shape
    kv_heads = data.shape[1]
    scale = dim ** -0.5 if scale is None else scale
    start = list(range(tokens + 1)) if start is None else list(start)
    out, sums = np.zeros(q.shape), np.full((tokens, heads), -np.inf)
    reach, far = np.zeros((tokens, heads)), np.zeros((tokens, heads))
    for b, length in enumerate(lengths):
        length = max(0, int(length))
        n = start[b + 1] - start[b]
        for i in range(n):
            p = length - n + i
            lo = max(0, p - window + 1) if window else 0
            if p < lo:
                continue
            t = np.arange(lo, p + 1)
            index = t // page
            if index.max() >= tables.shape[1] or not ((tables[b, index] >= 0) & (tables[b, index] < len(data))).all():
                out[start[b] + i], sums[start[b] + i] = np.nan, np.nan
                continue
            k, v = read(data, page, dim, tables[b, index].astype(np.int64) * page + t % page)
            for h in range(heads):
                kh, vh = k[:, h * kv_heads // heads], v[:, h * kv_heads // heads]
                x = kh @ q[start[b] + i, h] * scale
                with np.errstate(invalid="ignore"):
                    m = x.max()
                    w = np.exp(x - m)
                    out[start[b] + i, h] = w @ vh / w.sum()
                    sums[start[b] + i, h] = m + np.log(w.sum())
                    reach[start[b] + i, h] = (np.abs(kh) @ np.abs(q[start[b] + i, h])).max() * abs(scale)
                    far[start[b] + i, h] = np.abs(vh).max()
    return out, sums, reach, far


def to_numpy(x):
    return x.detach().cpu().to(torch.float64).numpy()
