"""Pages of 4-bit keys and values, in plain numpy and binary64: the format, the
quantisation, reading and writing rows, and attention over them.

TEST INFRASTRUCTURE ONLY; shares nothing with the library.  Pools are uint8
[pages, H_kv, 17, D / 2]; a tile's bytes are addressed one by one.
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
NAN_SCALE = 255


def offsets(D, kind):
    """(code byte, nibble, scale byte) of every (slot, dim) of a tile, [16, D] each."""
    s, d = np.meshgrid(np.arange(16), np.arange(D), indexing="ij")
    if kind == "k":
        return d // 32 * 256 + s * 16 + d % 32 // 2, d % 2, 8 * D + d // 32 * 16 + s
    return ((s // 4 * 16 + d % 16) * (D // 8) + 2 * (d // 16) + s % 4 // 2, s % 2,
            8 * D + s // 4 * (D // 8) + 4 * (d // 32) + s % 4)


def scale_value(e):
    e = np.asarray(e, dtype=np.int64)
    return np.where(e == NAN_SCALE, np.nan, np.ldexp(1.0, np.where(e == NAN_SCALE, 127, e) - 127))


def code_value(c):
    c = np.asarray(c)
    return np.where(c & 8, -1.0, 1.0) * E2M1[c & 7]


def quantize(x):
    """[..., D] real values -> (codes [..., D], scale bytes [..., D / 32])."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    finite = np.isfinite(b).all(-1)
    top = np.where(finite, np.abs(np.where(np.isfinite(b), b, 0)).max(-1), 0)
    m, e = np.frexp(top)                       # top = 2 m * 2^(e - 1), 1 <= 2 m < 2
    e = e - 3 + (m > 0.875)
    e = np.clip(np.where(top > 0, e, -127), -127, 125)
    y = np.where(np.isfinite(b), b, 0) / np.ldexp(1.0, e)[..., None]
    # the nearest code of each magnitude, the even one of two equally near
    mag = np.minimum(np.abs(y), 6.0)
    dist = np.abs(mag[..., None] - E2M1)
    near = dist == dist.min(-1, keepdims=True)
    lowest = near.argmax(-1)
    both = near.sum(-1) == 2
    c = np.where(both & (lowest % 2 == 1), lowest + 1, lowest) + 8 * np.signbit(y)
    c = np.where(finite[..., None], c, 0)
    e = np.where(finite, e + 127, NAN_SCALE)
    return c.reshape(x.shape).astype(np.uint8), e.astype(np.uint8)


def dequantize(codes, scales):
    D = codes.shape[-1]
    v = code_value(codes).reshape(codes.shape[:-1] + (D // 32, 32)) * scale_value(scales)[..., None]
    return v.reshape(codes.shape)


def read_pages(pool, pages, kind):
    """Real values [tokens, H_kv, D] of the pages, in order."""
    D = 2 * pool.shape[-1]
    t = pool[np.asarray(pages, dtype=np.int64)].reshape(-1, pool.shape[1], 17 * D // 2)
    byte, nib, sc = offsets(D, kind)
    c = (t[:, :, byte] >> (4 * nib).astype(np.uint8)) & 15
    return (code_value(c) * scale_value(t[:, :, sc])).transpose(0, 2, 1, 3).reshape(-1, pool.shape[1], D)


def write_row(pool, page, slot, row, kind):
    """Quantise one token's row [H_kv, D] into its slot, in place."""
    D = 2 * pool.shape[-1]
    byte, nib, sc = (a[slot] for a in offsets(D, kind))
    codes, scales = quantize(row)
    for h in range(pool.shape[1]):
        t = pool[page, h].reshape(-1)
        # the bytes of a row are distinct for V, shared by two dims for K
        for n in (0, 1):
            at = byte[nib == n]
            t[at] = (t[at] & (0xF0 if n == 0 else 0x0F)) | (codes[h][nib == n] << (4 * n))
        t[sc[::32]] = scales[h]
        pool[page, h] = t.reshape(17, D // 2)


def write(k_pool, v_pool, k_rows, v_rows, table, lens, new):
    """Append new[b] rows (concatenated over requests) to request b; lens advance."""
    i = 0
    for b, n in enumerate(new):
        for j in range(n):
            pos = int(lens[b]) + j
            page = int(table[b, pos // 16])
            write_row(k_pool, page, pos % 16, k_rows[i], "k")
            write_row(v_pool, page, pos % 16, v_rows[i], "v")
            i += 1
        lens[b] += n


def attention(q, k_pool, v_pool, table, lens, new, scale):
    """Rows of the last new[b] tokens of each request over its keys up to
    their own: (out [T, H_q, D], weights times |values| [T, H_q, D], the
    magnitude that roundings of weights and scores are relative to, and the
    largest sum of |products| of a row's scores [T, H_q, 1])."""
    T, H_q, D = q.shape
    H = k_pool.shape[1]
    out, mag, dot = np.zeros(q.shape), np.zeros(q.shape), np.zeros((T, H_q, 1))
    i = 0
    for b, n in enumerate(new):
        L = int(lens[b])
        pages = table[b, :(L + 15) // 16]
        k, v = read_pages(k_pool, pages, "k")[:L], read_pages(v_pool, pages, "v")[:L]
        for h in range(H_q):
            g = h // (H_q // H)
            if L == 0:
                continue
            s = (q[i:i + n, h] @ k[:, g].T) * float(np.float32(scale))
            s = np.where(np.arange(L)[None, :] > (L - n + np.arange(n))[:, None], -np.inf, s)
            w = np.exp(s - s.max(-1, keepdims=True))
            w /= w.sum(-1, keepdims=True)
            seen = np.arange(L)[None, :] <= (L - n + np.arange(n))[:, None]
            nan = (seen @ np.isnan(v[:, g])) > 0            # of a token that the row sees
            x = np.nan_to_num(v[:, g])
            out[i:i + n, h] = np.where(nan, np.nan, w @ x)
            mag[i:i + n, h] = np.where(nan, np.nan, w @ np.abs(x))
            dot[i:i + n, h, 0] = np.where(seen, np.abs(q[i:i + n, h]) @ np.abs(k[:, g]).T, 0).max(-1) * abs(scale)
        i += n
    return out, mag, dot
