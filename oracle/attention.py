"""CPU reference of the attention operators in float64: head norm and rotation,
the 4-bit cache's format read and written byte by byte, and attention with the
mask of decoding in blocks.  Shares no code with the kernels or the binding."""
from __future__ import annotations

import math

import numpy as np

PAGE = 64
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def scale_stride(D: int) -> int:
    return 4 * math.ceil(D / 32 / 4)


def tile_bytes(D: int) -> int:
    return 2 * (PAGE * D // 2 + PAGE * scale_stride(D))


def quantise_group(x):
    """(scale byte, 32 codes) of one group, from the definition: the smallest
    e >= -126 with max |x| <= 7 * 2^e, every element to the nearest magnitude,
    a tie to the even code, more than 6 to 6."""
    x = np.asarray(x, dtype=np.float64)
    if not np.isfinite(x).all():
        return 255, np.zeros(len(x), dtype=np.int64)
    top, e = float(np.abs(x).max()), -126
    if top > 0:
        e = max(-126, math.frexp(top / 7.0)[1] - 2)
        while top > 7.0 * 2.0 ** e:
            e += 1
    codes = []
    for v in x:
        a = abs(float(v)) / 2.0 ** e
        gaps = np.abs(MAGNITUDES - a)
        best = np.flatnonzero(gaps == gaps.min())
        c = int(best[0]) if len(best) == 1 or best[0] % 2 == 0 else int(best[1])
        codes.append(c + (8 if math.copysign(1.0, float(v)) < 0 else 0))
    return e + 127, np.array(codes)


def value_of(byte: int, code):
    """What codes of a group with this scale byte stand for."""
    if byte == 255:
        return np.full(np.shape(code), np.nan)
    code = np.asarray(code)
    return np.where(code >= 8, -1.0, 1.0) * MAGNITUDES[code & 7] * 2.0 ** (byte - 127)


def put(tile, D: int, value: bool, token: int, x):
    """Write one token's D elements into a tile (uint8 array of tile_bytes(D))."""
    codes_at = PAGE * D // 2 if value else 0
    scales_at = PAGE * D + (PAGE * scale_stride(D) if value else 0)
    for g in range(D // 32):
        byte, c = quantise_group(x[32 * g:32 * g + 32])
        for n in range(16):
            tile[codes_at + (g * PAGE + token) * 16 + n] = c[2 * n] | c[2 * n + 1] << 4
        tile[scales_at + token * scale_stride(D) + g] = byte


def get(tile, D: int, value: bool, token: int):
    """One token's D elements out of a tile."""
    codes_at = PAGE * D // 2 if value else 0
    scales_at = PAGE * D + (PAGE * scale_stride(D) if value else 0)
    out = np.empty(D)
    for g in range(D // 32):
        at = codes_at + (g * PAGE + token) * 16
        raw = np.asarray(tile[at:at + 16]).astype(np.int64)
        c = np.stack([raw & 15, raw >> 4], axis=1).reshape(-1)
        out[32 * g:32 * g + 32] = value_of(int(tile[scales_at + token * scale_stride(D) + g]), c)
    return out


def norm_rope(x, weight, eps, cos, sin, interleaved):
    """One head's row: RMS norm (weight None: none), then the rotation of its
    first 2 len(cos) elements."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / math.sqrt(float(np.mean(x * x)) + eps) * np.asarray(weight, dtype=np.float64)
    y = x.copy()
    half = len(cos)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[a] = x[a] * cos[i] - x[b] * sin[i]
        y[b] = x[b] * cos[i] + x[a] * sin[i]
    return y


def visible(p: int, blk: int, length: int) -> int:
    """How many of the first keys a query at position p sees."""
    if blk == 0:
        return length
    return max(0, min(length, (p // blk + 1) * blk))


def attend(q, k, v, scale, blk, start):
    """q [n, H, D], k, v [len, Hk, D] (float64): out, lse, and for the bounds of
    the tests the attention of |v| and the largest sum of |q_d k_d| of a row."""
    n, H, D = q.shape
    length, Hk = k.shape[:2]
    out, av = np.zeros((n, H, D)), np.zeros((n, H, D))
    lse, sabs = np.full((n, H), -np.inf), np.zeros((n, H))
    for i in range(n):
        m = visible(start + i, blk, length)
        if m == 0:
            continue
        for h in range(H):
            kk, vv = k[:m, h // (H // Hk)], v[:m, h // (H // Hk)]
            s = kk @ q[i, h] * scale
            top = s.max()
            w = np.exp(s - top)
            lse[i, h] = top + math.log(w.sum())
            w /= w.sum()
            out[i, h], av[i, h] = w @ vv, w @ np.abs(vv)
            sabs[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
    return out, lse, av, sabs
