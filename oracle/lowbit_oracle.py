"""MXFP4 matrices, their products, and AdamW over lists of tensors with 8-bit moments, in numpy on the host.

Written from the definitions (OCP microscaling formats: E2M1 values, one E8M0 scale per 32; E4M3 values), value by value in
64 bits, nothing blocked or fused.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def nearest_e2m1(a):
    """Codes 0..7 of magnitudes a >= 0: the nearest grid value, ties to the even code, beyond the largest: the largest."""
    a = np.asarray(a, dtype=np.float64)
    code = np.zeros(a.shape, dtype=np.uint8)
    for k in range(1, 8):
        middle = (GRID[k - 1] + GRID[k]) / 2
        code[(a > middle) | ((a == middle) & (k % 2 == 0))] = k
    return code


def quantize(x):
    """(codes [rows][cols], scale bytes [rows][ceil(cols / 32)]) of a float matrix, codes one to a byte."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    codes, scales = np.zeros((rows, cols), np.uint8), np.zeros((rows, (cols + 31) // 32), np.uint8)
    for b in range(scales.shape[1]):
        part = x[:, 32 * b:32 * b + 32]
        top = np.max(np.abs(part), axis=1)
        fine = np.isfinite(part).all(axis=1)
        with np.errstate(all="ignore"):
            e = np.where(top > 0, np.frexp(np.where(fine, top, 1.0))[1] - 1 - 2, -127)
        e = np.maximum(e, -127)
        scales[:, b] = np.where(fine, e + 127, 255)
        safe = np.where(fine[:, None], part, 0.0)
        codes[:, 32 * b:32 * b + 32] = nearest_e2m1(np.abs(safe) * np.exp2(-e.astype(np.float64))[:, None]) + 8 * (np.signbit(safe) & fine[:, None])
    return codes, scales


def values(codes, scales):
    v = np.where(codes >= 8, -1.0, 1.0) * GRID[codes & 7]
    f = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return v * np.repeat(f, 32, axis=1)[:, :codes.shape[1]]


def pack(codes, scales, pad_scale=0):
    """The two byte arrays of the layout that pac.h describes."""
    rows, cols = codes.shape
    blocks = (cols + 31) // 32
    full = np.zeros((rows, 32 * blocks), np.uint8)
    full[:, :cols] = codes
    packed = (full[:, 0::2] | (full[:, 1::2] << 4)).astype(np.uint8)
    out = np.full(((rows + 127) // 128, 2 * ((cols + 255) // 256), 32, 4, 4), pad_scale, np.uint8)
    for r in range(rows):
        for b in range(blocks):
            out[r // 128, b // 4, r % 32, r % 128 // 32, b % 4] = scales[r, b]
    return packed, out


def mix(x):
    x = x.astype(np.uint64)
    for shift, factor in ((16, 0x85EBCA6B), (13, 0xC2B2AE35)):
        x = (x ^ (x >> np.uint64(shift))) * np.uint64(factor) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random_bits(seed, step, place, n, first=0):
    """32 random bits per element of the tensor at `place` in the list."""
    one = lambda v: mix(np.array([v & 0xFFFFFFFF], dtype=np.uint64))  # noqa: E731
    k = int(one(seed + 0x9E3779B9 * step)[0])
    k = int(one(k + 0x9E3779B9 * (place + 1))[0])
    k = int(one(k + (first >> 32))[0])
    return mix((np.arange(n, dtype=np.uint64) + np.uint64(first & 0xFFFFFFFF)) ^ np.uint64(k))


def e4m3_values():
    c = np.arange(128)
    e, f = c >> 3, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * np.exp2(e - 7.0))
    v[127] = np.nan
    return v


def encode_e4m3(x, bits16, keep_positive):
    """(codes, constants) of magnitudes x (float32) in blocks of 256; every operation rounded to fp32 as the definition says."""
    f = np.float32
    n, nb = x.size, (x.size + 255) // 256
    codes, consts = np.zeros(n, np.uint8), np.zeros(nb, f)
    for b in range(nb):
        at = slice(256 * b, min(n, 256 * b + 256))
        part = x[at].astype(f)
        if not np.isfinite(part).all():
            consts[b] = np.nan
            continue
        top = part.max()
        if top < f(2.0 ** -100):
            continue
        consts[b] = top / f(448)
        r = np.minimum(part * (f(448) / top), f(448))
        # neighbours of r and the share of the way from one to the other, in units of 2^-16 of it
        grid = e4m3_values()[:127]
        lo = np.searchsorted(grid, r.astype(np.float64), side="right") - 1
        gap = np.where(lo < 8, 2.0 ** -9, np.exp2((lo >> 3) - 10.0))
        share = (r.astype(np.float64) - grid[lo]) / gap
        up = np.floor(share * 2 ** 20) + bits16[at].astype(np.float64) * 16 >= 2 ** 20
        c = lo + up
        if keep_positive:
            c = np.where((r > 0) & (c == 0), 1, c)
        codes[at] = c
    return codes, consts


def adamw(p, g, m, v, hp, step, decay, grad_scale=1.0):
    """One step in fp32 with every operation rounded, in the order of the definition."""
    f = np.float32
    lr, b1, b2, eps, wd = (f(hp[k]) for k in ("lr", "beta1", "beta2", "eps", "weight_decay"))
    bc1, bc2 = f(1 - float(b1) ** step), f(1 - float(b2) ** step)
    g = g.astype(f) * f(grad_scale)
    m = b1 * m + (f(1) - b1) * g
    v = b2 * v + ((f(1) - b2) * g) * g
    d = (lr * wd) * p if decay else f(0)
    return (p - d) - (lr * (m / bc1)) / (np.sqrt(v / bc2) + eps), m, v
