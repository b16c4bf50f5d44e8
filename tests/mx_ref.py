"""Plain implementation of the microscaled operators in float64 (numpy), from the
formats' definition: an element is looked up in the table of its format's values.
Shares no code with the kernels or the binding."""
from __future__ import annotations

import numpy as np

FP4, FP8 = 0, 1


def table(fmt):
    """The non-negative finite values by code."""
    if fmt == FP4:
        return np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    c = np.arange(0x7F)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7.0))


def nearest(a, fmt):
    """Codes of non-negative numbers: nearest, ties to the even code, saturating."""
    t = table(fmt)
    mid = (t[1:] + t[:-1]) / 2
    c = np.searchsorted(mid, a, side="left")  # a == mid[c]: a tie between c and c + 1
    tie = (c < len(mid)) & (a == mid[np.minimum(c, len(mid) - 1)])
    return np.where(tie & (c % 2 == 1), c + 1, c)


def quantize(x, fmt):
    """x [R][K] float64 -> (codes uint8 [R][K], one each; scale bytes [R][ceil(K/32)])."""
    R, K = x.shape
    nb = -(-K // 32)
    full = np.zeros((R, nb * 32))
    full[:, :K] = x
    b = full.reshape(R, nb, 32)
    bad = ~np.isfinite(b).all(-1)
    top = np.where(bad, 0.0, np.abs(np.where(np.isfinite(b), b, 0)).max(-1))
    e = np.where(top > 0, np.frexp(top)[1] - 1, -1000) - (2 if fmt == FP4 else 8)
    e = np.maximum(e, -127)
    v = np.where(bad[..., None], 0.0, np.where(np.isfinite(b), b, 0)) / 2.0 ** e[..., None]
    codes = nearest(np.abs(v), fmt) | (np.signbit(v) << (3 if fmt == FP4 else 7))
    return (codes.reshape(R, -1)[:, :K].astype(np.uint8),
            np.where(bad, 255, e + 127).astype(np.uint8))


def elements(codes, fmt):
    bits = 3 if fmt == FP4 else 7
    m = codes & ((1 << bits) - 1)
    t = np.append(table(fmt), np.nan) if fmt == FP8 else table(fmt)
    return t[m] * np.where(codes >> bits, -1.0, 1.0)


def scales(b):
    return np.where(b == 255, np.nan, 2.0 ** (b.astype(np.float64) - 127))


def values(codes, sb, fmt):
    """float64 [R][K]"""
    return elements(codes, fmt) * np.repeat(scales(sb), 32, axis=1)[:, :codes.shape[1]]


def pack_bytes(codes, fmt):
    """One code each -> the dense bytes of whole blocks (zeros past K)."""
    R, K = codes.shape
    full = np.zeros((R, -(-K // 32) * 32), np.uint8)
    full[:, :K] = codes
    return full[:, 0::2] | (full[:, 1::2] << 4) if fmt == FP4 else full


def unpack_bytes(b, K, fmt):
    if fmt == FP8:
        return b[:, :K]
    return np.stack([b & 15, b >> 4], -1).reshape(b.shape[0], -1)[:, :K]


def tiled(codes, sb):
    """fp4 codes [N][K] and scale bytes -> the tiled bytes, word for word as the
    header describes them."""
    N, K = codes.shape
    T, S, C = -(-N // 32), -(-K // 128), -(-K // 512)
    full = np.zeros((T * 32, S * 128), np.uint8)
    full[:N, :K] = codes
    sfull = np.zeros((T * 32, C * 16), np.uint8)
    sfull[:N, :sb.shape[1]] = sb
    out, sout = np.zeros((T, S * 2048), np.uint8), np.zeros((T, C * 512), np.uint8)
    for t in range(T):
        for j in range(2):
            for l in range(64):
                g, i = l // 16, l % 16
                n = 32 * t + 8 * (i // 4) + 4 * j + i % 4
                for s in range(S):
                    e = full[n, 128 * s + 32 * g:128 * s + 32 * g + 32]
                    at = 2048 * s + 1024 * j + 16 * l
                    out[t, at:at + 16] = e[0::2] | (e[1::2] << 4)
                for c in range(C):
                    for b in range(4):
                        sout[t, 512 * c + 8 * l + 4 * j + b] = sfull[n, 16 * c + 4 * b + g]
    return out, sout


def silu(x):
    return x / (1 + np.exp(-x))


def rmsnorm(h, w, eps):
    return h / np.sqrt((h * h).mean(-1, keepdims=True) + eps) * w


def half_step(a, fmt):
    """Half the distance of the format's values around |a| (in units of the scale)."""
    low, places = (0, 1) if fmt == FP4 else (-6, 3)
    e = np.floor(np.log2(np.maximum(np.abs(a), 2.0 ** low)))
    return 2.0 ** (e - places - 1)
