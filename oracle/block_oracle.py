"""What stands around the linear layers, on the CPU from its formulas, in float64 unless a definition names fp32: test infrastructure only.

    rms norm      h = x + residual;  rstd = 1 / sqrt(mean h^2 + eps);  y = h rstd gain
    its backward  v = dy gain;  dx = rstd (v - h rstd^2 mean(v h)) + dh;  dgain = sum dy h rstd
    8-bit rows    s = max(max|v| (1 / 127), 2^-126);  q = rint(v (1 / s)), each step in fp32
    8-bit layer   z = s_x s_w (sum q_x q_w) + bias
    dropout       y = keep x 65536 / (65536 - t) + residual;  keep: 16 bits of Philox 4x32-10 are t or more
"""
from __future__ import annotations

import numpy as np

GROUP = 32
MASK = 0xFFFFFFFF


def rms_norm(h, gain=None, eps=1e-6):
    """(rstd, y)"""
    h = np.asarray(h, np.float64)
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    y = h * rstd[:, None]
    return rstd, y if gain is None else y * np.asarray(gain, np.float64)


def rms_norm_backward(dy, h, rstd, gain=None, dh=None):
    """(dx, dgain)"""
    dy, h, rstd = np.asarray(dy, np.float64), np.asarray(h, np.float64), np.asarray(rstd, np.float64)[:, None]
    v = dy if gain is None else dy * np.asarray(gain, np.float64)
    dx = rstd * (v - h * rstd ** 2 * (v * h).mean(1, keepdims=True))
    return dx if dh is None else dx + np.asarray(dh, np.float64), (dy * h * rstd).sum(0)


def rows_save(v):
    """(codes, scales) of a two-dimensional array of fp32 values."""
    v = np.asarray(v, np.float32)
    samples, features = v.shape
    fine = np.isfinite(v).all(1)
    w = np.where(fine[:, None], v, np.float32(0))
    with np.errstate(under="ignore"):
        s = np.maximum(np.abs(w).max(1) * (np.float32(1) / np.float32(127)), np.float32(2.0 ** -126)).astype(np.float32)
        q = np.rint((w * (np.float32(1) / s)[:, None]).astype(np.float32))
    codes = np.zeros((samples, -(-features // GROUP) * GROUP), np.int8)
    codes[:, :features] = q
    return codes, np.where(fine, s, np.float32(np.nan)).astype(np.float32)


def norm_rows(h, gain=None, eps=1e-6):
    """(codes, scales) of the norm's 8-bit rows: those of h gain, their scales times rstd; of h 2^k gain, times rstd 2^-k, where rstd is not a
    normal number, h gain is too small for the least step or beyond fp32, 2^k the power of two below rstd (2^-126 to 2^126).  Rows of finite values."""
    h = np.asarray(h, np.float32)
    g = np.ones(h.shape[1], np.float32) if gain is None else np.asarray(gain, np.float32)
    with np.errstate(divide="ignore", over="ignore", under="ignore", invalid="ignore"):
        rstd = 1.0 / np.sqrt((h.astype(np.float64) ** 2).mean(1) + eps)
        k = np.clip(np.floor(np.log2(rstd)), -126, 126)
        most = np.abs(h * g).max(1)
        far = ~((rstd > 2.0 ** -126) & (rstd < 2.0 ** 126))
        k = np.where(far | ((most > 0) & (most < 2.0 ** -119) & (rstd > 1)) | (~(most < np.inf) & (rstd < 1)), k, 0)
        codes, scales = rows_save((h * np.exp2(k).astype(np.float32)[:, None]) * g)
    return codes, scales.astype(np.float64) * rstd * np.exp2(-k)


def rows_load(codes, scales, features):
    return codes[:, :features].astype(np.float64) * np.asarray(scales, np.float64)[:, None]


def int8_sums(x_codes, w_codes):
    """Integers below 2^53: exact in float64 too, and faster there."""
    return x_codes.astype(np.float64) @ w_codes.astype(np.float64).T


def philox(counter, key):
    """Four words of four, with plain integers: the published generator, ten rounds."""
    a, b, c, d = counter
    k0, k1 = key
    for _ in range(10):
        p, q = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = (q >> 32) ^ b ^ k0, q & MASK, (p >> 32) ^ d ^ k1, p & MASK
        k0, k1 = (k0 + 0x9E3779B9) & MASK, (k1 + 0xBB67AE85) & MASK
    return a, b, c, d


def bits(samples, features, seed, offset):
    out = np.zeros((samples, -(-features // 8) * 8), np.int64)
    offset &= (1 << 64) - 1
    for m in range(samples):
        for k in range(out.shape[1] // 8):
            words = philox((k, m, offset & MASK, offset >> 32), (seed & MASK, seed >> 32))
            for w, v in enumerate(words):
                out[m, 8 * k + 2 * w], out[m, 8 * k + 2 * w + 1] = v & 0xFFFF, v >> 16
    return out[:, :features]


def dropout(x, p, seed, offset, residual=None):
    """(keep, y)"""
    x = np.asarray(x, np.float64)
    t = round(p * 65536)
    keep = bits(*x.shape, seed, offset) >= t
    y = np.where(keep, x * (65536 / (65536 - t) if t < 65536 else 0.0), 0.0)
    return keep, y if residual is None else y + np.asarray(residual, np.float64)
