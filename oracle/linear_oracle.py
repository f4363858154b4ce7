"""The linear layer with 8-bit activation checkpoints, in float64 on the CPU, from its formulas: test infrastructure only.

    z = x w^T + bias;  y = act(z) + residual;  dz = dy act'(z^);  dbias = sum dz;  dw = dz^T x^;  dx = dz w

A checkpoint keeps groups of 32 features of a sample as integers times a power of two.
"""
from __future__ import annotations

import numpy as np
from scipy.special import erfc, expit

GROUP = 32
BOUNDS = {"f32": (-126, 121), "bf16": (-126, 121), "f16": (-24, 9)}


def save(v, kind):
    """(codes, exponent bytes) of a two-dimensional array."""
    v = np.asarray(v, np.float64)
    lo, hi = BOUNDS[kind]
    samples, features = v.shape
    groups = -(-features // GROUP)
    codes = np.zeros((samples, groups * GROUP), np.int8)
    exps = np.zeros((samples, groups), np.uint8)
    for g in range(groups):
        part = v[:, g * GROUP:(g + 1) * GROUP]
        fine = np.isfinite(part).all(1)
        absmax = np.abs(np.where(fine[:, None], part, 0.0)).max(1)
        e = np.full(samples, lo)
        for s in range(samples):
            if absmax[s] > 0:
                k = int(np.floor(np.log2(absmax[s]))) - 9          # well below; then the smallest that takes it under 127.5
                while absmax[s] >= 127.5 * 2.0 ** k:
                    k += 1
                e[s] = min(max(k, lo), hi)
        q = np.clip(np.rint(np.where(fine[:, None], part, 0.0) * 2.0 ** -e[:, None].astype(np.float64)), -127, 127)
        codes[:, g * GROUP:g * GROUP + part.shape[1]] = q
        exps[:, g] = np.where(fine, e + 127, 255)
    return codes, exps


def load(codes, exps, features):
    f = np.where(exps == 255, np.nan, 2.0 ** (exps.astype(np.float64) - 127))
    f = np.where(exps == 0, 0.0, f)
    return (codes.astype(np.float64) * np.repeat(f, GROUP, 1))[:, :features]


def activate(z, act):
    if act == "relu":
        return np.where(z < 0, 0.0, z)
    if act == "gelu":
        return z * 0.5 * erfc(-z / np.sqrt(2.0))
    if act == "silu":
        return z * expit(z)
    return np.asarray(z, np.float64)


def slope(z, act):
    if act == "relu":
        return np.where(np.isnan(z), np.nan, (z > 0).astype(np.float64))
    if act == "gelu":
        return 0.5 * erfc(-z / np.sqrt(2.0)) + z * np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
    if act == "silu":
        s = expit(z)
        return s + z * s * (1.0 - s)
    return np.ones_like(z, dtype=np.float64)


def forward(x, w, bias=None, residual=None, act="none"):
    """(z, y)"""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    y = activate(z, act)
    return z, y if residual is None else y + np.asarray(residual, np.float64)


def activation_backward(dy, z_held, act):
    """(dz before rounding, dbias)"""
    dz = np.asarray(dy, np.float64) * (slope(z_held, act) if act != "none" else 1.0)
    return dz, dz.sum(0)


def input_grad(dz, w):
    return np.asarray(dz, np.float64) @ np.asarray(w, np.float64)


def weight_grad(dz, x_held):
    return np.asarray(dz, np.float64).T @ x_held
