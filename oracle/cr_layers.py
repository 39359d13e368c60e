"""Layers in 64 bits: group norm with activation and dropout, dropout masks, 8-bit codes and products (NumPy).

Written from the formulas; shares no code with the library.
"""
from __future__ import annotations

import numpy as np

_U = np.uint64


def _mix(z):
    z = np.asarray(z, dtype=_U)
    with np.errstate(over="ignore"):
        z = (z ^ (z >> _U(30))) * _U(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> _U(27))) * _U(0x94D049BB133111EB)
    return z ^ (z >> _U(31))


def dropout_numbers(count: int, seed: int, offset: int) -> np.ndarray:
    """The 16-bit numbers of `count` elements from index `offset` on."""
    i = np.arange(count, dtype=_U) + _U(offset)
    with np.errstate(over="ignore"):
        words = _mix(_mix(_U(seed)) + (i // _U(4) + _U(1)) * _U(0x9E3779B97F4A7C15))
    return ((words >> (_U(16) * (i % _U(4)))) & _U(0xFFFF)).astype(np.int64)


def dropout_factors(shape, p: float, seed: int, offset: int) -> np.ndarray:
    """0 for a dropped element, the scale of the kept ones elsewhere."""
    t = int(np.floor(p * 65536 + 0.5))
    if t == 65536:
        return np.zeros(shape)
    keep = dropout_numbers(int(np.prod(shape)), seed, offset).reshape(shape) >= t
    return keep * (65536.0 / (65536 - t))


def _per_channel(v, channels):
    return np.repeat(v, channels // v.shape[1], axis=1)[:, None, :]


def _sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1 / (1 + e), e / (1 + e))


def group_norm(x, gamma, beta, groups, eps, act="none", factors=None):
    """(y, mean, rstd, z) of x [samples, positions, channels]."""
    x = np.asarray(x, dtype=np.float64)
    n, s, c = x.shape
    v = x.reshape(n, s, groups, c // groups)
    mean = v.mean(axis=(1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    rstd = 1 / np.sqrt(var + eps)
    z = (x - _per_channel(mean, c)) * _per_channel(rstd, c)
    z = z * (1.0 if gamma is None else np.asarray(gamma, np.float64)) + (0.0 if beta is None else np.asarray(beta, np.float64))
    y = {"none": lambda: z, "relu": lambda: np.maximum(z, 0), "silu": lambda: z * _sigmoid(z)}[act]()
    return (y if factors is None else y * factors), mean, rstd, z


def group_norm_backward(dy, x, gamma, beta, groups, eps, act="none", factors=None, partitions=1):
    """(dx, dgamma, dbeta, z, |terms| of dgamma, |terms| of dbeta) with the parameter gradients per partition."""
    x = np.asarray(x, dtype=np.float64)
    n, s, c = x.shape
    _, mean, rstd, z = group_norm(x, gamma, beta, groups, eps)
    xhat = (x - _per_channel(mean, c)) * _per_channel(rstd, c)
    dz = np.asarray(dy, dtype=np.float64) * (1.0 if factors is None else factors)
    if act == "relu":
        dz = dz * (z > 0)
    elif act == "silu":
        sg = _sigmoid(z)
        dz = dz * sg * (1 + z * (1 - sg))
    dxhat = dz * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    split = (n, s, groups, c // groups)
    m1 = dxhat.reshape(split).mean(axis=(1, 3))
    m2 = (dxhat * xhat).reshape(split).mean(axis=(1, 3))
    dx = _per_channel(rstd, c) * (dxhat - _per_channel(m1, c) - xhat * _per_channel(m2, c))
    by = lambda t: t.reshape(partitions, -1, c).sum(axis=1) if n else np.zeros((partitions, c))  # noqa: E731
    return dx, by(dz * xhat), by(dz), z, by(np.abs(dz * xhat)), by(np.abs(dz))


def quantize_rows(x):
    """(codes int64, scale float32) of the rows of x (float32 values), each step in the precision that defines it."""
    x = np.asarray(x, dtype=np.float32)
    codes = np.zeros(x.shape, dtype=np.int64)
    scale = np.zeros(x.shape[0], dtype=np.float32)
    for r in range(x.shape[0]):
        if not np.isfinite(x[r]).all():
            scale[r] = np.nan
            continue
        top = np.max(np.abs(x[r]))
        if top < np.float32(2.0 ** -120):
            continue
        scale[r] = top / np.float32(127)
        codes[r] = np.clip(np.rint(x[r] * (np.float32(127) / top)), -127, 127)
    return codes, scale


def int8_product(x, w, x_scale, w_scale, bias=None):
    """(y, the integer sums) in 64 bits."""
    sums = np.asarray(x, dtype=np.int64) @ np.asarray(w, dtype=np.int64).T
    y = sums.astype(np.float64) * np.asarray(x_scale, np.float64)[:, None] * np.asarray(w_scale, np.float64)[None, :]
    return (y if bias is None else y + np.asarray(bias, np.float64)), sums
