"""CPU oracle for the paged key/value cache and the attention over it.  TEST INFRASTRUCTURE ONLY.

Plain numpy, written from the formulas (rotary positions, Eq. (1) of the paper in its asymmetric case with one group per
head, softmax attention).  `rotate_heads_by_position` and `quantise_heads` take the type to compute in: float64 is the
definition, float32 is the definition with every operation rounded, which is what the library promises for the numbers that go
into the cache.  Attention is float64 throughout.
"""
from __future__ import annotations

import numpy as np

from oracle.smoothrot_oracle import fwht_pow2, pack_uint4


def angles(max_pos: int, d: int, base: float = 10000.0) -> np.ndarray:
    """fp32 [max_pos, d]: cosines, then sines."""
    a = np.arange(max_pos, dtype=np.float64)[:, None] * base ** (-np.arange(0, d, 2, dtype=np.float64) / d)
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def hadamard_heads(x: np.ndarray) -> np.ndarray:
    """x [.., d] times H_d / sqrt(d), butterflies over strides 1, 2, 4, .. in x's own type, then one product."""
    d = x.shape[-1]
    y, h = x.copy(), 1
    while h < d:
        v = y.reshape(*x.shape[:-1], d // (2 * h), 2, h)
        a, b = v[..., 0, :].copy(), v[..., 1, :].copy()
        y = np.stack([a + b, a - b], -2).reshape(x.shape)
        h *= 2
    return y * x.dtype.type(1 / np.sqrt(d))


def rotate_heads_by_position(x, positions, cos_sin, pairs=False, hadamard=False, dtype=np.float64) -> np.ndarray:
    """x fp16 [T, heads, d] -> the same in `dtype`; positions are cut to the table; cos_sin None: no rotation."""
    x = np.asarray(x).astype(dtype)
    d = x.shape[-1]
    if cos_sin is not None:
        row = np.asarray(cos_sin)[np.clip(positions, 0, len(cos_sin) - 1)].astype(dtype)[:, None, :]
        c, s = row[..., :d // 2], row[..., d // 2:]
        y = np.empty_like(x)
        if pairs:
            a, b = x[..., 0::2], x[..., 1::2]
            y[..., 0::2], y[..., 1::2] = a * c - b * s, b * c + a * s
        else:
            a, b = x[..., :d // 2], x[..., d // 2:]
            y[..., :d // 2], y[..., d // 2:] = a * c - b * s, b * c + a * s
        x = y
    return hadamard_heads(x) if hadamard else x


def quantise_heads(v, clip=0.95, dtype=np.float64):
    """v fp16 [.., d] -> (codes uint8 [.., d], scale [..], zero [..]) of every row, computed in `dtype`."""
    v = np.asarray(v).astype(dtype)
    clip = dtype(np.float32(clip))
    hi, lo = clip * v.max(-1), clip * v.min(-1)
    scale = np.where(hi == lo, dtype(1), (hi - lo) * dtype(1 / 15))
    zero = -np.rint(lo / scale)
    codes = np.clip(np.rint(v / scale[..., None]) + zero[..., None], 0, 15)
    return codes.astype(np.uint8), scale, zero


def values_of(codes, scale, zero) -> np.ndarray:
    return (codes.astype(np.float64) - np.asarray(zero, np.float64)[..., None]) * np.asarray(scale, np.float64)[..., None]


def unpack_uint4(q) -> np.ndarray:
    q = np.asarray(q)
    return np.stack([q & 15, q >> 4], -1).reshape(*q.shape[:-1], 2 * q.shape[-1])


def attend(q, k, v, scale, seen):
    """One head: q [n, d], k, v [m, d], seen bool [n, m].  (o [n, d], weights [n, m] summing to 1 or 0, scores.)"""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    s = q @ k.T * scale
    masked = np.where(seen, s, -np.inf)
    top = masked.max(-1, keepdims=True, initial=-np.inf)
    p = np.exp(masked - np.where(np.isfinite(top), top, 0))
    total = p.sum(-1, keepdims=True)
    p = p / np.where(total == 0, 1, total)
    return p @ v, p, s


def causal(n: int, m: int) -> np.ndarray:
    """Row i of n sees key j of m where j <= i + m - n."""
    return np.arange(m)[None, :] <= np.arange(n)[:, None] + (m - n)
