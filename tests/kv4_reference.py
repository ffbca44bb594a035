"""Plain reference of a cache held in 4 bits (numpy): what a row stands for, bit for bit in the
library's binary32 arithmetic, and attention over such rows in 64 bits."""
from __future__ import annotations

import numpy as np

GROUP, GQA = 32, 4
BASE = 10000.0


def bf16(x):
    """x rounded to bfloat16 (ties to even; NaN stays NaN), as float32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), r)


def in_type(x, dtype):
    return bf16(x) if dtype == "bf16" else np.asarray(x, np.float32)


def table(pos, d):
    a = np.asarray(pos, np.float64)[:, None] * BASE ** (-2.0 * np.arange(d // 2) / d)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def rotate32(x, pos):
    """x [n, heads, D] float32, every product and sum rounded."""
    d = x.shape[-1]
    c, s = (t[:, None] for t in table(pos, d))
    a, b = x[..., :d // 2], x[..., d // 2:]
    with np.errstate(invalid="ignore", over="ignore"):
        return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def rotate64(x, pos):
    d = x.shape[-1]
    c, s = (t[:, None].astype(np.float64) for t in table(pos, d))
    a, b = x[..., :d // 2].astype(np.float64), x[..., d // 2:].astype(np.float64)
    return np.concatenate([a * c - b * s, b * c + a * s], axis=-1)


def held(x):
    """The numbers that x [..., D] float32 is held as (float32, exact)."""
    x = np.asarray(x, np.float32)
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    most = np.abs(g).max(axis=-1, keepdims=True)          # (NaN wins)
    fine = np.isfinite(most)
    s = np.where(fine, most, np.float32(0)) / np.float32(7)
    _, e = np.frexp(s)
    step = np.ldexp(np.float32(1), np.maximum(e - 7, -20)).astype(np.float32)
    s = np.minimum(np.rint(s / step) * step, np.float32(9344))
    with np.errstate(invalid="ignore"):
        c = np.clip(np.rint(g / np.where(s > 0, s, np.float32(1))), -7, 7)
    return np.where(fine, c * s, np.float32(np.nan)).reshape(x.shape).astype(np.float32)


def attention(q, qpos, k, v, seen):
    """q [t, 4 H, D] un-rotated; k (rotated), v [n, H, D]; seen[i]: number of rows that token i sees.
    64-bit; [t, 4 H, D]."""
    t, hq, d = q.shape
    x = rotate64(q, qpos).reshape(t, hq // GQA, GQA, d)
    out = np.zeros((t, hq // GQA, GQA, d))
    for i in range(t):
        kk, vv = k[:seen[i]].astype(np.float64), v[:seen[i]].astype(np.float64)
        s = np.einsum("hgd,nhd->hgn", x[i], kk) / np.sqrt(d)
        w = np.exp(s - s.max(axis=-1, keepdims=True))
        out[i] = np.einsum("hgn,nhd->hgd", w / w.sum(axis=-1, keepdims=True), vv)
    return out.reshape(t, hq, d)
