"""CPU oracle for the operators around the linear layers: the norm between two
blocks, the 4-bit key/value rows, the rotation, and attention.

TEST INFRASTRUCTURE ONLY: imported by the tests and the smoke check, never by
the library.  Plain numpy in float64; the quantizer works in float32 where its
definition does, because a code is the outcome of those roundings.

    norm       y = x or rms(x) (post + o);  r = residual + scale gate y;  rms(r) (w + o)
    rotation   (x1, x2) -> (x1 cos - x2 sin, x2 cos + x1 sin),  x2 = x1's partner D/2 on
    row        s = (max - min) / 15, z = -min / s, q = round(x / s + z) in 0..15
    attention  softmax(scale Q K^T) V over the visible keys, zeros where there are none
"""
from __future__ import annotations

import numpy as np

from .awq_oracle import to_f16
from .bf16_oracle import to_bf16

__all__ = ["round16", "rms_norm_block", "rotate", "quant_rows", "cached_rows", "attend", "attend_bound"]


def round16(v, dtype: str):
    """float64 values rounded once to 'f16' or 'bf16', as float64."""
    v = np.asarray(v, dtype=np.float64)
    return to_f16(v).astype(np.float64) if dtype == "f16" else to_bf16(v)


def rms_norm_block(x, residual=None, weight=None, post=None, gate=None, scale=1.0, offset=0.0, eps=1e-6):
    """(normed or None, r) in float64."""
    def rms(t):
        return t / np.sqrt((t * t).mean(-1, keepdims=True) + eps)
    y = np.asarray(x, np.float64)
    if post is not None:
        y = rms(y) * (post + offset)
    if gate is not None:
        y = y * gate
    r = scale * y + (0.0 if residual is None else residual)
    return (None if weight is None else rms(r) * (weight + offset)), r


def rotate(x, cos, sin):
    """x [tokens, heads, D], cos and sin [tokens, D/2], in x's precision."""
    h = x.shape[-1] // 2
    a, b, c, s = x[..., :h], x[..., h:], cos[:, None], sin[:, None]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def quant_rows(x, dtype: str):
    """Rows [..., D] of float32 -> (codes, scales, zero-points), the last two as
    float64 values of the 16-bit type.  Every step is a float32 operation."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
        f = np.float32(1) / np.float32(15)
        s = round16((hi * f - lo * f).astype(np.float64), dtype).astype(np.float32)
        flat = (s <= np.float32(2.0 ** -100)) | (np.abs(lo) > np.float32(32768) * s)
        z = round16((-lo / s).astype(np.float64), dtype).astype(np.float32)
        q = np.clip(np.rint(x * (np.float32(1) / s) + z), 0, 15)
    bad = ~np.isfinite(x).all(-1, keepdims=True) | np.isinf(s)
    q = np.where(flat | bad, 0, q)
    z = np.where(bad, 0, np.where(flat, -1, z)).astype(np.float64)
    s = np.where(bad, np.nan, np.where(flat, round16(lo.astype(np.float64), dtype), s.astype(np.float64)))
    return q.astype(np.uint8), s, z


def cached_rows(x, dtype: str):
    """What rows of float32 stand for once cached (float64, not rounded)."""
    q, s, z = quant_rows(x, dtype)
    return s * (q.astype(np.float64) - z)


def attend(q, k, v, scale, last):
    """One head: q [n, D], k and v [m, D]; query i sees the keys 0..last[i]."""
    out = np.zeros((q.shape[0], v.shape[1]))
    for i in range(q.shape[0]):
        m = min(int(last[i]) + 1, k.shape[0])
        if m <= 0:
            continue
        a = scale * (k[:m] @ q[i])
        p = np.exp(a - a.max())
        out[i] = (p / p.sum()) @ v[:m]
    return out


def attend_bound(q, k, v, scale, last):
    """sum_j p_j |v_j|: what a relative error of every weight p_j can change."""
    return attend(q, k, np.abs(v), scale, last)
