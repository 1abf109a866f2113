"""CPU oracle of the paged key-value cache and of the attention over it.  TEST INFRASTRUCTURE ONLY; shares no code with the HIP library.

The cache's quantiser is the AbsMax INT8 of Sec. 3.1 per token and head (decided in fp32: one quotient, one product, round half to even);
attention is the definition in fp64, row by row."""
from __future__ import annotations

import numpy as np

F32, F64 = np.float32, np.float64


def bf16(x):
    """fp32 values rounded to bf16 (ties to even; NaN kept), as fp32."""
    x = np.ascontiguousarray(x, F32)
    u = x.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> np.uint64(16)) & np.uint64(1))) & np.uint64(0xFFFF0000)).astype(np.uint32).view(F32).reshape(x.shape)
    return np.where(np.isnan(x), F32(np.nan), r)


def quantise(x):
    """Codes (int8) and steps (fp32) of the rows of the last axis; a row with an infinity or a NaN has the step NaN."""
    x = np.asarray(x, F32)
    bad = ~np.isfinite(x).all(-1)
    top = np.maximum(np.abs(np.where(np.isfinite(x), x, F32(0))).max(-1), F32(1e-5)).astype(F32)
    with np.errstate(all="ignore"):
        codes = np.clip(np.rint((x * (F32(128) / top)[..., None]).astype(F32)), -128, 127)
    codes = np.where(bad[..., None], 0, codes).astype(np.int8)
    return codes, np.where(bad, F32(np.nan), top / F32(128)).astype(F32)


def stored(x, int8):
    """What the cache stands for after x has been written (fp32 values)."""
    if not int8:
        return bf16(x)
    codes, step = quantise(x)
    return (codes.astype(F32) * step[..., None]).astype(F32)


def attention_row(q, k, v, seen, scale):
    """One row of one head: q [d], k, v [L][d], seen [L] bool.  Returns (o, lse, a) with a = sum p |v|, in fp64."""
    if not seen.any():
        return np.zeros(v.shape[1]), -np.inf, np.zeros(v.shape[1])
    k, v = k[seen].astype(F64), v[seen].astype(F64)
    s = scale * (k @ np.asarray(q, F64))
    m = s.max()
    p = np.exp(s - m)
    total = p.sum()
    return (p @ v) / total, m + np.log(total), (p @ np.abs(v)) / total


def visible(length, position, causal=True, window=0):
    """Which of `length` tokens a row at `position` sees."""
    t = np.arange(length)
    if position < 0:
        return np.zeros(length, bool)
    if not causal:
        return np.ones(length, bool)
    seen = t <= position
    if window:
        seen &= t > position - window
    return seen
