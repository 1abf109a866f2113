"""CPU oracle of rotary positions, of attention over packed rows with its gradient, and of the AdamW step.  TEST INFRASTRUCTURE ONLY; shares no code with
the HIP library.  Definitions in fp64, sequence by sequence and head by head; only the codes of 8-bit states are decided in fp32, as they are defined."""
from __future__ import annotations

import numpy as np

from .attention_oracle import visible

F32, F64 = np.float32, np.float64


def rope(x, freqs, positions, layout, inverse=False, scale=1.0):
    """x [T][heads][d], freqs [rot / 2] turns per position, positions [T]; layout "half" or "pairs"."""
    y, rot = np.array(x, F64), 2 * len(freqs)
    first = np.arange(rot // 2) if layout == "half" else 2 * np.arange(rot // 2)
    second = first + (rot // 2 if layout == "half" else 1)
    turns = np.asarray(positions, F64)[:, None] * np.asarray(freqs, F64)
    z = scale * np.exp((-2j if inverse else 2j) * np.pi * (turns - np.rint(turns)))[:, None, :]
    turned = (y[..., first] + 1j * y[..., second]) * z
    y[..., first], y[..., second] = turned.real, turned.imag
    return y


def seen_by(n, causal=True, window=0):
    """[row][token] of a sequence of n rows."""
    return np.stack([visible(n, i, causal, window) for i in range(n)]) if n else np.zeros((0, 0), bool)


def self_attention(q, k, v, seen, scale):
    """One head of one sequence: q, k, v [n][d].  Returns o, lse and p [row][token] in fp64."""
    s = np.where(seen, scale * (np.asarray(q, F64) @ np.asarray(k, F64).T), -np.inf)
    top = s.max(1, keepdims=True)
    e = np.exp(s - top)
    total = e.sum(1, keepdims=True)
    return (e / total) @ np.asarray(v, F64), (top + np.log(total))[:, 0], e / total


def self_attention_gradients(do, q, k, v, lse, seen, scale):
    """From the lse that the forward pass left.  Returns dq, dk, dv, p and dS."""
    do, q, k, v = (np.asarray(x, F64) for x in (do, q, k, v))
    p = np.where(seen, np.exp(np.where(seen, scale * (q @ k.T) - np.asarray(lse, F64)[:, None], 0.0)), 0.0)
    dp = do @ v.T
    ds = p * (dp - (p * dp).sum(1, keepdims=True))
    ds[seen.sum(1) == 1] = 0.0                                       # (p is 1 whatever the score)
    return scale * (ds @ k), scale * (ds.T @ q), p.T @ do, p, ds


def nearest_codes(x, top):
    """Codes (whole numbers) of |x| under the law code^2 step, and the step, of blocks [..][256]; quotients in fp32, ties to even."""
    x = np.abs(np.asarray(x, F32))
    step = np.maximum(x.max(-1, keepdims=True) * F32(1.0 / top ** 2), F32(2.0 ** -126)).astype(F32)
    y = (x * (F32(1) / step)).astype(F32).astype(F64)
    code = np.floor(np.sqrt(y))                                      # exact in fp64 for fp32 squares; the border above is (code + 1/2)^2
    border = (code + 0.5) ** 2
    code = np.where((y > border) | ((y == border) & (code % 2 == 1)), code + 1, code)
    return np.minimum(code, top), step


def blocks(x):
    x = np.asarray(x).reshape(-1)
    return np.concatenate([x, np.zeros(-len(x) % 256, x.dtype)]).reshape(-1, 256)


def decode(qm, qr, steps):
    """(m, r) in fp32 of 8-bit states [blocks][256]."""
    qm, qr = np.asarray(qm, F32), np.asarray(qr, F32)
    return (qm * np.abs(qm) * steps[:, :1]).astype(F32), (qr * qr * steps[:, 1:]).astype(F32)


def moments(g, m, v, beta1, beta2, grad_scale):
    """The new moments in fp32, every product and sum rounded, and sqrt v correctly rounded."""
    g = (np.asarray(g, F32) * F32(grad_scale)).astype(F32)
    m = (np.asarray(m, F32) * F32(beta1)).astype(F32) + (g * F32(1.0 - beta1)).astype(F32)
    v = (np.asarray(v, F32) * F32(beta2)).astype(F32) + ((g * F32(1.0 - beta2)).astype(F32) * g).astype(F32)
    return m, v, np.sqrt(v.astype(F64)).astype(F32)


def adamw_weight(w, m, v, step, lr, weight_decay, beta1, beta2, eps):
    """The new weight in fp64 from the new moments."""
    w, m, v = (np.asarray(x, F64) for x in (w, m, v))
    return w - lr * weight_decay * w - lr * (m / (1.0 - beta1 ** step)) / (np.sqrt(v / (1.0 - beta2 ** step)) + eps)
