"""Plain 64-bit forms of the operators around the 4-bit store, in numpy, and what their tests share."""
from fractions import Fraction
import math

import numpy as np

GROUP = 32
# 2 pi to 60 digits, as a fraction: far positions are reduced exactly before anything is rounded
TWO_PI = Fraction("6.28318530717958647692528676655900576839433879875021164194988")


def grid_positions(T, t0, h, w):
    n = np.arange(T, dtype=np.int64)
    return np.stack([t0 + n // (h * w), n // w % h, n % w], -1)


def frequencies(axes, theta=10000.0):
    return np.asarray([theta ** (-2.0 * i / n) for n in axes for i in range(n // 2)], np.float64)


def norm_rope(x, pos, axes, halves=False, weight=None, norm=True, eps=1e-6, freq=None):
    """x [H, T, d] float64; returns (y, size of the pair an element turns in)."""
    x = np.asarray(x, np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * np.asarray(weight, np.float64)
    freq = frequencies(axes) if freq is None else np.asarray(freq, np.float64)
    y, size, start, k = x.copy(), np.abs(x), 0, 0
    for axis, n in enumerate(axes):
        for i in range(n // 2):
            a, b = (start + i, start + n // 2 + i) if halves else (start + 2 * i, start + 2 * i + 1)
            f = Fraction(float(freq[k]))
            ang = np.asarray([float((int(p) * f) % TWO_PI) for p in pos[:, axis]])
            c, s = np.cos(ang), np.sin(ang)
            y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
            size[..., a] = size[..., b] = np.hypot(x[..., a], x[..., b])
            k += 1
        start += n
    return y, size


def scale_of(a):
    """The scale of a group whose largest magnitude is a (float64, a > 0 finite)."""
    m, e = math.frexp(float(np.float32(np.float32(a) / np.float32(7))))
    return min(max(math.ldexp(math.ceil(m * 32) / 32, e), 2.0 ** -126), 2.0 ** 122)


def quantise(x):
    """x [..., d] -> (codes 0..15 int, scales float64 [..., d/32], values float64)."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    a = np.abs(g).max(-1)
    s = np.vectorize(lambda v: math.nan if not math.isfinite(v) else scale_of(v) if v > 0 else 0.0, otypes=[np.float64])(a)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        n = np.rint(g / s[..., None])  # half to even
    n = np.clip(np.nan_to_num(n, nan=0.0), -7, 7)
    n[~np.isfinite(s)] = 0
    v = n * s[..., None]
    return (n + 8).astype(np.int64).reshape(x.shape), s, v.reshape(x.shape)


def code_bytes(codes):
    """Codes [..., d] -> bytes [..., d/2] in the store's layout."""
    w = codes.reshape(*codes.shape[:-1], -1, 8).astype(np.uint64)
    word = np.zeros(w.shape[:-1], np.uint64)
    for i in range(4):
        word |= w[..., 2 * i] << np.uint64(4 * i)
        word |= w[..., 2 * i + 1] << np.uint64(16 + 4 * i)
    return np.ascontiguousarray(word.astype("<u4")).view(np.uint8).reshape(*codes.shape[:-1], -1)


def values_of(code_bytes_, scales):
    """Bytes [..., d/2] and scales [..., d/32] -> float64 values."""
    w = np.ascontiguousarray(code_bytes_).view("<u4").astype(np.int64)
    out = np.zeros((*w.shape, 8))
    for i in range(4):
        out[..., 2 * i] = ((w >> (4 * i)) & 15) - 8
        out[..., 2 * i + 1] = ((w >> (16 + 4 * i)) & 15) - 8
    out = out.reshape(*w.shape[:-1], -1)
    return (out.reshape(*out.shape[:-1], -1, GROUP) * np.asarray(scales, np.float64)[..., None]).reshape(out.shape)


def attention(Q, K, V, q_off, vis, active, scale=None):
    """Q [H_q, rows, d], K / V [H_kv, logical tokens, d], float64.  Returns {row: (O [H_q, d], lse [H_q], sum p|v| [H_q, d],
    largest |q||k| scale)} of the active chunks' rows, stacked per chunk."""
    H_q, _, d = Q.shape
    H_kv = K.shape[0]
    group = H_q // H_kv
    scale = d ** -0.5 if not scale else scale
    O, lse, A = np.zeros_like(Q), np.full(Q.shape[:2], -np.inf), np.zeros_like(Q)
    size = 0.0
    for c in active:
        r = slice(q_off[c], q_off[c + 1])
        n = vis[c]
        if n == 0 or q_off[c] == q_off[c + 1]:
            continue
        for h in range(H_q):
            k, v = K[h // group, :n], V[h // group, :n]
            s = Q[h, r] @ k.T * scale
            m = s.max(-1, keepdims=True)
            p = np.exp(s - m)
            z = p.sum(-1, keepdims=True)
            O[h, r], lse[h, r], A[h, r] = p / z @ v, (m + np.log(z))[:, 0], p / z @ np.abs(v)
            size = max(size, float(np.linalg.norm(Q[h, r], axis=-1).max() * np.linalg.norm(k, axis=-1).max() * scale))
    return O, lse, A, size
