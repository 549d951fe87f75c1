"""64-bit oracle of the block-8 cache (append with rotation, attention) and of
adjusted logits, written from the definitions in include/kvq.h."""

import numpy as np

BLOCK, RING = 32, 64


def to_bits(x, bits, least):
    """x (float64) to the nearest number of `bits` significant bits with steps of at
    least 2^least, ties to even."""
    x = np.asarray(x, dtype=np.float64)
    _, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - bits, least))
    return np.rint(x / step) * step


def to_type(x, dtype):
    """x rounded to "fp16", "bf16", "fp32" or "e4m3" (as float64)."""
    bits, least = {"fp16": (11, -24), "bf16": (8, -133), "fp32": (24, -149), "e4m3": (4, -9)}[dtype]
    y = to_bits(x, bits, least)
    return np.clip(y, -448.0, 448.0) if dtype == "e4m3" else y


def rotate(x, cos, sin, paired):
    """x [T, H, 128] rotated by cos, sin [T, r]."""
    x, r = np.array(x, dtype=np.float64), cos.shape[1]
    a, b = (slice(0, 2 * r, 2), slice(1, 2 * r, 2)) if paired else (slice(0, r), slice(r, 2 * r))
    c, s = cos[:, None].astype(np.float64), sin[:, None].astype(np.float64)
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def quantize(x):
    """(codes as values, scale) of one block x [32, 128]."""
    m = np.abs(x).max()
    s = float(np.clip(to_type(m / 448.0, "fp32"), 2.0 ** -60, 2.0 ** 60)) if m > 0 else 1.0
    return to_type(to_type(x / s, "fp32"), "e4m3"), s


class Sequence:
    """The keys or values of one (sequence, kv-head), as a cache keeps them: every token in
    its 16-bit type (keys rotated)."""

    def __init__(self):
        self.rows = np.zeros((0, 128))

    def append(self, rows, length):
        """Tokens [length - len(rows), length); whatever stood there is replaced."""
        self.rows = np.concatenate([self.rows[:length - len(rows)], rows])

    def seen(self):
        """All tokens as attention sees them."""
        full = len(self.rows) // BLOCK * BLOCK
        out = self.rows.copy()
        for t in range(0, full, BLOCK):
            c, s = quantize(self.rows[t:t + BLOCK])
            out[t:t + BLOCK] = c * s
        return out


def attend(q, k, v, scale=None, window=0, sinks=0):
    """q [n, gq, 128] of the newest n tokens over k, v [L, 128] (as seen): out, and for an
    error bound the weighted magnitudes sum_j p_j |v_j|."""
    n, gq, d = q.shape
    L = len(k)
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out = np.zeros((n, gq, d))
    size = np.zeros((n, gq, d))
    j = np.arange(L)
    for t in range(n):
        p = L - n + t
        if p < 0:
            continue
        seen = j <= p
        if window:
            seen &= (j > p - window) | (j < sinks)
        s = (q[t].astype(np.float64) @ k[seen].T) * scale
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        out[t], size[t] = w @ v[seen], w @ np.abs(v[seen])
    return out, size


def adjust(z, history=(), prompt=0, repetition=1.0, frequency=0.0, presence=0.0, bias=(),
           allowed=None):
    """One row: history a list of ids, bias a list of (id, value), allowed a bool array."""
    z = np.array(z, dtype=np.float64)
    V = len(z)
    rep = float(repetition) if repetition > 0 else 1.0
    for i in set(h for h in history if 0 <= h < V):
        z[i] = z[i] / rep if z[i] > 0 else z[i] * rep
    said = [h for h in history[max(0, prompt):] if 0 <= h < V]
    for i in set(said):
        z[i] -= float(frequency) * said.count(i) + float(presence)
    for i, x in dict(bias).items():
        if 0 <= i < V:
            z[i] += x
    if allowed is not None:
        z[~np.asarray(allowed)] = -np.inf
    return z
