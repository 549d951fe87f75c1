"""Oracle: causal attention of a chunk of new tokens over the low-bit cache,
with an optional sliding window and first tokens that stay visible.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__``).

The n_q queries of a sequence are its last tokens: query t stands at position
p = L - n_q + t and sees token j when 0 <= j <= p and (window == 0 or
j > p - window or j < sinks).  A query that sees nothing (p < 0) gives zero.
Everything is float64 on the dequantized cache.
"""

import numpy as np

from . import quant


def visible(L, n_q, window=0, sinks=0):
    """Boolean [n_q, L]."""
    p = np.arange(L - n_q, L)[:, None]
    j = np.arange(L)[None]
    seen = j <= p
    if window:
        seen &= (j > p - window) | (j < sinks)
    return seen


def chunk_attention(q, heads, window=0, sinks=0, scale=None):
    """One sequence: q [n_q, Hq, 128], heads the Hkv ``quant.quantize_head``
    dicts.  Returns float64 [n_q, Hq, 128] and, of the same shape, the sums of
    p_j |v_j| that rounding errors are measured by."""
    q = np.asarray(q, dtype=np.float64)
    n_q, hq, d = q.shape
    gq = hq // len(heads)
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for h, qh in enumerate(heads):
        khat, vhat = quant.dequantize_head(qh)
        seen = visible(khat.shape[0], n_q, window, sinks)
        live = seen.any(axis=1)
        for i in range(h * gq, (h + 1) * gq):
            s = np.where(seen[live], (q[live, i] @ khat.T) * scale, -np.inf)
            if not s.size:
                continue
            w = np.exp(s - s.max(axis=1, keepdims=True))
            w /= w.sum(axis=1, keepdims=True)
            out[live, i] = w @ vhat
            size[live, i] = w @ np.abs(vhat)
    return out, size


def score_rounding(q, heads, scale=None):
    """The largest change of any score of one sequence when every key is
    rounded to fp16: scale * sum_c |q_c| |k_c| 2^-11, largest over all."""
    q = np.abs(np.asarray(q, dtype=np.float64))
    n_q, hq, d = q.shape
    gq = hq // len(heads)
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    worst = 0.0
    for h, qh in enumerate(heads):
        khat, _ = quant.dequantize_head(qh)
        if khat.shape[0]:
            s = q[:, h * gq:(h + 1) * gq].reshape(-1, d) @ np.abs(khat).T
            worst = max(worst, s.max() * scale * 2.0 ** -11)
    return worst
