"""Oracle: the next token by temperature, top-k, top-p and min-p from given
random numbers, in float64.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__``).

Tokens are ordered by value descending, lowest index first.  With
d = (z - max z) / T and e = exp(d): the first k; of those, the tokens whose
predecessors hold less than p times their e-sum; of those, the tokens with
e >= m; the first token in any case, -inf never.  The token is the kept one
with the largest d - ln(-ln u).  T <= 0 is greedy.
"""

import numpy as np


def kept(z, T=1.0, k=0, p=1.0, m=0.0):
    """Kept token ids in the order of the tokens."""
    z = np.asarray(z, dtype=np.float64)
    order = np.argsort(-z, kind="stable")
    if not T > 0:
        return order[:1]
    first = order[0]
    e = np.exp((z - z[first]) / T)
    if k > 0:
        order = order[:k]
    if p < 1:
        w = e[order]
        n = int((np.cumsum(w) - w < p * w.sum()).sum()) if p > 0 else 1
        order = order[:max(n, 1)]
    return np.array([i for i in order if (e[i] >= m or i == first) and z[i] > -np.inf])


def sample_row(z, u, T=1.0, k=0, p=1.0, m=0.0):
    """(token, logprob, margin): margin is how far the winning key is ahead of
    the next kept one's (inf where there is none)."""
    z = np.asarray(z, dtype=np.float64)
    zmax = z.max()
    if zmax == -np.inf:
        return -1, -np.inf, np.inf
    d = (z - zmax) / (T if T > 0 else 1.0)
    lse = np.log(np.exp(d).sum())
    ids = np.sort(kept(z, T, k, p, m))
    if u is None:
        ids = kept(z, 0.0)
        key = np.zeros(1)
    else:
        with np.errstate(divide="ignore"):
            key = d[ids] - np.log(-np.log(np.asarray(u, dtype=np.float64)[ids]))
    i = int(np.argmax(key))
    rest = np.delete(key, i)
    margin = float(key[i] - rest.max()) if rest.size and np.isfinite(rest.max()) else np.inf
    return int(ids[i]), float(d[ids[i]] - lse), margin
