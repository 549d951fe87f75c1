"""Flat rows whose kept part outgrows the list, temperatures at the ends of the range,
rows whose sampled logits say nothing: every row's token is one that the limits keep
and its key within 1e-4 of the best, at least nine rows in ten have a winner that leads
by more and take it, and every row's logprob is its token's.

The limits are those of include/kvq.h in 64 bits.  A token at the very end of what
top-p keeps may go either way: its predecessors' share is within 1e-5 of p."""

import numpy as np
import pytest
import torch

from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu


def _kept(z, T, k, p, slack):
    """Ids kept by top-k, then top-p (p widened by slack), in the order of the tokens."""
    order = np.argsort(-z, kind="stable")
    order = order[z[order] > -np.inf]
    w = np.exp((z[order] - z[order[0]]) / T)
    if k > 0:
        order, w = order[:k], w[:k]
    if p < 1:
        n = int((np.cumsum(w) - w < (p + slack) * w.sum()).sum())
        order = order[:max(n, 1)]
    return order


def _compare(z, u, T, k, p):
    B = z.shape[0]
    dev = [torch.tensor(x, dtype=d).cuda() for x, d in (
        (T, torch.float32), (k, torch.int32), (p, torch.float32))]
    r = kvq.kvq_sample(z.cuda(), u.cuda(), *dev)
    token, logprob = r["token"].cpu().numpy(), r["logprob"].cpu().numpy()
    compared = 0
    for b in range(B):
        x = z[b].numpy().astype(np.float64)
        t = min(max(float(np.float32(T[b])), 1e-30), 1e30)
        d = (x - x.max()) / t
        key = d - np.log(-np.log(u[b].numpy().astype(np.float64)))
        sure = _kept(x, t, k[b], float(np.float32(p[b])), -1e-5)
        may = _kept(x, t, k[b], float(np.float32(p[b])), 1e-5)
        assert token[b] in may
        assert key[token[b]] >= key[sure].max() - 1e-4
        top = np.sort(key[may])[-2:]
        if len(top) < 2 or top[1] - top[0] > 1e-4:
            compared += 1
            best = may[np.argmax(key[may])]
            assert token[b] == best or best not in sure
        want = d[token[b]] - np.log(np.exp(d).sum())
        assert abs(logprob[b] - want) <= 1e-5 + 1e-6 * abs(want)
    assert compared >= 0.9 * B


@pytest.mark.parametrize("B", [2, 20, 40, 90])
def test_flat_rows(kvq_lib, B):
    z = synth.logits(3, B, 150001, sigma=0.7)
    u = torch.rand(z.shape, generator=synth.generator(4)).clamp_min(1e-7)
    p = ([0.99, 0.999, 0.5, 0.9, 1.0] * (B // 5 + 1))[:B]
    k = ([0, 100000, 0, 60000, 30000] * (B // 5 + 1))[:B]
    _compare(z, u, [1.0] * B, k, p)


@pytest.mark.parametrize("V", [500, 40000])
def test_temperatures(kvq_lib, V):
    T = [float("inf"), 1e38, 1e-38, 1e-44, 1e-20, 1e20, 0.7, 1.3, 5.0, 40.0]
    z = synth.logits(1, len(T), V)
    z[:, ::7] = -np.inf
    u = torch.rand(z.shape, generator=synth.generator(2)).clamp_min(1e-7)
    _compare(z, u, T, [0] * 10, [1.0] * 10)
    _compare(z, u, T, [20] * 10, [0.7] * 10)


@pytest.mark.parametrize("masked", [-np.inf, -1e9])
def test_unsampled_rows(kvq_lib, masked):
    V = 100000
    z = torch.full((4, V), masked)
    z[0, 20000] = 1.0
    z[1, [30001, 99]] = torch.tensor([2.0, 1.5])
    z[2, 50000:50100] = synth.logits(5, 1, 100)[0]
    z[3] = synth.logits(6, 1, V)[0]
    z[3, 20001] = 300.0
    u = torch.rand(z.shape, generator=synth.generator(7)).clamp_min(1e-7)
    _compare(z, u, [1.0] * 4, [0, 0, 30, 0], [1.0, 0.9, 0.8, 0.9])
    _compare(z, u, [1.0] * 4, [0] * 4, [1.0] * 4)
