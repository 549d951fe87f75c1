"""kvq_sample against the float64 oracle.

A row's token must be the oracle's wherever the oracle's winner leads by more
than 1e-4 (keys of about 10 in fp32: a few 1e-6 of rounding), and every seeded
row here does unless it is skipped by that rule; logprob within 1e-5 absolute
+ 1e-6 relative (fp32 exp, exact sums).
"""

import numpy as np
import pytest
import torch

from oracle import sample as osample
from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu


def _noise(seed, B, V):
    return torch.rand(B, V, generator=synth.generator(seed))


def _dev(x, dtype=torch.float32):
    return None if x is None else torch.as_tensor(x, dtype=dtype).cuda()


def _check(z, u, T=None, k=None, p=None, m=None, strided=False):
    B, V = z.shape
    zd, ud = z.cuda(), (None if u is None else u.cuda())
    if strided:
        hold = torch.full((2, B, V + 5), 50.0, device="cuda")
        hold[:, :, 1:V + 1] = torch.stack([zd, ud])
        zd, ud = hold[0, :, 1:V + 1], hold[1, :, 1:V + 1]
    r = kvq.kvq_sample(zd, ud, _dev(T), _dev(k, torch.int32), _dev(p), _dev(m))
    tok, lp = r["token"].cpu().numpy(), r["logprob"].cpu().numpy()
    compared = 0
    for b in range(B):
        f = [np.float32(x[b]) if x is not None else d for x, d in ((T, 1.0), (p, 1.0), (m, 0.0))]
        t, l, margin = osample.sample_row(z[b].numpy(), None if u is None else u[b].numpy(), f[0],
                                          k[b] if k is not None else 0, f[1], f[2])
        if margin > 1e-4 or margin == 0:      # 0: equal logits with equal numbers
            compared += 1
            assert tok[b] == t, (b, tok[b], t)
            if np.isinf(l):
                assert lp[b] == l
            else:
                assert abs(lp[b] - l) <= 1e-5 + 1e-6 * abs(l), (b, lp[b], l)
    assert compared >= 0.9 * B
    return r


@pytest.mark.parametrize("V", [1, 2, 7, 31, 32, 1000, 4097, 32000, 128256, 152063, 262144])
def test_vocabularies(kvq_lib, V):
    B = 5
    z = synth.logits(V, B, V)
    k = [0, 1, 3, 50, V]
    _check(z, _noise(V + 1, B, V), [1.0, 0.7, 1.3, 0.8, 2.0], k, [0.9, 1.0, 0.5, 0.95, 0.99],
           [0.0, 0.0, 0.1, 0.0, 0.01])


@pytest.mark.parametrize("what", ["none", "k", "p", "m", "all"])
def test_each_limit(kvq_lib, what):
    B, V = 24, 5003
    z, u = synth.logits(3, B, V), _noise(4, B, V)
    k = [1 + 7 * b * b for b in range(B)] if what in ("k", "all") else None
    p = [0.02 + 0.04 * b for b in range(B)] if what in ("p", "all") else None
    m = [0.5 ** (1 + b % 12) for b in range(B)] if what in ("m", "all") else None
    _check(z, u, None if what == "none" else [0.5 + 0.1 * b for b in range(B)], k, p, m)


def test_limits_beyond_their_ranges(kvq_lib):
    """k <= 0 and p >= 1 and m <= 0 keep all; p <= 0 and m > 1 the first token;
    T <= 0 is greedy."""
    z, u = synth.logits(5, 10, 3001), _noise(6, 10, 3001)
    _check(z, u, [1, 1, 1, 1, 1, 0, -1, 1e-3, 1e4, 1], [-4, 0, 0, 9999999, 0, 0, 5, 0, 0, 2],
           [1.0, 1.5, 0.0, -1.0, 1.0, 1.0, 1.0, 0.9, 0.5, 1.0], [-1, 0, 0, 0, 1.5, 0, 0, 0, 0, 1.0])


def test_greedy_without_noise(kvq_lib):
    z = synth.logits(7, 6, 20011)
    r = _check(z, None, [1.0, 0.5, 0, 2, 1, 1], [3] * 6)
    assert r["token"].cpu().tolist() == z.argmax(-1).tolist()


def test_ties(kvq_lib):
    """Equal values go by index: limits cut inside runs of equal logits, whole
    rows are equal, +0 ties with -0."""
    V = 4099
    z = torch.stack([torch.zeros(V), torch.randint(0, 3, (V,), generator=synth.generator(8)).float(),
                     torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0), torch.full((V,), -7.5)])
    u = _noise(9, 4, V)
    for k in (1, 2, 31, 1000, V - 1):
        _check(z, u, None, [k] * 4)
    for p in (0.001, 0.3, 0.99):
        _check(z, u, None, None, [p] * 4)
    _check(z, u, None, [700] * 4, [0.5] * 4)
    _check(z, torch.full((4, V), 0.5), None, [100] * 4)      # equal keys: the lowest index
    big = torch.zeros(2, 200000)
    big[1, 77777] = 1.0
    _check(big, _noise(10, 2, 200000), None, [123456, 150001], [0.7, 0.25])


def test_forbidden_tokens(kvq_lib):
    """-inf is never taken; a row of -inf alone gives -1; one free token."""
    V = 3001
    z = synth.logits(11, 6, V)
    z[0] = -np.inf
    z[1] = -np.inf
    z[1, V - 1] = -3.0
    z[2, :V - 2] = -np.inf
    z[3, ::2] = -np.inf
    z[4, 1::2] = -np.inf
    u = _noise(12, 6, V)
    r = _check(z, u, [1.0] * 6, [0, 0, 5, 2000, 0, 0], [1, 1, 1, 1, 0.999, 1])
    assert r["token"][:2].cpu().tolist() == [-1, V - 1]


def test_extreme_noise_and_logits(kvq_lib):
    """u = 0 is never preferred but a lone kept token is taken all the same;
    u just below 1; logits of 1e30 and spreads that underflow."""
    V = 1000
    z = synth.logits(13, 4, V)
    u = _noise(14, 4, V)
    u[0] = 0.0
    u[1] = 1.0 - 2.0 ** -24
    z[2] *= 1e30
    z[3] *= 40.0
    z[3, 10] = 3e38
    _check(z, u, [1.0] * 4, [1, 0, 0, 0])


def test_strided_rows(kvq_lib):
    _check(synth.logits(15, 7, 30001), _noise(16, 7, 30001), [0.9] * 7, [40] * 7, [0.9] * 7,
           strided=True)


def test_frequencies(kvq_lib):
    """20000 draws from one row follow its renormalised probabilities: each
    count within 5 standard deviations."""
    V, N = 64, 20000
    z = synth.logits(17, 1, V, sigma=1.0)
    zz = z.cuda().expand(N, V).contiguous()
    u = torch.rand(N, V, generator=synth.generator(18)).cuda()
    r = kvq.kvq_sample(zz, u, torch.full((N,), 0.9, device="cuda"),
                       torch.full((N,), 20, dtype=torch.int32, device="cuda"),
                       torch.full((N,), 0.9, device="cuda"))
    n = torch.bincount(r["token"].long().cpu(), minlength=V).numpy()
    keep = osample.kept(z[0].numpy(), np.float32(0.9), 20, np.float32(0.9))
    p = np.zeros(V)
    p[keep] = np.exp(z[0].numpy().astype(np.float64)[keep] / 0.9)
    p /= p.sum()
    assert n[p == 0].sum() == 0
    assert (np.abs(n - N * p) <= 5 * np.sqrt(N * p * (1 - p)) + 1).all()


def test_many_rows_repeat_and_stream(kvq_lib):
    B, V = 700, 8000
    z, u = synth.logits(19, B, V), _noise(20, B, V)
    p = [0.9] * B
    r = _check(z, u, None, None, p)
    side = torch.cuda.Stream()
    zd, ud, pd = z.cuda(), u.cuda(), _dev(p)
    side.wait_stream(torch.cuda.current_stream())
    o = kvq.kvq_sample(zd, ud, top_p=pd, outputs=dict(token=torch.empty_like(r["token"]),
                                                      logprob=None), stream=side)
    side.synchronize()
    assert torch.equal(o["token"], r["token"])
