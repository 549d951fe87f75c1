"""kvq_sample at temperatures whose reciprocal is not finite, on flat rows whose
kept part outgrows the list, and on rows whose sampled logits say nothing.

The token must be the float64 oracle's wherever its winner leads by more than
1e-4; logprob within 1e-5 + 1e-6 relative."""

import numpy as np
import pytest
import torch

from oracle import sample as osample
from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu


def _compare(z, u, T, k, p, m):
    B, V = z.shape
    dev = [torch.tensor(x, dtype=d).cuda() for x, d in (
        (T, torch.float32), (k, torch.int32), (p, torch.float32), (m, torch.float32))]
    r = kvq.kvq_sample(z.cuda(), u.cuda(), *dev)
    tok, lp = r["token"].cpu().numpy(), r["logprob"].cpu().numpy()
    for b in range(B):
        t = min(max(T[b], 1e-30), 1e30) if T[b] > 0 else T[b]     # the documented range
        want, logp, margin = osample.sample_row(z[b].numpy(), u[b].numpy(), np.float32(t), k[b],
                                                np.float32(p[b]), np.float32(m[b]))
        if margin > 1e-4:
            assert tok[b] == want, (b, tok[b], want)
            assert abs(lp[b] - logp) <= 1e-5 + 1e-6 * abs(logp), (b, lp[b], logp)


@pytest.mark.parametrize("V", [500, 40000])
def test_temperatures_at_the_ends(kvq_lib, V):
    T = [float("inf"), 1e38, 1e-38, 1e-44, 1e-20, 1e20]
    z = synth.logits(1, len(T), V)
    z[:, ::7] = -np.inf
    u = torch.rand(z.shape, generator=synth.generator(2))
    _compare(z, u, T, [0] * 6, [1.0] * 6, [0.0] * 6)
    _compare(z, u, T, [20] * 6, [0.7] * 6, [0.0] * 6)


@pytest.mark.parametrize("B", [2, 20, 40, 90])
def test_flat_rows_go_beyond_the_list(kvq_lib, B):
    """Limits that keep most of a long, flat row, for every number of CTAs a row."""
    V = 150001
    z = synth.logits(3, B, V, sigma=0.7)
    u = torch.rand(z.shape, generator=synth.generator(4))
    p = [0.99, 0.999, 0.5, 0.9, 1.0] * (B // 5 + 1)
    k = [0, 100000, 0, 60000, 30000] * (B // 5 + 1)
    _compare(z, u, [1.0] * B, k[:B], p[:B], [0.0] * B)


def test_the_sample_misses_every_free_token(kvq_lib):
    """One, two and a hundred free tokens in a row of forbidden ones, at places
    that the eight sampled stretches do not hold; a peak far above the rest."""
    V = 100000
    z = torch.full((4, V), -np.inf)
    z[0, 20000] = 1.0
    z[1, [30001, 99]] = torch.tensor([2.0, 1.5])
    z[2, 50000:50100] = synth.logits(5, 1, 100)[0]
    z[3] = synth.logits(6, 1, V)[0]
    z[3, 20001] = 300.0
    u = torch.rand(z.shape, generator=synth.generator(7))
    _compare(z, u, [1.0] * 4, [0, 0, 30, 0], [1.0, 0.9, 0.8, 0.9], [0.0] * 4)
    _compare(z, u, [0.5] * 4, [2] * 4, [1.0] * 4, [0.3] * 4)
    _compare(z, u, [1.0] * 4, [0] * 4, [1.0] * 4, [0.0] * 4)
