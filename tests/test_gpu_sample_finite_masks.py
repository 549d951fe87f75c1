"""Draws without limits from rows whose few free tokens stand far above all others:
forbidden tokens masked by a finite number, wherever the free ones stand.

The reference is the definition in 64 bits: the largest (z - max z) / T -
ln(-ln u).  Its token is required wherever it leads by more than 1e-4: a key is
below 50 where it can win, and three fp32 roundings of it are below 1e-5.  The
logprob: 1e-5 + 1e-6 relative (fp32 exp of each term, sums exact or in fp32 of what
weighs nothing)."""

import numpy as np
import pytest
import torch

from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu

LOWEST = float(np.finfo(np.float32).min)


def _compare(z, u, T):
    got = kvq.kvq_sample(z.cuda(), u.cuda(), torch.full((z.shape[0],), T, device="cuda"))
    token, logprob = got["token"].cpu().numpy(), got["logprob"].cpu().numpy()
    compared = 0
    for b in range(z.shape[0]):
        x = z[b].numpy().astype(np.float64)
        d = (x - x.max()) / float(np.float32(T))
        with np.errstate(divide="ignore"):
            key = d - np.log(-np.log(u[b].numpy().astype(np.float64)))
        first, second = np.argsort(-key, kind="stable")[:2]
        # a near-tie may go either way, to no third token
        assert token[b] in (first, second)
        if key[first] - key[second] > 1e-4:
            compared += 1
            assert token[b] == first
        want = d[token[b]] - np.log(np.exp(d).sum())
        assert abs(logprob[b] - want) <= 1e-5 + 1e-6 * abs(want)
    assert compared >= 0.9 * z.shape[0]


@pytest.mark.parametrize("mask", [-20.0, -40.0, -1e4, -1e7, -1e8, -1e9, LOWEST])
@pytest.mark.parametrize("V", [8200, 16384, 20480, 128256])
def test_masked_by_a_number(kvq_lib, V, mask):
    """50 free tokens at places spread over the row; batches that take eight, four,
    two and one CTAs a row."""
    for B in (6, 20, 40, 90):
        z = torch.full((B, V), mask)
        free = synth.logits(V + B, B, 50)
        for b in range(B):
            at = (1100 + (7919 * b) % (V - 1200)) if b else 1100
            z[b, at:at + 50] = free[b]
        _compare(z, torch.rand(z.shape, generator=synth.generator(B)), 1.0)


@pytest.mark.parametrize("V", [16384, 128256])
def test_additive_masks(kvq_lib, V):
    """A number added to ordinary logits of the forbidden tokens; temperatures that
    make it small and large."""
    B = 6
    z = synth.logits(V, B, V)
    kept = z[:, 1100:1150].clone()
    z -= 1e7
    z[:, 1100:1150] = kept
    u = torch.rand(z.shape, generator=synth.generator(3))
    for T in (0.3, 1.0, 5.0):
        _compare(z, u, T)


@pytest.mark.parametrize("lead", [5.0, 30.0, 34.0, 100.0, 3e4, 1e30])
def test_one_token_far_ahead(kvq_lib, lead):
    V = 128256
    z = synth.logits(4, 6, V)
    z[:, 20001] = lead
    _compare(z, torch.rand(z.shape, generator=synth.generator(5)), 1.0)
