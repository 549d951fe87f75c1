"""Rows with fewer free tokens than top_k keeps, together with top_p: both limits are
looked for in the same counts, and the first is not reached.  The second search must
not write its result while the first one's is still being read; that is looked up in
the source, the tokens are compared on the GPU.

Tokens are the float64 oracle's wherever its winner leads by more than 1e-4; logprob
within 1e-5 + 1e-6 relative, as in the other sampling tests."""

import re
from pathlib import Path

import numpy as np
import pytest
import torch

from oracle import sample as osample
from paper_2607_16248_gb300 import kvq, synth

SOURCE = Path(__file__).resolve().parents[1] / "paper_2607_16248_gb300" / "csrc" / "sample.cu"


def test_every_search_result_is_read_behind_a_barrier():
    """In threshold(), between the read of s.range and the first return stands a
    barrier: find_range of the next limit writes s.range."""
    text = re.sub(r"//.*", "", SOURCE.read_text())
    body = text[text.index("__device__ u64 threshold("):]
    body = body[body.index("= s.range;"):]
    assert "__syncthreads();" in body[:body.index("return")]


@pytest.mark.gpu
@pytest.mark.parametrize("free", [1, 20, 300])
@pytest.mark.parametrize("B,V", [(1, 128256), (3, 128256), (20, 50000), (40, 50000), (90, 50000),
                                 (5, 3000)])
def test_more_asked_than_free(kvq_lib, free, B, V):
    z = torch.full((B, V), -np.inf)
    logits = synth.logits(V + free, B, free)
    g = synth.generator(free)
    for b in range(B):
        z[b, torch.randperm(V, generator=g)[:free]] = logits[b]
    u = torch.rand(z.shape, generator=synth.generator(7))
    k, p, T = free + 30, np.float32(0.95), np.float32(0.8)
    got = kvq.kvq_sample(z.cuda(), u.cuda(), torch.full((B,), float(T), device="cuda"),
                         torch.full((B,), k, dtype=torch.int32, device="cuda"),
                         torch.full((B,), float(p), device="cuda"))
    token, logprob = got["token"].cpu().numpy(), got["logprob"].cpu().numpy()
    compared = 0
    for b in range(B):
        at = torch.nonzero(z[b] > -np.inf)[:, 0].numpy()
        # the free tokens alone, in their order: the others change nothing
        want, logp, margin = osample.sample_row(z[b].numpy()[at], u[b].numpy()[at], T, k, p)
        assert token[b] in at[osample.kept(z[b].numpy()[at], T, k, p)]
        if margin > 1e-4:
            compared += 1
            assert token[b] == at[want]
            assert abs(logprob[b] - logp) <= 1e-5 + 1e-6 * abs(logp)
    assert compared >= 0.9 * B
