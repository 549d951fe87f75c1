"""A wait of the chunk attention's roles that runs out is reported whichever role
waited, frees the others, and leaves the context usable."""

import time

import pytest
import torch

import _util
from oracle import chunk as ochunk
from paper_2607_16248_gb300 import build, kvq, synth


@pytest.mark.gpu
@pytest.mark.parametrize("role", [0, 1, 2])
def test_every_role_reports(kvq_lib, role):
    kvq.selftest_chunk_wait_timeout(role)      # loads the kernel
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    flag = kvq.selftest_chunk_wait_timeout(role)
    torch.cuda.synchronize()
    # 10 ms, where the other roles' own limit is about a second
    assert time.perf_counter() - t0 < 0.4
    assert int(flag.item()) == kvq.FLAG_WAIT_TIMEOUT
    cfg = kvq.CacheConfig(batch=1, n_q_heads=8, n_kv_heads=2, bits_k=2, bits_v=2, max_len=1024)
    cache, kv = _util.make_cache(cfg, [700], 3)
    q = synth.queries(4, 9, 8).view(1, 9, 8, 128)
    out = kvq.kvq_chunk_attn(cache, q.cuda())[0].double().cpu()
    ref, _ = ochunk.chunk_attention(q[0].numpy(), _util.oracle_heads(cfg, *kv[0]))
    assert cache.flags() == 0
    ref = torch.from_numpy(ref)
    assert (out - ref).pow(2).mean().sqrt() <= 1.5e-3 * ref.pow(2).mean().sqrt()


def test_refusals():
    build.build()
    for role, flag, status in ((3, 0x100000, 1), (-1, 0x100000, 1), (0, None, 1),
                               (0, 0x100002, 5)):
        assert kvq.lib().kvq_selftest_chunk_wait_timeout(role, flag, None) == status
