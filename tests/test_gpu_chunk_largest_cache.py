"""kvq_chunk_attn on a cache declared with the largest max_len, 2^31 - 32 (paged, so
that nothing but the block table has that many entries): windows and sinks up to the
largest 32-bit numbers against the float64 oracle, with the tolerance of the other
chunk tests (1.5e-3 of the results' rms)."""

import numpy as np
import pytest
import torch

import _util
from oracle import chunk as ochunk
from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def largest(kvq_lib):
    cfg = kvq.CacheConfig(batch=1, n_q_heads=4, n_kv_heads=1, bits_k=4, bits_v=4,
                          max_len=2 ** 31 - 32)
    cache = kvq.QuantKVCache(cfg, n_pages=32)
    k, v = synth.kv_heads(21, 1, 700)
    blocks = kvq.blocks_written(0, 700)
    cache.map_blocks(0, blocks, list(blocks))
    kvq.kvq_pack(cache, k[None].cuda(), v[None].cuda())
    return cfg, cache, _util.oracle_heads(cfg, k, v)


@pytest.mark.parametrize("n_q", [1, 40, 900])
@pytest.mark.parametrize("window,sinks", [(0, 0), (5, MOST), (MOST, MOST), (MOST, 0),
                                          (2 ** 31 - 200, 7), (1, 2 ** 31 - 100), (300, 40)])
def test_largest_numbers(largest, n_q, window, sinks):
    cfg, cache, heads = largest
    q = synth.queries(22, n_q, 4).view(1, n_q, 4, 128)
    out = kvq.kvq_chunk_attn(cache, q.cuda(), window=window, sinks=sinks)
    got = out.double().cpu().numpy()[0]
    assert cache.flags() == 0
    ref, _ = ochunk.chunk_attention(q[0].numpy(), heads, window, sinks)
    assert (got[:max(0, n_q - 700)] == 0).all()
    assert np.sqrt(((got - ref) ** 2).mean()) <= 1.5e-3 * np.sqrt((ref ** 2).mean())
