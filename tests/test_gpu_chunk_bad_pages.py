"""Chunk attention over a paged cache with a block mapped outside the pool: whatever the number, it
is flagged, and the block is treated alike."""

import pytest
import torch

from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [1, 2, 4, 8])
def test_every_number_outside_is_flagged(kvq_lib, bits):
    cfg = kvq.CacheConfig(batch=1, n_q_heads=8, n_kv_heads=2, bits_k=bits, bits_v=bits,
                          max_len=512)
    paged = kvq.QuantKVCache(cfg, n_pages=16)
    k, v = synth.kv_heads(5, 2, 400)
    paged.map_blocks(0, range(12), range(12))
    kvq.kvq_pack(paged, k[None].cuda(), v[None].cuda())
    q = synth.queries(6, 4, 8).view(1, 4, 8, 128).cuda()
    kvq.kvq_chunk_attn(paged, q)
    assert paged.flags() == 0
    outs = []
    for page in (-1, 16, 2 ** 31 - 1, -2 ** 31 + 1, -2 ** 31):
        paged.map_blocks(0, [3], [page])
        paged.seq_region()[cfg.batch] = 0
        outs.append(kvq.kvq_chunk_attn(paged, q))
        assert paged.flags() == kvq.FLAG_BAD_PAGE, page
        assert torch.equal(outs[-1], outs[0])
