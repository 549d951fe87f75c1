"""Windows and sinks up to the largest 32-bit number: what holds every token equals the
call without a window."""

import pytest
import torch

import _util
from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.mark.parametrize("n_q", [1, 40])
@pytest.mark.parametrize("window,sinks", [(MOST, 0), (MOST, MOST), (2048, 3), (1, MOST),
                                          (700, MOST - 100), (MOST - 1, 5)])
def test_all_tokens_are_seen(kvq_lib, n_q, window, sinks):
    cfg = kvq.CacheConfig(batch=3, n_q_heads=8, n_kv_heads=2, bits_k=4, bits_v=2, max_len=2048)
    cache, _ = _util.make_cache(cfg, [1500, 20, 0], 11)
    q = synth.queries(12, 3 * n_q, 8).view(3, n_q, 8, 128).cuda()
    want = kvq.kvq_chunk_attn(cache, q).float()
    got = kvq.kvq_chunk_attn(cache, q, window=window, sinks=sinks).float()
    torch.cuda.synchronize()
    assert cache.flags() == 0
    # the work is cut at other tokens: a few fp16 roundings of weights and results
    assert (got - want).abs().max() <= 4 * 2.0 ** -11 * want.abs().max()
