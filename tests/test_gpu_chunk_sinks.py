"""Rows whose first token takes nearly all the weight and has no value: the result is
the tail, thousands of tokens that weigh a millionth of the first.

A query is 4 s + noise for a vector of signs s, the first key c s, the other keys lie
across s; c puts the first token's score about 15 nats above the others', so that it
has 0.997 to 0.9995 of the weight of 4096 tokens (0.99 or less of few).  The other
values have deviation 200, so results are normal fp16 numbers.

Bound on the rms error, relative to the results' rms: rounding of the keys changes
the tail's weights by 6e-4 and the first token's score (15 nats, 128 equal terms of
relative error 2^-11 / sqrt(3)) by 4e-4; rounding of the weights, which leave with
2^7 as the first token's, 2^-24 / sqrt(12) of their spacing below 2^-14 against a
mean of 2^-15: 6e-4; the result's own rounding 2e-4.  In all 9e-4; 2.5e-3 is asked.
Without the factor 2^7 the third part would be 7e-2."""

import math

import numpy as np
import pytest
import torch

import _util
from oracle import chunk as ochunk
from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bk,bv", [(8, 8), (8, 2), (4, 4)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (3000, 4)])
@pytest.mark.parametrize("n_q", [64, 5])
def test_first_token_without_value(kvq_lib, bk, bv, window, sinks, n_q):
    L, hq, hkv, batch = 4096, 32, 8, 19
    cfg = kvq.CacheConfig(batch=batch, n_q_heads=hq, n_kv_heads=hkv, bits_k=bk, bits_v=bv,
                          max_len=L)
    g = synth.generator(5)
    s = torch.sign(torch.randn(128, generator=g))
    k = 0.5 * torch.randn(hkv, L, 128, generator=g)
    k -= (k @ s)[..., None] * s / 128
    ahead = math.log(0.999 / 0.001 * (window or L))
    k[:, 0] = ahead / (4 * 128 / math.sqrt(128)) * s
    v = 200.0 * torch.randn(hkv, L, 128, generator=g)
    v[:, 0] = 0.0
    k, v = k.half(), v.half()
    q = (4 * s + torch.randn(n_q, hq, 128, generator=g)).half()
    cache = kvq.QuantKVCache(cfg)
    kvq.kvq_pack(cache, k.cuda().expand(batch, -1, -1, -1).contiguous(),
                 v.cuda().expand(batch, -1, -1, -1).contiguous())
    out = kvq.kvq_chunk_attn(cache, q.cuda().expand(batch, -1, -1, -1), window=window,
                             sinks=sinks)
    torch.cuda.synchronize()
    assert cache.flags() == 0
    ref, _ = ochunk.chunk_attention(q.numpy(), _util.oracle_heads(cfg, k, v), window, sinks)
    rms = np.sqrt((ref ** 2).mean())
    assert rms > 1e-3
    for b in (0, batch - 1):
        err = np.sqrt(((out[b].double().cpu().numpy() - ref) ** 2).mean())
        assert err <= 2.5e-3 * rms, f"{err / rms:.3g}"
