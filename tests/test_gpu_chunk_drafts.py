"""Drafts that are verified and dropped again, by the rule of include/kvq.h: with no
group leaving the window behind the first token of the call, every query sees what a
decode step sees, and after the length is lowered the cache is as if the drafts had
never been there, bit for bit."""

import pytest
import torch

import _util
from paper_2607_16248_gb300 import kvq, synth

RESIDUAL = 128


def _room(L):
    """The most tokens of a call on a sequence of L whose drafts may be dropped."""
    n = 1
    while n < 40 and not kvq.blocks_written(L + 1, n, RESIDUAL):
        n += 1
    return n


def test_the_rule_leaves_room():
    """The call's first token may finish a group, a draft may not: 32 tokens after it
    has, down to one just before."""
    assert [_room(L) for L in (0, 126, 127, 128, 157, 158, 159, 160, 191)] == \
        [40, 33, 32, 31, 2, 1, 32, 31, 32]


@pytest.mark.gpu
@pytest.mark.parametrize("bk,bv", [(1, 1), (2, 4)])
@pytest.mark.parametrize("L", [1, 126, 158, 159, 160, 187, 500, 511])
@pytest.mark.parametrize("paged", [False, True])
def test_dropped_drafts_leave_no_trace(kvq_lib, bk, bv, L, paged):
    cfg = kvq.CacheConfig(batch=1, n_q_heads=8, n_kv_heads=2, bits_k=bk, bits_v=bv, max_len=768)
    n = min(_room(L), 7)
    k, v = (x[None].cuda() for x in synth.kv_heads(31, 2, 700))
    dk, dv = (x[None].cuda() for x in synth.kv_heads(32, 2, n))
    q = synth.queries(33, n, 8).view(1, n, 8, 128).cuda()

    def made():
        cache = kvq.QuantKVCache(cfg, n_pages=24 if paged else None)
        if paged:
            cache.map_blocks(0, range(24), range(24))
        kvq.kvq_pack(cache, k[:, :, :L].contiguous(), v[:, :, :L].contiguous())
        return cache

    cache, plain = made(), made()
    kvq.kvq_pack(cache, dk, dv)
    got = kvq.kvq_chunk_attn(cache, q)
    # each query against a decode step's view
    step = made()
    for t in range(n):
        kvq.kvq_pack(step, dk[:, :, t:t + 1].contiguous(), dv[:, :, t:t + 1].contiguous())
        one = kvq.kvq_chunk_attn(step, q[:, t:t + 1].contiguous())
        # other cuts of the same sums: a few fp16 roundings of weights and results
        diff = (one.float() - got[:, t:t + 1].float()).abs().max()
        assert diff <= 4 * 2.0 ** -11 * one.float().abs().max(), t
    # keep the first token and half of the drafts
    keep = L + 1 + (n - 1) // 2
    cache.seq_lens()[0] = keep
    kvq.kvq_pack(plain, dk[:, :, :keep - L].contiguous(), dv[:, :, :keep - L].contiguous())
    for m in (1, 2, 30, 3, 1):
        at = int(plain.seq_lens()[0])
        for c in (cache, plain):
            kvq.kvq_pack(c, k[:, :, at:at + m].contiguous(), v[:, :, at:at + m].contiguous())
        qq = synth.queries(at, m, 8).view(1, m, 8, 128).cuda()
        assert torch.equal(kvq.kvq_chunk_attn(cache, qq), kvq.kvq_chunk_attn(plain, qq))
        a = kvq.kvq_decode_attn(cache, qq[:, -1].contiguous())
        assert torch.equal(a, kvq.kvq_decode_attn(plain, qq[:, -1].contiguous()))
    total = int(plain.seq_lens()[0])
    for h in range(2):
        _util.assert_head_equal(_util.head_arrays(cache, 0, h, total),
                                _util.head_arrays(plain, 0, h, total))
    assert cache.flags() == 0
