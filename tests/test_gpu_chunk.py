"""kvq_chunk_attn against the float64 oracle.

Tolerances (before any run): with E the largest change of a score when keys
are rounded to fp16, a weight changes by at most a factor e^(2E); values,
weights and the result are rounded once each (2^-11 relative each, 2^-12 of
rounding to nearest is not relied on), and fp32 accumulation of up to 2^17
terms in tensor-core trees stays below 2^-12 of the sum of magnitudes.  So
|out - ref| <= (e^(2E) - 1 + 4 * 2^-11) * sum p|v| + 2^-24 for every element.
The rms of the error over a case is far smaller: independent key roundings
perturb a score by sqrt(sum q^2 k^2) * scale * 2^-11 / sqrt(12), about 6e-4
for these keys, and an output by at most twice that, plus 2e-4 for its own
rounding: 1.5e-3 of the rms of the reference.
"""

import math

import numpy as np
import pytest
import torch

import _util
from oracle import chunk as ochunk
from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu


def _queries(seed, batch, n_q, hq):
    return synth.queries(seed, batch * n_q, hq).view(batch, n_q, hq, 128)


def _check(got, q, cfg, kv, window=0, sinks=0, scale=None):
    got = got.float().cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all()
    for b, (k, v) in enumerate(kv):
        heads = _util.oracle_heads(cfg, k, v)
        qb = q[b].cpu().numpy()
        ref, size = ochunk.chunk_attention(qb, heads, window, sinks, scale)
        E = ochunk.score_rounding(qb, heads, scale)
        bound = (math.expm1(2 * E) + 4 * 2.0 ** -11) * size + 2.0 ** -24
        worst = (np.abs(got[b] - ref) - bound).max()
        assert worst <= 0, f"sequence {b}: {worst:.3g} over the bound"
        rms = np.sqrt((ref ** 2).mean())
        if ref.size and rms > 0:
            err = np.sqrt(((got[b] - ref) ** 2).mean())
            assert err <= 1.5e-3 * rms, f"sequence {b}: rms error {err / rms:.3g}"


def _run(cfg, lengths, n_q, seed, window=0, sinks=0, **kw):
    cache, kv = _util.make_cache(cfg, lengths, seed)
    q = _queries(seed + 7, cfg.batch, n_q, cfg.n_q_heads)
    out = kvq.kvq_chunk_attn(cache, q.cuda(), window=window, sinks=sinks, **kw)
    torch.cuda.synchronize()
    assert cache.flags() == 0
    _check(out, q, cfg, kv, window, sinks, kw.get("softmax_scale"))
    return cache, kv, q, out


def _cfg(batch=1, hq=8, hkv=2, bk=2, bv=2, max_len=2048, **kw):
    return kvq.CacheConfig(batch=batch, n_q_heads=hq, n_kv_heads=hkv, bits_k=bk, bits_v=bv,
                           max_len=max_len, **kw)


@pytest.mark.parametrize("bk", [1, 2, 4, 8])
@pytest.mark.parametrize("bv", [1, 2, 4, 8])
def test_code_widths(kvq_lib, bk, bv):
    _run(_cfg(bk=bk, bv=bv), [677], 37, 10 * bk + bv)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (4, 4), (10, 2), (7, 1), (16, 2)])
@pytest.mark.parametrize("n_q", [1, 33])
def test_query_groups(kvq_lib, hq, hkv, n_q):
    _run(_cfg(hq=hq, hkv=hkv, bk=4, bv=1), [500], n_q, 20 + hq)


@pytest.mark.parametrize("L", [1, 2, 31, 33, 127, 128, 129, 159, 160, 161, 255, 256, 257, 289, 1024])
@pytest.mark.parametrize("n_q", [1, 2, 65])
def test_lengths(kvq_lib, L, n_q):
    """Lengths around block, tile and window edges; queries ahead of the first
    token (L < n_q) give zero rows."""
    cache, kv, q, out = _run(_cfg(bk=2, bv=4), [L], n_q, 30 + L)
    for t in range(max(0, n_q - L)):
        assert (out[0, t] == 0).all()


def test_empty_and_ragged_sequences(kvq_lib):
    _run(_cfg(batch=5, bk=1, bv=1), [0, 1, 130, 1100, 300], 40, 41)


@pytest.mark.parametrize("n_q,hq,hkv", [(300, 8, 2), (257, 5, 1), (64, 8, 1), (128, 2, 2), (513, 4, 1)])
@pytest.mark.parametrize("bk,bv", [(1, 1), (4, 8)])
def test_long_chunks(kvq_lib, n_q, hq, hkv, bk, bv):
    """Many row tiles, the last one partly filled; whole prompts too."""
    _run(_cfg(batch=2, hq=hq, hkv=hkv, bk=bk, bv=bv), [n_q, 900], n_q, 50 + n_q)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 4), (32, 33), (100, 0), (129, 160),
                                          (256, 5), (511, 64), (5000, 4)])
@pytest.mark.parametrize("n_q", [1, 19, 200])
def test_windows(kvq_lib, window, sinks, n_q):
    _run(_cfg(batch=2, bk=2, bv=1), [1100, 333], n_q, 60 + window, window, sinks)


@pytest.mark.parametrize("bk,bv", [(1, 2), (8, 4), (4, 1)])
@pytest.mark.parametrize("residual", [32, 256])
def test_residual_windows(kvq_lib, bk, bv, residual):
    _run(_cfg(bk=bk, bv=bv, residual=residual), [901], 70, 80 + residual, 300, 7)


@pytest.mark.parametrize("scale", [0.02, 0.5, 2.0])
def test_softmax_scale(kvq_lib, scale):
    """A scale of 2 gives scores in the hundreds: one token takes all."""
    _run(_cfg(bk=8, bv=8), [400], 20, 90, softmax_scale=scale)


def test_long_context_split(kvq_lib):
    """Few rows over a long cache: the tokens are shared by many CTAs."""
    _run(_cfg(batch=1, hq=8, hkv=1, bk=1, bv=2, max_len=16384), [16001], 3, 91)
    _run(_cfg(batch=3, hq=4, hkv=1, bk=4, bv=4, max_len=8192), [8100, 77, 4000], 1, 92)


def test_paged_equals_contiguous(kvq_lib):
    cfg = _cfg(batch=2, bk=2, bv=1, max_len=1024)
    lengths = [1001, 421]
    cache, kv, q, out = _run(cfg, lengths, 50, 95, 600, 40)
    paged = kvq.QuantKVCache(cfg, n_pages=64)
    perm = torch.randperm(64, generator=synth.generator(3)).tolist()
    used = 0
    for b, L in enumerate(lengths):
        blocks = kvq.blocks_written(0, L)
        paged.map_blocks(b, blocks, perm[used:used + len(blocks)])
        used += len(blocks)
        k, v = kv[b]
        kvq.kvq_pack(paged, k[None].cuda(), v[None].cuda(), batch_begin=b)
    got = kvq.kvq_chunk_attn(paged, q.cuda(), window=600, sinks=40)
    assert torch.equal(got, out) and paged.flags() == 0
    # blocks that no query of the call can see may be unmapped
    lo = lengths[0] - 50 - 600 + 1
    paged.map_blocks(0, range(2, lo // 32), [-1] * (lo // 32 - 2))
    got = kvq.kvq_chunk_attn(paged, q.cuda(), window=600, sinks=40)
    torch.cuda.synchronize()
    assert torch.equal(got, out) and paged.flags() == 0


def test_unmapped_block_sets_the_flag(kvq_lib):
    cfg = _cfg(bk=2, bv=2, max_len=512)
    paged = kvq.QuantKVCache(cfg, n_pages=16)
    k, v = synth.kv_heads(5, 2, 400)
    paged.map_blocks(0, range(8), range(8))
    kvq.kvq_pack(paged, k[None].cuda(), v[None].cuda())
    paged.map_blocks(0, [3], [99])
    out = kvq.kvq_chunk_attn(paged, _queries(6, 1, 4, 8).cuda())
    torch.cuda.synchronize()
    assert paged.flags() & kvq.FLAG_BAD_PAGE
    assert out.shape == (1, 4, 8, 128)


def test_strides_and_ranges_of_sequences(kvq_lib):
    cfg = _cfg(batch=3, bk=4, bv=2)
    cache, kv = _util.make_cache(cfg, [300, 700, 555], 96)
    q = _queries(97, 2, 21, 8)
    want = kvq.kvq_chunk_attn(cache, q.cuda(), batch_begin=1)
    # heads outside the tokens, and a wider row that holds q in its middle
    qt = q.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    wide = torch.full((2, 21, 10, 256), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, :, 1:9, 64:192] = q.cuda()
    holder = torch.full((2, 8, 21, 128), 7.0, dtype=torch.float16, device="cuda")
    got = kvq.kvq_chunk_attn(cache, qt, out=holder.transpose(1, 2), batch_begin=1)
    assert torch.equal(got, want)
    got = kvq.kvq_chunk_attn(cache, wide[:, :, 1:9, 64:192], batch_begin=1)
    assert torch.equal(got, want)
    one = kvq.kvq_chunk_attn(cache, q[:1].cuda().expand(2, 21, 8, 128), batch_begin=1)
    assert torch.equal(one[0], want[0])
    _check(want, q, cfg, kv[1:])


def test_stale_storage_is_not_read(kvq_lib):
    """NaN in every place that holds no token: unwritten pages and ring slots."""
    cfg = _cfg(batch=1, bk=2, bv=4, max_len=1024)
    cache = kvq.QuantKVCache(cfg)
    cache.buffer.fill_(0xff)
    cache.reset()
    k, v = synth.kv_heads(98, 2, 143)
    kvq.kvq_pack(cache, k[None].cuda(), v[None].cuda())
    q = _queries(99, 1, 9, 8)
    out = kvq.kvq_chunk_attn(cache, q.cuda())
    torch.cuda.synchronize()
    _check(out, q, cfg, [(k, v)])


def test_single_token_agrees_with_decode_attention(kvq_lib):
    cfg = _cfg(batch=2, hq=32, hkv=8, bk=1, bv=1, max_len=4096)
    cache, kv = _util.make_cache(cfg, [4000, 1234], 101)
    q = _queries(102, 2, 1, 32).cuda()
    a = kvq.kvq_chunk_attn(cache, q)[:, 0].float()
    b = kvq.kvq_decode_attn(cache, q[:, 0].contiguous()).float()
    assert ((a - b).pow(2).mean() / b.pow(2).mean()).sqrt() <= 2 * 1.5e-3


def test_chunks_repeat_bit_for_bit_and_leave_the_workspace_ready(kvq_lib):
    cfg = _cfg(batch=2, hq=8, hkv=1, bk=2, bv=2, max_len=8192)
    cache, kv = _util.make_cache(cfg, [8000, 900], 103)
    ws = kvq.chunk_workspace(cfg, 6)
    q = _queries(104, 2, 6, 8).cuda()
    first = kvq.kvq_chunk_attn(cache, q, workspace=ws)
    for _ in range(3):
        assert torch.equal(kvq.kvq_chunk_attn(cache, q, workspace=ws), first)


def test_on_another_stream_and_in_a_graph(kvq_lib):
    cfg = _cfg(bk=2, bv=2)
    cache, kv = _util.make_cache(cfg, [700], 105)
    q = _queries(106, 1, 11, 8).cuda()
    want = kvq.kvq_chunk_attn(cache, q)
    ws, out = kvq.chunk_workspace(cfg, 11), torch.zeros_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kvq.kvq_chunk_attn(cache, q, out=out, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    out.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kvq.kvq_chunk_attn(cache, q, out=out, workspace=ws)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
