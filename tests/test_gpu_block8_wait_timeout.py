"""A wait of the block-8 attention's kernels that runs out is reported, ends the kernel, and
leaves workspace and context usable."""

import time

import pytest
import torch

from paper_2607_16248_gb300 import build, kvq
from test_block8_refusals import CAPACITY, UNSUPPORTED, _cache, _cfg
from test_gpu_block8_edges import check, filled, ints


@pytest.mark.gpu
@pytest.mark.parametrize("batch,hkv,L,n", [(20, 8, 700, 2), (3, 2, 12000, 1), (1, 8, 9000, 40),
                                           (2, 2, 3000, 300)])
def test_a_wait_that_runs_out(kvq_lib, batch, hkv, L, n):
    cfg, cache, seen = filled("fp16", batch, hkv, [L] * batch, (L + 31) // 32 * 32, seed=60)
    q = torch.randn(batch * n, cfg.n_q_heads, 128,
                    generator=torch.Generator().manual_seed(61)).half().cuda()
    lengths, ws = ints([L] * batch), kvq.block8_workspace(cfg, n)
    want = kvq.kvq_block8_attn(cache, q, lengths, workspace=ws)
    kvq.selftest_block8_wait_timeout(cache, q, lengths, ws)     # loads the kernel
    torch.cuda.synchronize()
    cache.clear_flags()
    t0 = time.perf_counter()
    kvq.selftest_block8_wait_timeout(cache, q, lengths, ws)
    torch.cuda.synchronize()
    # two or three waits of 10 ms a warp, where the kernels' own limits are one and two seconds
    assert time.perf_counter() - t0 < 0.4
    assert cache.flags() == kvq.FLAG_WAIT_TIMEOUT
    assert (ws[:4 * 152] == 0).all()
    cache.clear_flags()
    out = kvq.kvq_block8_attn(cache, q, lengths, workspace=ws)
    assert torch.equal(out, want) and cache.flags() == 0
    check(cfg, out, q, [L] * batch, [n] * batch, seen)


def test_refusals():
    """Checked as the attention's arguments are, and what it has no kernel for."""
    import ctypes
    build.build()
    fake = 0x100000

    def call(max_new, **kw):
        c, cache = _cfg(**kw), _cache()
        b = kvq._Block8Batch(fake, fake, 4, max_new)
        p = kvq._Block8Attn(0, 0, 0.0, kvq._Pair(1024, 128), kvq._Pair(1024, 128))
        return kvq.lib().kvq_selftest_block8_wait_timeout(
            ctypes.byref(c), ctypes.byref(cache), ctypes.byref(b), fake, fake + 4096,
            ctypes.byref(p), fake, 0, None)

    assert call(2) == CAPACITY and call(9) == CAPACITY
    assert call(3) == UNSUPPORTED and call(8) == UNSUPPORTED
    assert call(1, dtype=torch.bfloat16) == UNSUPPORTED
    assert call(1, n_q_heads=18, n_kv_heads=2) == UNSUPPORTED
