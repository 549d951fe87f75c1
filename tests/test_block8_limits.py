"""Limits of the block-8 calls, at both sides, before anything is enqueued (no GPU is needed)."""

import pytest

from paper_2607_16248_gb300 import build, kvq
from test_block8_refusals import ARG, CAPACITY, SHAPE, _attn, _cfg


@pytest.fixture(scope="module")
def L():
    build.build()
    return kvq.lib()


def test_softmax_scales(L):
    """A scale whose product with log2 e is no fp32 number is refused."""
    for scale in (0.0, 1e-45, 2.0 ** 127):
        assert _attn(L, scale=scale) == CAPACITY, kvq.last_error()
    for scale in (2.0 ** 127 * (1 + 2.0 ** -23), 3.4e38):
        assert _attn(L, scale=scale) == ARG and "softmax_scale" in kvq.last_error()


def tiles(rows):
    return -(-rows // 256) if rows > 128 else 1


@pytest.mark.parametrize("batch,hkv,gq,max_len,max_new", [
    # caches of long texts: each of them is within what a call's units can count
    (64, 8, 4, 131072, 16384), (5, 8, 4, 131072, 131072), (64, 8, 4, 40960, 40960),
    (64, 8, 4, 131072, 131072), (512, 8, 8, 131072, 4), (8192, 8, 4, 4096, 4096),
    # the ends: units of blocks (one token each), of row tiles
    (8192, 8, 1, 149696, 1), (8192, 8, 1, 149728, 1), (8192, 1024, 1, 1088, 1),
    (8192, 1024, 1, 1120, 1), (1, 1, 1, 2 ** 31 - 32, 1), (1, 1, 1, 2 ** 31 - 32, 32512),
    (1, 1, 1, 2 ** 31 - 32, 32513), (512, 8, 4, 131072, 32640), (512, 8, 4, 131072, 32768)])
def test_units(L, batch, hkv, gq, max_len, max_new):
    """A call is refused where one of its kernels could not count its units in 32 bits."""
    blocks, rows = batch * hkv * (7 * max_len // 32 + 16), max_new * gq
    most = max(blocks, batch * hkv * tiles(rows) * (-(-max_len // 128) + 3) if rows > 32 else 0)
    cfg = _cfg(batch=batch, n_q_heads=hkv * gq, n_kv_heads=hkv, max_len=max_len)
    status = _attn(L, cfg=cfg, max_new=max_new, ws_bytes=0)
    assert status == (CAPACITY if most < 2 ** 31 else SHAPE), (most / 2 ** 31, kvq.last_error())
