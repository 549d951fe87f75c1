"""The host's bound on a call's units of work is the kernel's own count for full
sequences: ceil(max_len / 128) tiles and three more for every row tile of up to 256
query rows, below 2^31."""

import ctypes

import pytest

from paper_2607_16248_gb300 import build, kvq


@pytest.mark.parametrize("batch,hq,hkv,n_q,max_len,fits", [
    # one row an item: 65535 * 2048 items of 13, 14 and 15 tiles
    (65535, 2048, 2048, 1, 13 * 128, True),
    (65535, 2048, 2048, 1, 13 * 128 + 32, False),
    (65535, 2048, 2048, 1, 14 * 128, False),
    # 256 rows an item, 2^20 items of 1500, 2044 and 2045 tiles
    (1024, 8192, 1024, 32, 1500 * 128, True),
    (1024, 8192, 1024, 32, 2044 * 128, True),
    (1024, 8192, 1024, 32, 2044 * 128 + 32, False),
])
def test_units(batch, hq, hkv, n_q, max_len, fits):
    rows = n_q * hq // hkv
    tiles = -(-rows // 256) if rows > 128 else 1
    assert (batch * hkv * tiles * (-(-max_len // 128) + 3) < 2 ** 31) == fits
    build.build()
    cfg = kvq.CacheConfig(batch=batch, n_q_heads=hq, n_kv_heads=hkv, bits_k=1, bits_v=1,
                          max_len=max_len)
    n = kvq.lib().kvq_chunk_workspace_bytes(ctypes.byref(cfg.c()), n_q, batch)
    assert (n > 0) == fits, kvq.last_error()


def test_workspace_takes_one_of_two_sizes():
    build.build()

    def size(n_q, batch, count, max_len=4096):
        cfg = kvq.CacheConfig(batch=batch, n_q_heads=32, n_kv_heads=8, bits_k=2, bits_v=2,
                              max_len=max_len)
        return kvq.lib().kvq_chunk_workspace_bytes(ctypes.byref(cfg.c()), n_q, count)

    small = {size(n_q, b, c, m) for n_q in (1, 32) for b, c in ((1, 1), (64, 3), (64, 64))
             for m in (64, 65536)}
    large = {size(n_q, b, c) for n_q in (33, 4096) for b, c in ((1, 1), (64, 3), (64, 64))}
    assert len(small) == len(large) == 1
    assert 0 < small.pop() < large.pop()
