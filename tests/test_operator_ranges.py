"""Numbers that do not fit the library's 32-bit arguments are refused, not cut."""

from types import SimpleNamespace

import pytest
import torch

from paper_2607_16248_gb300 import kvq


@pytest.mark.parametrize("kw", [dict(window=2 ** 31), dict(window=2 ** 32 + 5),
                                dict(window=4, sinks=2 ** 32)])
def test_windows_beyond_32_bits(kw):
    cfg = kvq.CacheConfig(batch=1, n_q_heads=2, n_kv_heads=1, bits_k=2, bits_v=2, max_len=64)
    with pytest.raises(ValueError, match="window and sinks"):
        kvq.kvq_chunk_attn(SimpleNamespace(cfg=cfg), torch.zeros(1, 1, 2, 128).half(), **kw)
