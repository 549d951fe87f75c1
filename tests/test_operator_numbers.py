"""Numbers outside their 32-bit arguments, at either end, are refused and not cut to
their low bits: windows, sinks, ranges of sequences, sizes of views that repeat."""

from types import SimpleNamespace

import pytest
import torch

from paper_2607_16248_gb300 import build, kvq

CFG = kvq.CacheConfig(batch=4, n_q_heads=2, n_kv_heads=1, bits_k=2, bits_v=2, max_len=64)


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()


@pytest.mark.parametrize("kw", [dict(window=-2 ** 32), dict(window=-2 ** 32 + 5),
                                dict(window=4, sinks=-2 ** 32 + 1), dict(window=4, sinks=-2 ** 40),
                                dict(batch_begin=2 ** 32 + 1), dict(batch_begin=-2 ** 32),
                                dict(batch_begin=2 ** 31)])
def test_chunk_arguments(kw):
    with pytest.raises(ValueError, match="32 bits"):
        kvq.kvq_chunk_attn(SimpleNamespace(cfg=CFG), torch.zeros(1, 1, 2, 128).half(), **kw)


@pytest.mark.parametrize("shape", [(2 ** 32 + 1, 1), (1, 2 ** 32 + 1)])
def test_chunk_sizes(shape):
    q = torch.zeros(1, 1, 2, 128).half().expand(*shape, 2, 128)
    with pytest.raises(ValueError, match="32 bits"):
        kvq.kvq_chunk_attn(SimpleNamespace(cfg=CFG), q, out=q)


@pytest.mark.parametrize("n_q,count", [(2 ** 32 + 4, 1), (4, 2 ** 32 + 1), (-2 ** 32 + 4, 1)])
def test_workspace_sizes(n_q, count):
    with pytest.raises(ValueError, match="32 bits"):
        kvq.chunk_workspace(CFG, n_q, count, device="meta")


@pytest.mark.parametrize("shape", [(2 ** 32 + 1, 5), (1, 2 ** 32 + 5)])
def test_sample_sizes(shape):
    with pytest.raises(ValueError, match="32 bits"):
        kvq.kvq_sample(torch.zeros(1, 1).expand(*shape))
