"""A workspace whose elements do not lie side by side is refused: its numel says
nothing about the bytes behind its address."""

import pytest
import torch

import _util
from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu


def test_workspaces_that_are_not_contiguous(kvq_lib):
    cfg = kvq.CacheConfig(batch=1, n_q_heads=4, n_kv_heads=1, bits_k=2, bits_v=2, max_len=512)
    cache, _ = _util.make_cache(cfg, [300], 3)
    q = synth.queries(4, 3, 4).view(1, 3, 4, 128).cuda()
    n = kvq.chunk_workspace(cfg, 3).numel()
    whole = torch.zeros(n, 2, dtype=torch.uint8, device="cuda")
    for bad in (torch.zeros(16, dtype=torch.uint8, device="cuda").expand(n // 16 + 1, 16),
                whole[:, :1], whole[:, 0], whole.view(2, n)[:, :n // 2 + 16]):
        assert not bad.is_contiguous()
        with pytest.raises(ValueError, match="workspace"):
            kvq.kvq_chunk_attn(cache, q, workspace=bad)
    want = kvq.kvq_chunk_attn(cache, q)
    assert torch.equal(kvq.kvq_chunk_attn(cache, q, workspace=whole.view(2 * n)), want)
