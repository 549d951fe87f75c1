"""What kvq_chunk_attn and kvq_sample allocate for themselves when they are called
for another stream: the allocator must not hand it out while the call still waits or
runs there.  The other stream is held for about 0.1 s; meanwhile the memory that the
current stream's allocator would reuse is filled with zeros."""

import pytest
import torch

import _util
from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu


def _held(side):
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)


def test_chunk_workspace_and_result(kvq_lib):
    cfg = kvq.CacheConfig(batch=2, n_q_heads=8, n_kv_heads=2, bits_k=2, bits_v=2, max_len=2048)
    cache, _ = _util.make_cache(cfg, [2000, 1500], 3)
    q = synth.queries(4, 2 * 5, 8).view(2, 5, 8, 128).cuda()
    want = kvq.kvq_chunk_attn(cache, q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    _held(side)
    got = kvq.kvq_chunk_attn(cache, q, stream=side)
    n = kvq.chunk_workspace(cfg, 5).numel()
    for _ in range(4):
        torch.empty(n, dtype=torch.uint8, device="cuda").zero_()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_sample_results(kvq_lib):
    z = synth.logits(5, 3, 40000).cuda()
    want = kvq.kvq_sample(z)
    torch.cuda.synchronize()
    freed = [torch.empty(3, dtype=torch.int32, device="cuda") for _ in range(8)]
    for t in freed:
        t.zero_()
    side = torch.cuda.Stream()
    _held(side)
    del freed, t
    got = kvq.kvq_sample(z, stream=side)
    late = [torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    assert torch.equal(got["token"], want["token"])
    assert torch.equal(got["logprob"], want["logprob"])
    assert all((x == 0).all() for x in late)
