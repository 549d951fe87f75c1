"""Calls of two kernels of which the second starts early (chunks and their join, the stream of
logits and its patches), captured into CUDA graphs and replayed with other contents; adjusted
logits on another stream."""

import numpy as np
import pytest
import torch

from paper_2607_16248_gb300 import kvq
from test_gpu_block8_edges import check, filled, ints

pytestmark = pytest.mark.gpu


def captured(call):
    call()                       # (kernels are loaded outside)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    return graph, out


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("own", [False, True])
def test_chunks_beside_tokens(kvq_lib, dtype, own):
    """Two graphs over one workspace (or each over its own, made in the capture), replayed in
    turn with other queries and lengths."""
    cfg, cache, seen = filled(dtype, 3, 2, [900, 700, 40], 928, seed=50)
    g = torch.Generator().manual_seed(51)
    ws = kvq.block8_workspace(cfg, 120)
    made = []
    for counts in ([120, 1, 3], [1, 90, 20]):
        n = sum(counts)
        q = torch.zeros(n, cfg.n_q_heads, 128, dtype=cfg.dtype, device="cuda")
        starts, lengths = ints(np.concatenate([[0], np.cumsum(counts)])), ints([900, 700, 40])
        graph, out = captured(lambda: kvq.kvq_block8_attn(
            cache, q, lengths, starts=starts, max_new=120, workspace=None if own else ws))
        made.append((counts, q, starts, lengths, graph, out))
    other = kvq.block8_workspace(cfg, 120)
    for step in range(12):
        counts, q, starts, lengths, graph, out = made[step % 2]
        q.copy_(torch.randn(q.shape, generator=g))
        now = [900 - 32 * (step // 2), 700 - 64 * (step // 4), 40]
        lengths.copy_(ints(now))
        graph.replay()
        want = kvq.kvq_block8_attn(cache, q, ints(now), starts=starts, max_new=120,
                                   workspace=other)
        assert torch.equal(out, want), step
        if step < 2: check(cfg, out, q, now, counts, seen)
    assert cache.flags() == 0


def inputs(rows, vocab, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kw = dict(device="cuda", generator=g)
    n = 300 * rows
    return dict(
        logits=(4 * torch.randn(rows, vocab, **kw)).bfloat16(),
        history=torch.randint(0, vocab, (n,), dtype=torch.int32, **kw),
        repetition=1 + torch.rand(rows, **kw), frequency=torch.rand(rows, **kw),
        bias_ids=torch.randint(0, vocab, (20 * rows,), dtype=torch.int32, **kw),
        bias_values=torch.randn(20 * rows, **kw),
        mask=torch.randint(-2 ** 31, 2 ** 31, (rows, (vocab + 31) // 32), dtype=torch.int32, **kw))


@pytest.mark.parametrize("rows,vocab", [(64, 152063), (3, 32000)])
def test_adjusted_logits(kvq_lib, rows, vocab):
    """By two kernels (many logits, short lists) and by one; replayed, and on another stream."""
    lists = dict(history_starts=ints([300 * b for b in range(rows + 1)]),
                 bias_starts=ints([20 * b for b in range(rows + 1)]))
    x = inputs(rows, vocab, 1)
    graph, out = captured(lambda: kvq.kvq_adjust_logits(**x, **lists))
    side = torch.cuda.Stream()
    for seed in range(2, 7):
        for n, t in inputs(rows, vocab, seed).items():
            x[n].copy_(t)
        graph.replay()
        want = kvq.kvq_adjust_logits(**x, **lists)
        assert torch.equal(out, want)
        assert not torch.equal(want, x["logits"].float())
        side.wait_stream(torch.cuda.current_stream())
        got = kvq.kvq_adjust_logits(**x, **lists, stream=side)
        side.synchronize()
        assert torch.equal(got, want)
