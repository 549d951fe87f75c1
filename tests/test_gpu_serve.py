"""The serving example end to end: chunked prompt, windowed single tokens with
pages handed back, restored logits, sampled tokens."""

import importlib.util
from pathlib import Path

import pytest
import torch

from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu

PATH = Path(__file__).resolve().parents[1] / "examples" / "serve.py"


@pytest.fixture(scope="module")
def serve():
    spec = importlib.util.spec_from_file_location("serve_example", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_tokens_repeat_and_pages_are_handed_back(kvq_lib, serve):
    args = dict(prompt=1500, chunk=400, steps=40, window=512, sinks=4, layers=2, vocab=5000)
    ids, stack = serve.serve(**args)
    again, _ = serve.serve(**args)
    assert torch.equal(ids, again)
    assert ((ids >= 0) & (ids < 5000)).all()
    for layer in stack:
        assert layer.cache.flags() == 0
        assert layer.cache.seq_lens().cpu().tolist() == [1540] == [layer.length]
        # the window's packed blocks and the sinks' one
        assert len(layer.mapped) <= (512 - 128) // 32 + 3


def test_window_does_not_depend_on_what_was_handed_back(kvq_lib, serve):
    """A step on a cache whose old pages are gone equals the step on a whole one."""
    cfg = kvq.CacheConfig(batch=1, n_q_heads=8, n_kv_heads=2, bits_k=2, bits_v=2, max_len=2048)
    window, sinks = 300, 33
    layer = serve.Layer(cfg, 64, window, sinks)
    whole = kvq.QuantKVCache(cfg)
    k, v = synth.kv_heads(3, 2, 1200)
    ws = {n: kvq.chunk_workspace(cfg, n) for n in (100, 1)}
    at = 0
    for n in [100] * 11 + [1] * 100:
        q = synth.queries(50 + at, n, 8).view(1, n, 8, 128).cuda()
        kk, vv = (x[None, :, at:at + n].contiguous().cuda() for x in (k, v))
        got = layer.step(q, kk, vv, ws[n])
        kvq.kvq_pack(whole, kk, vv)
        want = kvq.kvq_chunk_attn(whole, q, window=window, sinks=sinks, workspace=ws[n])
        assert torch.equal(got, want), at
        at += n
    assert layer.cache.flags() == 0 and len(layer.mapped) < 16
