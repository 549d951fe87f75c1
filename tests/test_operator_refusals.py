"""What kvq_chunk_attn and kvq_sample refuse, before anything is enqueued (no
GPU is needed), and the oracles they are tested against."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import attention, chunk, quant, sample
from paper_2607_16248_gb300 import build, kvq, synth

FAKE = 0x100000


@pytest.fixture(scope="module")
def L():
    build.build()
    return kvq.lib()


def _chunk(L, q=FAKE, out=FAKE, n_q=4, window=0, sinks=0, scale=0.0, qs=(16384, 4096, 128),
           os=(16384, 4096, 128), begin=0, count=2, ws=FAKE, ws_bytes=None, cfg=None, cache=None):
    cfg = cfg or kvq.CacheConfig(batch=2, n_q_heads=32, n_kv_heads=8, bits_k=2, bits_v=2,
                                 max_len=4096)
    c = cfg.c()
    p = kvq._ChunkParams(n_q, window, sinks, scale, (ctypes.c_int64 * 3)(*qs),
                         (ctypes.c_int64 * 3)(*os))
    cache = cache or kvq._Cache(FAKE, FAKE, FAKE, FAKE)
    need = L.kvq_chunk_workspace_bytes(ctypes.byref(c), 4, 2)
    assert need > 0
    return L.kvq_chunk_attn(ctypes.byref(c), ctypes.byref(cache), q, out, ctypes.byref(p), begin,
                            count, ws, need - 1 if ws_bytes is None else ws_bytes, None)


def test_chunk_refusals(L):
    assert _chunk(L) == 4 and "workspace" in kvq.last_error()      # all else is in order
    ARG, SHAPE, ALIGN = 1, 2, 5
    for status, kw in (
            (ARG, dict(q=None)), (ARG, dict(out=None)), (ALIGN, dict(q=FAKE + 2)),
            (ALIGN, dict(out=FAKE + 8)), (ARG, dict(n_q=0)), (ARG, dict(n_q=4097)),
            (SHAPE, dict(count=0)), (SHAPE, dict(count=3)), (SHAPE, dict(begin=1)),
            (SHAPE, dict(begin=-1)), (ARG, dict(window=-1)), (ARG, dict(sinks=-1)),
            (ARG, dict(scale=-1.0)), (ARG, dict(scale=float("nan"))),
            (ARG, dict(scale=float("inf"))), (ALIGN, dict(qs=(16384, 4092, 128))),
            (ARG, dict(qs=(-16384, 4096, 128))), (ARG, dict(os=(0, 4096, 128))),
            (ARG, dict(os=(16384, 4096, 64))), (ALIGN, dict(os=(16384, 4096, 130))),
            (ARG, dict(ws=None)), (ALIGN, dict(ws=FAKE + 4)),
            (ARG, dict(cache=kvq._Cache(None, FAKE, FAKE, FAKE)))):
        assert _chunk(L, **kw) == status, (kw, kvq.last_error())
        assert kvq.last_error()


def test_chunk_workspace_sizes(L):
    cfg = kvq.CacheConfig(batch=2, n_q_heads=32, n_kv_heads=8, bits_k=2, bits_v=2, max_len=4096)
    c = cfg.c()
    for n_q, count in ((0, 1), (4097, 1), (1, 0), (1, 3)):
        assert L.kvq_chunk_workspace_bytes(ctypes.byref(c), n_q, count) == 0
    assert L.kvq_chunk_workspace_bytes(ctypes.byref(c), 4096, 2) > 0


def _sample(L, z=FAKE, zs=1000, u=FAKE, us=1000, B=4, V=1000, t=FAKE, k=FAKE, p=FAKE, m=FAKE,
            token=FAKE, lp=FAKE):
    return L.kvq_sample(z, zs, u, us, B, V, t, k, p, m, token, lp, None)


def test_sample_refusals(L):
    top = L.kvq_sample_max_vocab()
    assert top == 262144
    for status, kw in ((1, dict(z=None)), (1, dict(token=None)), (2, dict(B=0)),
                       (2, dict(B=65536)), (2, dict(V=0)), (3, dict(V=top + 1, zs=top + 1)),
                       (1, dict(zs=999)), (1, dict(us=-1)), (5, dict(z=FAKE + 2)),
                       (5, dict(k=FAKE + 1)), (5, dict(lp=FAKE + 3))):
        assert _sample(L, **kw) == status, (kw, kvq.last_error())


def test_binding_refusals(L):
    with pytest.raises(TypeError):
        kvq.kvq_sample(torch.zeros(2, 8))                 # not a CUDA tensor
    with pytest.raises(ValueError):
        kvq.kvq_sample(torch.zeros(8))


def test_chunk_oracle_is_the_decode_oracle_per_query():
    rng = np.random.default_rng(0)
    k, v = synth.kv_heads(1, 2, 300)
    q = rng.standard_normal((3, 4, 128)).astype(np.float16)
    heads = [quant.quantize_head(k[h].numpy(), v[h].numpy(), 2, 4, 128) for h in range(2)]
    out, size = chunk.chunk_attention(q, heads)
    assert np.allclose(out[2], attention.decode_attention(q[2], heads))
    assert (np.abs(out) <= size + 1e-12).all()
    seen = chunk.visible(300, 3, window=10, sinks=4)
    assert seen.sum(1).tolist() == [14, 14, 14] and seen[0, 288:298].all() and seen[:, :4].all()
    assert chunk.visible(2, 4).sum(1).tolist() == [0, 0, 1, 2]


def test_sample_oracle_by_hand():
    z = np.log([0.5, 0.2, 0.2, 0.1])
    assert osorted(z) == [0, 1, 2, 3]
    assert sample.kept(z, k=2).tolist() == [0, 1]
    assert sample.kept(z, p=0.45).tolist() == [0]
    assert sample.kept(z, p=0.6).tolist() == [0, 1]
    assert sample.kept(z, k=2, p=0.72).tolist() == [0, 1]     # 0.5 / 0.7 = 0.714
    assert sample.kept(z, k=2, p=0.70).tolist() == [0]
    assert sample.kept(z, m=0.3).tolist() == [0, 1, 2]
    u = np.exp(-np.array([1.0, 0.1, 1.0, 1.0]))
    tok, lp, _ = sample.sample_row(z, u)                      # keys ln(p / -ln u)
    assert tok == 1 and abs(lp - np.log(0.2)) < 1e-12
    assert sample.sample_row(np.full(3, -np.inf), u[:3])[0] == -1


def osorted(z):
    return sample.kept(z).tolist()
