"""What kvq_block8_append, kvq_block8_attn and kvq_adjust_logits refuse, before anything is
enqueued (no GPU is needed), and their oracle by hand."""

import ctypes

import numpy as np
import pytest
import torch

from oracle import block8
from paper_2607_16248_gb300 import build, kvq

FAKE = 0x100000
ARG, SHAPE, UNSUPPORTED, CAPACITY, ALIGN = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def L():
    build.build()
    return kvq.lib()


def _cfg(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, max_len=1024)
    base.update(kw)
    return kvq.Block8Config(**base).c()


def _cache(n_pages=10, **kw):
    names = ("k_codes", "v_codes", "scales", "k_ring", "v_ring", "block_table", "flags")
    return kvq._Block8Cache(*(kw.get(n, FAKE) for n in names), n_pages)


def test_the_packed_structs_are_the_headers():
    for packed, ct in ((kvq._BATCH, kvq._Block8Batch), (kvq._APPEND, kvq._Block8Append),
                       (kvq._ATTN, kvq._Block8Attn), (kvq._ADJUST, kvq._AdjustParams)):
        assert packed.size == ctypes.sizeof(ct)
    values = list(range(1, 19))
    x = kvq._Block8Append.from_buffer_copy(kvq._APPEND.pack(*values))
    assert (x.k, x.positions, x.n_positions, x.paired, x.q_out_stride[1]) == (1, 7, 8, 10, 18)
    x = kvq._AdjustParams.from_buffer_copy(kvq._ADJUST.pack(*range(1, 23)))
    assert (x.logits, x.mask_rows, x.mask_stride, x.dtype, x.n_masks) == (1, 13, 16, 17, 22)
    x = kvq._Block8Attn.from_buffer_copy(kvq._ATTN.pack(1, 2, 0.5, 3, 4, 5, 6))
    assert (x.window, x.sinks, x.softmax_scale, x.out_stride[1]) == (1, 2, 0.5, 6)


def test_config(L):
    for status, kw in ((0, {}), (SHAPE, dict(batch=0)), (SHAPE, dict(batch=8193)),
                       (SHAPE, dict(n_q_heads=7)), (UNSUPPORTED, dict(n_q_heads=66)),
                       (SHAPE, dict(n_q_heads=0)), (SHAPE, dict(n_q_heads=2048, n_kv_heads=2048)),
                       (UNSUPPORTED, dict(head_dim=64)), (UNSUPPORTED, dict(block=16)),
                       (SHAPE, dict(max_len=100)), (SHAPE, dict(max_len=0)),
                       (UNSUPPORTED, dict(dtype=torch.float32))):
        c = _cfg(**kw)
        assert L.kvq_block8_validate_config(ctypes.byref(c)) == status, (kw, kvq.last_error())


def _append(L, cfg=None, cache=None, lengths=FAKE, starts=FAKE, n=4, max_new=4, **kw):
    c = cfg or _cfg()
    batch = kvq._Block8Batch(lengths, starts, n, max_new)
    p = kvq._Block8Append()
    values = dict(k=FAKE, v=FAKE, q=FAKE, q_out=FAKE + 4096, cos=FAKE, sin=FAKE, positions=None,
                  n_positions=100, rot_dim=128, paired=0, k_stride=(256, 128),
                  v_stride=(256, 128), q_stride=(1024, 128), q_out_stride=(1024, 128))
    values.update(kw)
    for name, value in values.items():
        setattr(p, name, kvq._Pair(*value) if "stride" in name else value)
    cache = cache or _cache()
    return L.kvq_block8_append(ctypes.byref(c), ctypes.byref(cache), ctypes.byref(batch),
                               ctypes.byref(p), None)


def test_append_refusals(L):
    for status, kw in (
            (ARG, dict(lengths=None)), (ALIGN, dict(lengths=FAKE + 2)),
            (ALIGN, dict(starts=FAKE + 1)),
            (SHAPE, dict(n=0)), (SHAPE, dict(n=2 ** 26)), (ARG, dict(max_new=0)),
            (ARG, dict(max_new=1025)), (SHAPE, dict(starts=None, n=5)), (ARG, dict(k=None)),
            (ARG, dict(v=None)), (ARG, dict(q=None)), (ARG, dict(q_out=None)),
            (ALIGN, dict(k=FAKE + 8)), (ALIGN, dict(q_out=FAKE + 2)),
            (ALIGN, dict(k_stride=(260, 128))), (ARG, dict(v_stride=(-256, 128))),
            (ARG, dict(q_out_stride=(64, 128))), (ARG, dict(q_out_stride=(1024, 0))),
            (ARG, dict(q_out=FAKE, q_out_stride=(2048, 128))), (UNSUPPORTED, dict(rot_dim=130)),
            (UNSUPPORTED, dict(rot_dim=12)), (UNSUPPORTED, dict(rot_dim=-8)), (ARG, dict(cos=None)),
            (ALIGN, dict(sin=FAKE + 4)), (ARG, dict(n_positions=0)),
            (ALIGN, dict(positions=FAKE + 2)), (ARG, dict(cache=_cache(k_codes=None))),
            (ARG, dict(cache=_cache(flags=None))), (ALIGN, dict(cache=_cache(v_ring=FAKE + 8))),
            (ALIGN, dict(cache=_cache(block_table=FAKE + 2))), (ARG, dict(cache=_cache(n_pages=0))),
            (SHAPE, dict(cache=_cache(n_pages=2 ** 25 + 1)))):
        assert _append(L, **kw) == status, (kw, kvq.last_error())
        assert kvq.last_error()


def _attn(L, q=FAKE, out=FAKE + 4096, window=0, sinks=0, scale=0.0, qs=(1024, 128), os=(1024, 128),
          ws=FAKE, max_new=4, ws_bytes=None, cfg=None, cache=None, n=4):
    c = cfg or _cfg()
    batch = kvq._Block8Batch(FAKE, FAKE, n, max_new)
    p = kvq._Block8Attn(window, sinks, scale, kvq._Pair(*qs), kvq._Pair(*os))
    need = L.kvq_block8_workspace_bytes(ctypes.byref(_cfg()), 4)
    cache = cache or _cache()
    return L.kvq_block8_attn(ctypes.byref(c), ctypes.byref(cache), ctypes.byref(batch), q, out,
                             ctypes.byref(p), ws, need - 1 if ws_bytes is None else ws_bytes, None)


def test_attn_refusals(L):
    assert _attn(L) == CAPACITY and "workspace" in kvq.last_error()    # all else is in order
    for status, kw in (
            (ARG, dict(q=None)), (ARG, dict(out=None)), (ARG, dict(out=FAKE)),
            (ALIGN, dict(q=FAKE + 2)), (ALIGN, dict(out=FAKE + 8)), (ARG, dict(window=-1)),
            (ARG, dict(sinks=-1)),
            (ARG, dict(scale=-1.0)), (ARG, dict(scale=float("nan"))),
            (ARG, dict(scale=float("inf"))),
            (ALIGN, dict(qs=(1020, 128))), (ARG, dict(qs=(-8, 128))), (ARG, dict(os=(64, 128))),
            (ARG, dict(os=(1024, 0))), (ARG, dict(ws=None)), (ALIGN, dict(ws=FAKE + 4)),
            (ARG, dict(max_new=2000)), (ARG, dict(cache=_cache(scales=None))),
            (SHAPE, dict(cfg=_cfg(batch=8192, n_kv_heads=1024, n_q_heads=1024,
                                  max_len=1 << 30)))):
        assert _attn(L, **kw) == status, (kw, kvq.last_error())
    c = _cfg()
    for n in (0, 1025, -1):
        assert L.kvq_block8_workspace_bytes(ctypes.byref(c), n) == 0
    few, many = (L.kvq_block8_workspace_bytes(ctypes.byref(c), n) for n in (1, 1024))
    assert 0 < few < many


def _adjust(L, **kw):
    p = kvq._AdjustParams()
    values = dict(logits=FAKE, out=FAKE + 4096, history=FAKE, history_starts=FAKE,
                  prompt_lengths=FAKE, repetition=FAKE, frequency=FAKE, presence=FAKE,
                  bias_ids=FAKE, bias_values=FAKE, bias_starts=FAKE, mask=FAKE, mask_rows=None,
                  logits_stride=1000, out_stride=1000, mask_stride=32, dtype=2, rows=4, vocab=1000,
                  n_history=10, n_bias=10, n_masks=4)
    values.update(kw)
    for name, value in values.items():
        setattr(p, name, value)
    return L.kvq_adjust_logits(ctypes.byref(p), None)


def test_adjust_refusals(L):
    for status, kw in (
            (ARG, dict(logits=None)), (ARG, dict(out=None)), (UNSUPPORTED, dict(dtype=3)),
            (SHAPE, dict(rows=0)), (SHAPE, dict(rows=65536)), (SHAPE, dict(vocab=0)),
            (SHAPE, dict(vocab=2 ** 30 + 1)), (ARG, dict(out_stride=999)),
            (ARG, dict(logits_stride=-1)), (ARG, dict(out=FAKE, dtype=0)),
            (ARG, dict(out=FAKE, logits_stride=2000)), (ARG, dict(history=None)),
            (ARG, dict(history_starts=None)), (ARG, dict(bias_values=None)),
            (ARG, dict(bias_starts=None)),
            (ARG, dict(history=None, history_starts=None, n_history=0)),
            (ARG, dict(mask=None, mask_rows=FAKE)), (SHAPE, dict(n_masks=3)),
            (SHAPE, dict(n_masks=0)), (ARG, dict(mask_stride=31)), (SHAPE, dict(n_history=-1)),
            (SHAPE, dict(n_bias=2 ** 30)), (ALIGN, dict(logits=FAKE + 2)),
            (ALIGN, dict(logits=FAKE + 1, dtype=1)), (ALIGN, dict(out=FAKE + 2)),
            (ALIGN, dict(history=FAKE + 1)), (ALIGN, dict(mask=FAKE + 2))):
        assert _adjust(L, **kw) == status, (kw, kvq.last_error())


def test_binding_refusals(L):
    z = torch.zeros(2, 8)
    for call in (lambda: kvq.kvq_adjust_logits(z),
                 lambda: kvq.Block8Cache(kvq.Block8Config(1, 2, 1, 64), n_pages=2, device="cpu")):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: kvq.kvq_adjust_logits(z[0]),
                 lambda: kvq.Block8Cache(kvq.Block8Config(1, 2, 1, 64)),
                 lambda: kvq.Block8Cache(kvq.Block8Config(1, 2, 1, 64), n_pages=0),
                 lambda: kvq.Block8Config(2 ** 40, 2, 1, 64).c()):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(kvq.KvqError):
        kvq.Block8Cache(kvq.Block8Config(1, 3, 2, 64), n_pages=2)
    assert list(kvq.block8_written(0, 31)) == [] and list(kvq.block8_written(31, 34)) == [0, 1]


def test_oracle_by_hand():
    assert block8.to_type(1.0 + 2.0 ** -11, "fp16") == 1.0        # a tie goes to the even one
    assert block8.to_type(1.0 + 3 * 2.0 ** -11, "fp16") == 1.0 + 2.0 ** -9
    assert block8.to_type(465.0, "e4m3") == 448.0 and block8.to_type(17.0, "e4m3") == 16.0
    assert block8.to_type(2.0 ** -10, "e4m3") == 0.0
    assert block8.to_type(-2.0 ** -9, "e4m3") == -2.0 ** -9
    # torch's conversion goes by way of fp32, as a code's definition does
    grid = np.array([block8.to_type(block8.to_type(x, "fp32"), "e4m3")
                     for x in np.linspace(-460, 460, 3001)])
    near = torch.tensor(np.linspace(-460, 460, 3001)).clamp(-448, 448).to(torch.float8_e4m3fn)
    assert np.array_equal(grid, near.double().numpy())
    x = np.arange(128.0)[None, None]
    c, s = np.zeros((1, 2)), np.ones((1, 2))
    y = block8.rotate(x, c, s, False)                              # a quarter turn
    assert y[0, 0, :5].tolist() == [-2.0, -3.0, 0.0, 1.0, 4.0]
    assert block8.rotate(x, c, s, True)[0, 0, :5].tolist() == [-1.0, 0.0, -3.0, 2.0, 4.0]
    codes, scale = block8.quantize(np.full((32, 128), -4.0))
    assert (codes == -448.0).all() and scale == block8.to_type(4.0 / 448.0, "fp32")
    assert block8.quantize(np.zeros((32, 128)))[1] == 1.0
    z = block8.adjust([1.0, -1.0, 2.0, 0.0], history=[0, 1, 1, 9, -1], prompt=1, repetition=2.0,
                      frequency=0.5, presence=0.25, bias=[(2, 1.0), (2, 3.0), (7, 1.0)],
                      allowed=[True, True, True, False])
    assert z.tolist() == [0.5, -3.25, 5.0, -np.inf]
