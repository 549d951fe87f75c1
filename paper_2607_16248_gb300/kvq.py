"""Thin Python binding of the kvq C ABI (``include/kvq.h``).

Argument marshalling only: every step of the decode path runs in the CUDA
kernels of ``libkvq.so``.  PyTorch supplies device memory and the current CUDA
stream.  The library must have been built (``paper_2607_16248_gb300.build``);
a missing library or a non-CUDA tensor raises instead of falling back.
"""

import ctypes
import math
import struct
from dataclasses import dataclass
from pathlib import Path

import torch

_LIB_PATH = Path(__file__).resolve().with_name("libkvq.so")
_lib = None

STATUS_NAMES = {0: "KVQ_OK", 1: "KVQ_ERR_ARG", 2: "KVQ_ERR_SHAPE", 3: "KVQ_ERR_UNSUPPORTED",
                4: "KVQ_ERR_CAPACITY", 5: "KVQ_ERR_ALIGN", 6: "KVQ_ERR_CUDA"}
FLAG_OVERFLOW = 1
FLAG_WAIT_TIMEOUT = 2
FLAG_BAD_PAGE = 4
FLAG_BAD_BATCH = 8

# Every symbol include/kvq.h declares.
EXPORTS = (
    "kvq_last_error", "kvq_version", "kvq_validate_config", "kvq_page_bytes",
    "kvq_cache_layout", "kvq_cache_bind", "kvq_cache_reset", "kvq_pack",
    "kvq_page_pool_bytes", "kvq_paged_cache_layout", "kvq_paged_cache_bind",
    "kvq_attn_workspace_bytes", "kvq_attn_default_splits", "kvq_attn_splits_for_lengths",
    "kvq_workspace_init",
    "kvq_decode_attn", "kvq_decode_attn_f32", "kvq_decode_step", "kvq_decode_step_f32",
    "kvq_decode_attn_noalloc", "kvq_chunk_workspace_bytes", "kvq_chunk_attn",
    "kvq_block8_validate_config", "kvq_block8_append", "kvq_block8_workspace_bytes",
    "kvq_block8_attn", "kvq_adjust_logits",
    "kvq_sample_max_vocab", "kvq_sample", "dgap_workspace_bytes",
    "dgap_restore", "kvq_drift_max_vocab", "kvq_drift_metrics", "kvq_drift_window",
    "kvq_selftest_wait_timeout", "kvq_selftest_chunk_wait_timeout",
    "kvq_selftest_block8_wait_timeout",
)
NOALLOC_SCRATCH_BYTES = 4 << 20


class KvqError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class _Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "n_q_heads", "n_kv_heads", "head_dim", "bits_k", "bits_v",
        "group", "residual", "max_len")]


class _Cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("k_resid", ctypes.c_void_p),
                ("v_resid", ctypes.c_void_p), ("seq_len", ctypes.c_void_p),
                ("block_table", ctypes.c_void_p), ("n_pages", ctypes.c_int32)]


class _DriftParams(ctypes.Structure):
    _fields_ = [("alpha", ctypes.c_float), ("window", ctypes.c_int32), ("k_max", ctypes.c_int32),
                ("eps", ctypes.c_float), ("rho_c", ctypes.c_float)]


class _ChunkParams(ctypes.Structure):
    _fields_ = [("n_q", ctypes.c_int32), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("q_stride", ctypes.c_int64 * 3),
                ("out_stride", ctypes.c_int64 * 3)]


class _Block8Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "n_q_heads", "n_kv_heads", "head_dim", "block", "max_len", "dtype")]


class _Block8Cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "k_codes", "v_codes", "scales", "k_ring", "v_ring", "block_table", "flags")] + [
        ("n_pages", ctypes.c_int32)]


class _Block8Batch(ctypes.Structure):
    _fields_ = [("lengths", ctypes.c_void_p), ("starts", ctypes.c_void_p),
                ("n_tokens", ctypes.c_int32), ("max_new", ctypes.c_int32)]


_Pair = ctypes.c_int64 * 2


class _Block8Append(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "k", "v", "q", "q_out", "cos", "sin", "positions")] + [
        (n, ctypes.c_int32) for n in ("n_positions", "rot_dim", "paired")] + [
        (n, _Pair) for n in ("k_stride", "v_stride", "q_stride", "q_out_stride")]


class _Block8Attn(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("sinks", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("q_stride", _Pair), ("out_stride", _Pair)]


class _AdjustParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "logits", "out", "history", "history_starts", "prompt_lengths", "repetition",
        "frequency", "presence", "bias_ids", "bias_values", "bias_starts", "mask",
        "mask_rows")] + [(n, ctypes.c_int64) for n in (
            "logits_stride", "out_stride", "mask_stride")] + [(n, ctypes.c_int32) for n in (
                "dtype", "rows", "vocab", "n_history", "n_bias", "n_masks")]


class _DgapParams(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int32), ("hidden", ctypes.c_int32), ("tau", ctypes.c_float)] + [
        (n, ctypes.c_void_p) for n in ("det_w1", "det_b1", "det_w2", "det_b2",
                                       "cor_w1", "cor_b1", "cor_w2", "cor_b2")]


def lib():
    """Load libkvq.so once (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with "
                               "paper_2607_16248_gb300.build.build()")
        L = ctypes.CDLL(str(_LIB_PATH))
        P, I32, SZ, F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_float
        I64 = ctypes.c_int64
        cfg_p = ctypes.POINTER(_Config)
        cache_p = ctypes.POINTER(_Cache)
        par_p = ctypes.POINTER(_DgapParams)
        cfg8_p, cache8_p = ctypes.POINTER(_Block8Config), ctypes.POINTER(_Block8Cache)
        sig = {
            "kvq_last_error": (ctypes.c_char_p, []),
            "kvq_version": (I32, []),
            "kvq_validate_config": (I32, [cfg_p]),
            "kvq_page_bytes": (SZ, [cfg_p]),
            "kvq_cache_layout": (I32, [cfg_p, ctypes.POINTER(SZ), ctypes.POINTER(SZ * 4)]),
            "kvq_cache_bind": (I32, [cfg_p, P, cache_p]),
            "kvq_page_pool_bytes": (SZ, [cfg_p, I32]),
            "kvq_paged_cache_layout": (I32, [cfg_p, ctypes.POINTER(SZ),
                                             ctypes.POINTER(SZ * 4)]),
            "kvq_paged_cache_bind": (I32, [cfg_p, P, P, I32, P, cache_p]),
            "kvq_cache_reset": (I32, [cfg_p, cache_p, P]),
            "kvq_pack": (I32, [cfg_p, cache_p, P, P, I32, I32, I32, P]),
            "kvq_attn_workspace_bytes": (SZ, [cfg_p, I32]),
            "kvq_attn_default_splits": (I32, [cfg_p]),
            "kvq_attn_splits_for_lengths": (I32, [cfg_p, ctypes.POINTER(I32)]),
            "kvq_workspace_init": (I32, [P, SZ, P]),
            "kvq_decode_attn": (I32, [cfg_p, cache_p, P, P, F32, I32, P, SZ, P]),
            "kvq_decode_attn_f32": (I32, [cfg_p, cache_p, P, P, F32, I32, P, SZ, P]),
            "kvq_decode_step": (I32, [cfg_p, cache_p, P, P, P, P, F32, I32, P, SZ, P]),
            "kvq_decode_step_f32": (I32, [cfg_p, cache_p, P, P, P, P, F32, I32, P, SZ, P]),
            "kvq_decode_attn_noalloc": (I32, [cfg_p, cache_p, P, P, F32, I32, P]),
            "kvq_chunk_workspace_bytes": (SZ, [cfg_p, I32, I32]),
            "kvq_chunk_attn": (I32, [cfg_p, cache_p, P, P, ctypes.POINTER(_ChunkParams), I32,
                                     I32, P, SZ, P]),
            "kvq_block8_validate_config": (I32, [cfg8_p]),
            "kvq_block8_append": (I32, [cfg8_p, cache8_p, P, P, P]),
            "kvq_block8_workspace_bytes": (SZ, [cfg8_p, I32]),
            "kvq_block8_attn": (I32, [cfg8_p, cache8_p, P, P, P, P, P, SZ, P]),
            "kvq_adjust_logits": (I32, [P, P]),
            "kvq_sample_max_vocab": (I32, []),
            "kvq_sample": (I32, [P, I64, P, I64, I32, I32, P, P, P, P, P, P, P]),
            "dgap_workspace_bytes": (SZ, [I32, I32, par_p]),
            "dgap_restore": (I32, [par_p, P, I32, I32, P, P, P, P, P, P, P, SZ, P]),
            "kvq_drift_max_vocab": (I32, []),
            "kvq_selftest_wait_timeout": (I32, [P, P]),
            "kvq_selftest_chunk_wait_timeout": (I32, [I32, P, P]),
            "kvq_selftest_block8_wait_timeout": (I32, [cfg8_p, cache8_p, P, P, P, P, P, SZ, P]),
            "kvq_drift_metrics": (I32, [P, P, I32, I32, ctypes.POINTER(_DriftParams),
                                        P, P, P, P, P, P]),
            "kvq_drift_window": (I32, [P, I32, I32, F32, P, P, P]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def last_error():
    return lib().kvq_last_error().decode()


def _check(status):
    if status != 0:
        raise KvqError(status, last_error())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _dev(t, dtype, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


# ---------------------------------------------------------------------------
# KV cache
# ---------------------------------------------------------------------------


@dataclass(frozen=True)
class CacheConfig:
    """KbVb cache shape (see kvq_config in include/kvq.h)."""
    batch: int
    n_q_heads: int
    n_kv_heads: int
    bits_k: int
    bits_v: int
    max_len: int
    residual: int = 128
    head_dim: int = 128
    group: int = 32

    def c(self):
        return _Config(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim,
                       self.bits_k, self.bits_v, self.group, self.residual, self.max_len)

    @property
    def ring(self):
        return self.residual + self.group

    @property
    def max_blocks(self):
        return self.max_len // self.group

    @property
    def page_bytes(self):
        return 512 * (self.bits_k + self.bits_v) + 1024

    def validate(self):
        c = self.c()
        _check(lib().kvq_validate_config(ctypes.byref(c)))

    def layout(self):
        c = self.c()
        total = ctypes.c_size_t()
        offs = (ctypes.c_size_t * 4)()
        _check(lib().kvq_cache_layout(ctypes.byref(c), ctypes.byref(total), ctypes.byref(offs)))
        return total.value, tuple(offs)


def packed_len(L, residual=128, group=32):
    """Tokens held in quantized blocks when L tokens are cached."""
    return group * (max(L - residual, 0) // group)


class QuantKVCache:
    """A KbVb cache bound through the C ABI.

    Contiguous (``n_pages=None``): one device buffer from kvq_cache_layout.
    Paged (``n_pages=N``): the fp16 rings and lengths in one buffer
    (kvq_paged_cache_layout), a pool of N page sets and a device block table
    [batch, max_len / 32] of int32 (all -1, i.e. unmapped, at first); the
    caller maps blocks with ``map_blocks`` before a call writes or reads them.
    """

    def __init__(self, cfg: CacheConfig, device="cuda", n_pages=None):
        self.cfg = cfg
        self.n_pages = n_pages
        c = cfg.c()
        self._cfg_ref = ctypes.byref(c)
        if n_pages is None:
            total, self.offsets = cfg.layout()
        else:
            tot = ctypes.c_size_t()
            offs = (ctypes.c_size_t * 4)()
            _check(lib().kvq_paged_cache_layout(ctypes.byref(c), ctypes.byref(tot),
                                                ctypes.byref(offs)))
            total, self.offsets = tot.value, tuple(offs)
        self._raw = torch.empty(total + 256, dtype=torch.uint8, device=device)
        shift = (-self._raw.data_ptr()) % 256
        self.buffer = self._raw[shift:shift + total]
        self._c = _Cache()
        if n_pages is None:
            self.pool = None
            self.block_table = None
            _check(lib().kvq_cache_bind(ctypes.byref(c), ctypes.c_void_p(self.buffer.data_ptr()),
                                        ctypes.byref(self._c)))
        else:
            nbytes = lib().kvq_page_pool_bytes(ctypes.byref(c), int(n_pages))
            if nbytes == 0:
                raise KvqError(1, last_error())
            self.pool = torch.zeros(nbytes, dtype=torch.uint8, device=device)
            self.block_table = torch.full((cfg.batch, cfg.max_blocks), -1, dtype=torch.int32,
                                          device=device)
            _check(lib().kvq_paged_cache_bind(
                ctypes.byref(c), ctypes.c_void_p(self.buffer.data_ptr()),
                ctypes.c_void_p(self.pool.data_ptr()), int(n_pages),
                ctypes.c_void_p(self.block_table.data_ptr()), ctypes.byref(self._c)))
        self._c_ref = ctypes.byref(self._c)
        self.reset()

    @property
    def paged(self):
        return self.n_pages is not None

    def map_blocks(self, b, blocks, page_sets):
        """Paged caches: block_table[b, blocks[i]] = page_sets[i] (a copy to
        the device on the current stream)."""
        if not self.paged:
            raise ValueError("map_blocks needs a paged cache")
        idx = torch.as_tensor(list(blocks), dtype=torch.long)
        val = torch.as_tensor(list(page_sets), dtype=torch.int32)
        self.block_table[b, idx.to(self.block_table.device)] = val.to(self.block_table.device)

    def reset(self, stream=None):
        c = self.cfg.c()
        _check(lib().kvq_cache_reset(ctypes.byref(c), ctypes.byref(self._c), _stream(stream)))

    # Views of the raw storage (layout of include/kvq.h).
    def pages(self):
        """Contiguous caches: the page array [batch, n_kv_heads, max_blocks,
        page_bytes]."""
        cfg = self.cfg
        if self.paged:
            raise ValueError("a paged cache has no page array: use head_pages")
        n = cfg.batch * cfg.n_kv_heads * cfg.max_blocks * cfg.page_bytes
        o = self.offsets[0]
        return self.buffer[o:o + n].view(cfg.batch, cfg.n_kv_heads, cfg.max_blocks,
                                         cfg.page_bytes)

    def pool_sets(self):
        """Paged caches: the pool as [n_pages, n_kv_heads, page_bytes]."""
        cfg = self.cfg
        return self.pool.view(self.n_pages, cfg.n_kv_heads, cfg.page_bytes)

    def head_pages(self, b, h, nb):
        """Blocks 0 .. nb - 1 of (sequence b, kv-head h) as [nb, page_bytes]
        (gathered through the block table for a paged cache)."""
        if not self.paged:
            return self.pages()[b, h, :nb]
        sets = self.block_table[b, :nb].long()
        return self.pool_sets()[sets, h]

    def resid(self):
        cfg = self.cfg
        n = cfg.batch * cfg.n_kv_heads * cfg.ring * cfg.head_dim * 2
        shape = (cfg.batch, cfg.n_kv_heads, cfg.ring, cfg.head_dim)
        k = self.buffer[self.offsets[1]:self.offsets[1] + n].view(torch.float16).view(shape)
        v = self.buffer[self.offsets[2]:self.offsets[2] + n].view(torch.float16).view(shape)
        return k, v

    def seq_region(self):
        o = self.offsets[3]
        return self.buffer[o:o + 4 * (2 * self.cfg.batch + 2)].view(torch.int32)

    def seq_lens(self):
        return self.seq_region()[:self.cfg.batch]

    def flags(self):
        return int(self.seq_region()[self.cfg.batch].item())


def blocks_written(L, n_new, residual=128, group=32):
    """Blocks a call that appends n_new tokens to a sequence of L tokens
    writes: [packed_len(L) / 32, packed_len(L + n_new) / 32)."""
    return range(packed_len(L, residual, group) // group,
                 packed_len(L + n_new, residual, group) // group)


def kvq_pack(cache: QuantKVCache, k_new, v_new, batch_begin=0, stream=None):
    """Append k_new/v_new fp16 [batch_count, n_kv_heads, n_new, 128] to
    sequences [batch_begin, batch_begin + batch_count)."""
    cfg = cache.cfg
    if k_new.dim() != 4 or k_new.shape != v_new.shape or k_new.shape[1] != cfg.n_kv_heads \
            or k_new.shape[3] != cfg.head_dim:
        raise ValueError("k_new/v_new must be [batch_count, n_kv_heads, n_new, 128]")
    c = cfg.c()
    _check(lib().kvq_pack(ctypes.byref(c), ctypes.byref(cache._c),
                          _dev(k_new, torch.float16, "k_new"), _dev(v_new, torch.float16, "v_new"),
                          k_new.shape[2], batch_begin, k_new.shape[0], _stream(stream)))


def attn_workspace(cfg: CacheConfig, n_splits=0, device="cuda"):
    c = cfg.c()
    n = lib().kvq_attn_workspace_bytes(ctypes.byref(c), n_splits)
    if n == 0:
        raise KvqError(1, last_error())
    return torch.zeros(n, dtype=torch.uint8, device=device)


def default_splits(cfg: CacheConfig):
    c = cfg.c()
    return lib().kvq_attn_default_splits(ctypes.byref(c))


def splits_for_lengths(cfg: CacheConfig, lengths):
    """kvq_attn_splits_for_lengths: the plan for host-known lengths, a split
    count (> 0, the split plan) or 0 (the flat plan)."""
    c = cfg.c()
    arr = (ctypes.c_int32 * cfg.batch)(*[int(x) for x in lengths])
    n = lib().kvq_attn_splits_for_lengths(ctypes.byref(c), arr)
    if n < 0:
        raise KvqError(1, last_error())
    return n


def _attn_out(q, out, out_dtype):
    """The output tensor and the entry-point suffix for its dtype."""
    if out is None:
        out = torch.empty(q.shape, dtype=out_dtype, device=q.device)
    if out.dtype == torch.float16:
        return out, ""
    if out.dtype == torch.float32:
        return out, "_f32"
    raise TypeError(f"out must be float16 or float32, got {out.dtype}")


def kvq_decode_attn(cache: QuantKVCache, q, out=None, softmax_scale=0.0, n_splits=0,
                    workspace=None, stream=None, out_dtype=torch.float16):
    """out = softmax(q K^T * scale) V over the cache; q fp16 [batch, n_q_heads, 128].

    out fp16 (the fp32 result rounded to nearest, kvq_decode_attn) or fp32
    (kvq_decode_attn_f32), picked by the dtype of ``out`` or ``out_dtype``."""
    cfg = cache.cfg
    if q.shape != (cfg.batch, cfg.n_q_heads, cfg.head_dim):
        raise ValueError(f"q must be [{cfg.batch}, {cfg.n_q_heads}, {cfg.head_dim}]")
    out, suffix = _attn_out(q, out, out_dtype)
    if out.shape != q.shape:
        raise ValueError("out must have the shape of q")
    if workspace is None:
        workspace = attn_workspace(cfg, n_splits, q.device)
    c = cfg.c()
    fn = getattr(lib(), "kvq_decode_attn" + suffix)
    _check(fn(ctypes.byref(c), ctypes.byref(cache._c), _dev(q, torch.float16, "q"),
              _dev(out, out.dtype, "out"), float(softmax_scale), n_splits,
              _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)))
    return out


def kvq_decode_step(cache: QuantKVCache, k_new, v_new, q, out=None, softmax_scale=0.0,
                    n_splits=0, workspace=None, stream=None, out_dtype=torch.float16):
    """Append one token per sequence (k_new / v_new fp16 [batch, n_kv_heads, 128])
    and attend (q fp16 [batch, n_q_heads, 128] -> out fp16, or fp32 as in
    kvq_decode_attn) in one call: the same results as kvq_pack then
    kvq_decode_attn."""
    cfg = cache.cfg
    if q.shape != (cfg.batch, cfg.n_q_heads, cfg.head_dim):
        raise ValueError(f"q must be [{cfg.batch}, {cfg.n_q_heads}, {cfg.head_dim}]")
    for name, t in (("k_new", k_new), ("v_new", v_new)):
        if t.shape != (cfg.batch, cfg.n_kv_heads, cfg.head_dim):
            raise ValueError(f"{name} must be [{cfg.batch}, {cfg.n_kv_heads}, {cfg.head_dim}]")
    out, suffix = _attn_out(q, out, out_dtype)
    if out.shape != q.shape:
        raise ValueError("out must have the shape of q")
    if workspace is None:
        workspace = attn_workspace(cfg, n_splits, q.device)
    c = cfg.c()
    fn = getattr(lib(), "kvq_decode_step" + suffix)
    _check(fn(ctypes.byref(c), ctypes.byref(cache._c), _dev(k_new, torch.float16, "k_new"),
              _dev(v_new, torch.float16, "v_new"), _dev(q, torch.float16, "q"),
              _dev(out, out.dtype, "out"), float(softmax_scale), n_splits,
              _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)))
    return out


def kvq_decode_attn_noalloc(cache: QuantKVCache, q, out, softmax_scale=0.0, n_splits=0,
                            stream=None):
    """kvq_decode_attn_f32 with the library's built-in scratch array instead of
    a workspace, for callers that cannot allocate device memory per step.
    ``out`` (fp32, the shape of q) is required: this wrapper allocates
    nothing either.  Calls share the array: do not let two of them overlap on
    the GPU."""
    cfg = cache.cfg
    if q.shape != (cfg.batch, cfg.n_q_heads, cfg.head_dim):
        raise ValueError(f"q must be [{cfg.batch}, {cfg.n_q_heads}, {cfg.head_dim}]")
    if out is None or out.shape != q.shape:
        raise ValueError("out must be a preallocated fp32 tensor of q's shape")
    c = cfg.c()
    _check(lib().kvq_decode_attn_noalloc(ctypes.byref(c), ctypes.byref(cache._c),
                                         _dev(q, torch.float16, "q"),
                                         _dev(out, torch.float32, "out"), float(softmax_scale),
                                         n_splits, _stream(stream)))
    return out


def _in_32_bits(names, *numbers):
    """ctypes cuts an int to its argument's 32 bits without a word."""
    for x in numbers:
        if not -2147483648 <= x <= 2147483647:
            raise ValueError(f"{names} must fit 32 bits (got {x})")


def chunk_workspace(cfg: CacheConfig, n_q, batch_count=None, device="cuda"):
    """A workspace for kvq_chunk_attn of n_q queries per sequence."""
    c = cfg.c()
    batch_count = cfg.batch if batch_count is None else batch_count
    _in_32_bits("n_q and batch_count", n_q, batch_count)
    n = lib().kvq_chunk_workspace_bytes(ctypes.byref(c), n_q, batch_count)
    if n == 0:
        raise KvqError(1, last_error())
    return torch.empty(n, dtype=torch.uint8, device=device)


def _made_on(stream, make, *args):
    """make(*args) with ``stream`` (None: the current one) as the current stream:
    what a call allocates for itself belongs to the stream that it launches on, so
    the allocator hands its memory to no other stream while the call still runs."""
    if stream is None:
        return make(*args)
    with torch.cuda.stream(stream):
        return make(*args)


def _address(t, dtype, name):
    """Data pointer of a CUDA tensor of ``dtype`` whose last dimension is
    contiguous (the others may have any strides)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return t.data_ptr()


def _strides(t):
    # the stride of a dimension of size 1 says nothing
    return tuple(s if n > 1 else 0 for s, n in zip(t.stride()[:3], t.shape))


def kvq_chunk_attn(cache: QuantKVCache, q, out=None, window=0, sinks=0, softmax_scale=0.0,
                   batch_begin=0, workspace=None, stream=None):
    """Causal attention of the n_q newest tokens of sequences [batch_begin,
    batch_begin + batch_count), which kvq_pack has appended before: q fp16
    [batch_count, n_q, n_q_heads, 128] (strided views too) -> out fp16 of that
    shape.  window > 0: each query sees the ``window`` newest tokens up to its
    own and the first ``sinks`` tokens.  n_q = 1 is the windowed form of a
    decode step."""
    cfg, shape = cache.cfg, q.shape
    if len(shape) != 4 or shape[2] != cfg.n_q_heads or shape[3] != cfg.head_dim:
        raise ValueError(f"q must be [batch_count, n_q, {cfg.n_q_heads}, {cfg.head_dim}]")
    _in_32_bits("window and sinks", window, sinks)
    _in_32_bits("batch_begin, batch_count and n_q", batch_begin, shape[0], shape[1])
    if out is None:
        out = _made_on(stream, lambda: torch.empty(shape, dtype=torch.float16, device=q.device))
    elif out.shape != shape:
        raise ValueError("out must have the shape of q")
    batch_count, n_q = shape[0], shape[1]
    if workspace is None:
        workspace = _made_on(stream, chunk_workspace, cfg, n_q, batch_count, q.device)
    p = _ChunkParams(n_q, int(window), int(sinks), float(softmax_scale), _strides(q),
                     _strides(out))
    _check(lib().kvq_chunk_attn(cache._cfg_ref, cache._c_ref, _address(q, torch.float16, "q"),
                                _address(out, torch.float16, "out"), ctypes.byref(p),
                                batch_begin, batch_count,
                                _dev(workspace, torch.uint8, "workspace"),
                                workspace.numel(), _stream(stream)))
    return out


# ---------------------------------------------------------------------------
# Block-8 cache
# ---------------------------------------------------------------------------

_BLOCK8_TYPES = {torch.float16: 0, torch.bfloat16: 1}
_LOGIT_TYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
BLOCK8_RING = 64


@dataclass(frozen=True)
class Block8Config:
    """Shape of a block-8 cache (see kvq_block8_config in include/kvq.h)."""
    batch: int
    n_q_heads: int
    n_kv_heads: int
    max_len: int
    dtype: torch.dtype = torch.float16
    head_dim: int = 128
    block: int = 32

    def c(self):
        _in_32_bits("sizes", self.batch, self.n_q_heads, self.n_kv_heads, self.max_len)
        return _Block8Config(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim,
                             self.block, self.max_len, _BLOCK8_TYPES.get(self.dtype, -1))

    @property
    def max_blocks(self):
        return self.max_len // self.block

    def validate(self):
        c = self.c()
        _check(lib().kvq_block8_validate_config(ctypes.byref(c)))


def block8_written(length, n_new):
    """Blocks that appending n_new tokens to ``length`` completes."""
    return range(length // 32, (length + n_new) // 32)


class Block8Cache:
    """A paged cache of e4m3 blocks, one scale per 32 tokens and kv-head.

    ``n_pages`` makes its tensors (all blocks unmapped); ``tensors`` takes the
    caller's own: a dict of k_codes, v_codes (float8_e4m3fn [n_pages, n_kv_heads,
    32, 128]), scales (fp32 [n_pages, n_kv_heads, 2]), k_ring, v_ring (cfg.dtype
    [batch, n_kv_heads, 64, 128]).  ``block_table`` (int32 [batch, max_len / 32])
    may be shared by the caches of several layers.  Lengths are the caller's too:
    each call gets them."""

    def __init__(self, cfg: Block8Config, n_pages=None, device="cuda", tensors=None,
                 block_table=None):
        cfg.validate()
        self.cfg = cfg
        if (n_pages is None) == (tensors is None):
            raise ValueError("give either n_pages or tensors")
        h, d = cfg.n_kv_heads, cfg.head_dim
        if tensors is None:
            _in_32_bits("n_pages", n_pages)
            if n_pages < 1:
                raise ValueError(f"n_pages must be >= 1 (got {n_pages})")
            tensors = {n: torch.zeros(n_pages, h, 32, d, dtype=torch.uint8, device=device)
                       .view(torch.float8_e4m3fn) for n in ("k_codes", "v_codes")}
            tensors["scales"] = torch.ones(n_pages, h, 2, dtype=torch.float32, device=device)
            for n in ("k_ring", "v_ring"):
                tensors[n] = torch.zeros(cfg.batch, h, BLOCK8_RING, d, dtype=cfg.dtype,
                                         device=device)
        self.n_pages = tensors["scales"].shape[0]
        code, ring = (self.n_pages, h, 32, d), (cfg.batch, h, BLOCK8_RING, d)
        want = {"k_codes": (torch.float8_e4m3fn, code), "v_codes": (torch.float8_e4m3fn, code),
                "scales": (torch.float32, (self.n_pages, h, 2)), "k_ring": (cfg.dtype, ring),
                "v_ring": (cfg.dtype, ring)}
        for n, (dtype, shape) in want.items():
            if tuple(tensors[n].shape) != shape:
                raise ValueError(f"{n} must be {list(shape)}")
            _dev(tensors[n], dtype, n)
            setattr(self, n, tensors[n])
        self.device = self.scales.device
        self.dev = self.scales.get_device()
        if block_table is None:
            block_table = torch.full((cfg.batch, cfg.max_blocks), -1, dtype=torch.int32,
                                     device=self.device)
        elif tuple(block_table.shape) != (cfg.batch, cfg.max_blocks):
            raise ValueError(f"block_table must be [{cfg.batch}, {cfg.max_blocks}]")
        _dev(block_table, torch.int32, "block_table")
        self.block_table = block_table
        self._flags = torch.zeros(1, dtype=torch.int32, device=self.device)
        for t in (self.k_codes, self.v_codes, self.k_ring, self.v_ring, block_table):
            if t.device != self.device:
                raise ValueError("a cache's tensors must be on one device")
        self._cfg = cfg.c()
        self._c = _Block8Cache(*(t.data_ptr() for t in (
            self.k_codes, self.v_codes, self.scales, self.k_ring, self.v_ring, block_table,
            self._flags)), self.n_pages)
        self._cfg_ref, self._c_ref = ctypes.byref(self._cfg), ctypes.byref(self._c)

    def map_blocks(self, b, blocks, pages):
        """block_table[b, blocks[i]] = pages[i] (a copy on the current stream)."""
        idx = torch.as_tensor(list(blocks), dtype=torch.long)
        val = torch.as_tensor(list(pages), dtype=torch.int32)
        self.block_table[b, idx.to(self.device)] = val.to(self.device)

    def flags(self):
        return int(self._flags.item())

    def clear_flags(self):
        self._flags.zero_()


# The calls below pack their structs with these: a ctypes structure's fields cost more to
# set, one by one, than the smallest calls take on the GPU.
_BATCH = struct.Struct("@2P2i")             # kvq_block8_batch
_APPEND = struct.Struct("@7P3i8q")          # kvq_block8_append_params
_ATTN = struct.Struct("@2if4q")             # kvq_block8_attn_params
_ADJUST = struct.Struct("@13P3q6i")         # kvq_adjust_params


def _rows(t, n, heads, dtype, name, dev):
    """Address and strides (tokens, heads) of an [n, heads, 128] tensor on GPU `dev`."""
    if t.shape != (n, heads, 128):
        raise ValueError(f"{name} must be [{n}, {heads}, 128]")
    if t.dtype is not dtype or t.get_device() != dev:
        raise TypeError(f"{name} must be {dtype} on cuda:{dev}, got {t.dtype} on {t.device}")
    s0, s1, s2 = t.stride()
    if s2 != 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return t.data_ptr(), s0 if n > 1 else 0, s1 if heads > 1 else 0


def _list(t, n, dtype, name, dev):
    """Address of a contiguous 1-d tensor of n elements (None: any number) on GPU `dev`,
    0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != dev:
        raise TypeError(f"{name} must be {dtype} on cuda:{dev}, got {t.dtype} on {t.device}")
    if t.dim() != 1 or (n is not None and t.shape[0] != n) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous [{'n' if n is None else n}]")
    return t.data_ptr()


def _block8_batch(cache, n_tokens, lengths, starts, max_new):
    batch = cache.cfg.batch
    if starts is None:
        if n_tokens % batch:
            raise ValueError("without starts, every sequence has as many new tokens")
        if max_new not in (None, n_tokens // batch):
            raise ValueError("without starts, max_new is the tokens of each sequence")
        max_new = n_tokens // batch
    elif max_new is None:
        max_new = min(n_tokens, cache.cfg.max_len)
    if not (0 <= n_tokens <= 2147483647 and 0 <= max_new <= 2147483647):
        raise ValueError(f"n_tokens and max_new must be in [0, 2^31) (got {n_tokens}, {max_new})")
    return _BATCH.pack(_list(lengths, batch, torch.int32, "lengths", cache.dev),
                       _list(starts, batch + 1, torch.int32, "starts", cache.dev), n_tokens,
                       max_new), max_new


def _launch(dev, stream, fn, *args):
    """fn(*args, stream) with GPU `dev` current, on its current stream where none is given."""
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(dev)
    elif stream.device.index != dev:
        raise ValueError(f"stream must be on cuda:{dev}")
    else:
        handle = stream.cuda_stream
    was = torch._C._cuda_getDevice()
    if was == dev:
        status = fn(*args, handle)
    else:
        with torch.cuda.device(dev):
            status = fn(*args, handle)
    if status:
        _check(status)


def kvq_block8_append(cache: Block8Cache, k, v, lengths, starts=None, q=None, q_out=None,
                      cos=None, sin=None, paired=False, positions=None, max_new=None,
                      stream=None):
    """Append the newest tokens of each sequence, keys (and queries) rotated on the way.

    k, v [tokens, n_kv_heads, 128] and q [tokens, n_q_heads, 128] in cfg.dtype, strided
    views of one projection too; rows starts[b] .. starts[b + 1] - 1 are sequence b's
    (starts int32 [batch + 1] on the device; None: as many for each), the last of them
    at position lengths[b] - 1 (int32 [batch], new tokens included).  cos, sin fp32
    [n_positions, rot_dim / 2] (None: no rotation); ``paired`` rotates channels (2i,
    2i + 1) instead of (i, i + rot_dim / 2); ``positions`` int32 [tokens] are rows of
    the tables in place of the tokens' places.  Returns q_out (made if None; may be
    q), or None without q."""
    cfg, dev = cache.cfg, cache.dev
    n, dtype = k.shape[0], cfg.dtype
    batch, _ = _block8_batch(cache, n, lengths, starts, max_new)
    ka, k0, k1 = _rows(k, n, cfg.n_kv_heads, dtype, "k", dev)
    va, v0, v1 = _rows(v, n, cfg.n_kv_heads, dtype, "v", dev)
    qa = q0 = q1 = oa = o0 = o1 = 0
    if q is not None:
        qa, q0, q1 = _rows(q, n, cfg.n_q_heads, dtype, "q", dev)
        if q_out is None:
            q_out = _made_on(stream, lambda: torch.empty(q.shape, dtype=dtype,
                                                         device=cache.device))
        oa, o0, o1 = _rows(q_out, n, cfg.n_q_heads, dtype, "q_out", dev)
    elif q_out is not None:
        raise ValueError("q_out needs q")
    ca = sa = pa = n_pos = rot = 0
    if cos is not None or sin is not None:
        if cos is None or sin is None or cos.dim() != 2 or cos.shape != sin.shape:
            raise ValueError("cos and sin must both be [n_positions, rot_dim / 2]")
        n_pos, half = cos.shape
        rot = 2 * half
        if rot:
            for t, name in ((cos, "cos"), (sin, "sin")):
                if t.dtype is not torch.float32 or t.get_device() != dev:
                    raise TypeError(f"{name} must be float32 on cuda:{dev}")
                if not t.is_contiguous():
                    raise ValueError(f"{name} must be contiguous")
            ca, sa = cos.data_ptr(), sin.data_ptr()
            pa = _list(positions, n, torch.int32, "positions", dev)
    params = _APPEND.pack(ka, va, qa, oa, ca, sa, pa, n_pos, rot, 1 if paired else 0,
                          k0, k1, v0, v1, q0, q1, o0, o1)
    _launch(dev, stream, lib().kvq_block8_append, cache._cfg_ref, cache._c_ref, batch, params)
    return q_out


def block8_workspace(cfg: Block8Config, max_new, device="cuda"):
    """A workspace for kvq_block8_attn of up to max_new new tokens a sequence."""
    c = cfg.c()
    _in_32_bits("max_new", max_new)
    n = lib().kvq_block8_workspace_bytes(ctypes.byref(c), max_new)
    if n == 0:
        raise KvqError(1, last_error())
    return torch.zeros(n, dtype=torch.uint8, device=device)


def kvq_block8_attn(cache: Block8Cache, q, lengths, starts=None, max_new=None, window=0, sinks=0,
                    softmax_scale=0.0, out=None, workspace=None, stream=None):
    """Causal attention of the newest tokens of each sequence, which kvq_block8_append
    has appended: q [tokens, n_q_heads, 128] (rotated; strided views too) -> out of that
    shape.  lengths, starts as there; ``max_new`` is the most new tokens of any sequence
    (a smaller number serves single tokens and drafts faster).  window, sinks as in
    kvq_chunk_attn.  Without a ``workspace`` (block8_workspace of that max_new or more) each
    call makes and zeroes one."""
    cfg, dev = cache.cfg, cache.dev
    n = q.shape[0]
    batch, max_new = _block8_batch(cache, n, lengths, starts, max_new)
    _in_32_bits("window and sinks", window, sinks)
    qa, q0, q1 = _rows(q, n, cfg.n_q_heads, cfg.dtype, "q", dev)
    if out is None:
        out = _made_on(stream, lambda: torch.empty(q.shape, dtype=cfg.dtype,
                                                   device=cache.device))
    oa, o0, o1 = _rows(out, n, cfg.n_q_heads, cfg.dtype, "out", dev)
    if workspace is None:
        workspace = _made_on(stream, block8_workspace, cfg, max_new, cache.device)
    ws = _list(workspace, None, torch.uint8, "workspace", dev)
    params = _ATTN.pack(window, sinks, softmax_scale, q0, q1, o0, o1)
    _launch(dev, stream, lib().kvq_block8_attn, cache._cfg_ref, cache._c_ref, batch, qa, oa,
            params, ws, workspace.numel())
    return out


# ---------------------------------------------------------------------------
# Adjusted logits
# ---------------------------------------------------------------------------


def kvq_adjust_logits(logits, out=None, history=None, history_starts=None, prompt_lengths=None,
                      repetition=None, frequency=None, presence=None, bias_ids=None,
                      bias_values=None, bias_starts=None, mask=None, mask_rows=None,
                      stream=None):
    """Penalties for repeated tokens, biases and a grammar's mask on logits [rows, vocab]
    (fp32, fp16 or bf16; rows may be strided) -> fp32 ``out``, which may be the logits.

    history, bias_ids (int32) and bias_values (fp32) hold all rows' lists one behind the
    other, row b's at starts[b] .. starts[b + 1] - 1 (int32 [rows + 1]); the first
    prompt_lengths[b] tokens of a history were asked, the others answered.  repetition,
    frequency, presence are fp32 [rows]; mask int32 [n, ceil(vocab / 32)] of bits, row b's
    at mask_rows[b] (None: b).  All on the device."""
    shape = logits.shape
    if len(shape) != 2:
        raise ValueError("logits must be [rows, vocab]")
    rows, V = shape
    dev = logits.get_device()
    if dev < 0:
        raise TypeError("logits must be a CUDA tensor")
    _in_32_bits("rows and vocab", rows, V)
    dtype = _LOGIT_TYPES.get(logits.dtype)
    if dtype is None:
        raise TypeError(f"logits must be float32, float16 or bfloat16, got {logits.dtype}")
    f32, i32 = torch.float32, torch.int32
    if out is None:
        out = _made_on(stream, lambda: torch.empty(rows, V, dtype=f32, device=logits.device))
    elif out.shape != shape:
        raise ValueError("out must have the logits' shape")
    elif out.dtype is not f32 or out.get_device() != dev:
        raise TypeError(f"out must be float32 on cuda:{dev}")
    z0, z1 = logits.stride()
    o0, o1 = out.stride()
    if V > 1 and (z1 != 1 or o1 != 1):
        raise ValueError("the last dimension of logits and out must be contiguous")
    n_history = 0 if history is None else history.numel()
    n_bias = 0 if bias_ids is None else bias_ids.numel()
    if n_bias and (bias_values is None or bias_values.shape != bias_ids.shape):
        raise ValueError("bias_values must have the shape of bias_ids")
    mask_at = n_masks = mask_stride = 0
    if mask is not None:
        if mask.dim() != 2 or mask.shape[1] < (V + 31) // 32 or mask.stride(1) != 1:
            raise ValueError("mask must be [n, ceil(vocab / 32)], its rows contiguous")
        if mask.dtype is not i32 or mask.get_device() != dev:
            raise TypeError(f"mask must be int32 on cuda:{dev}")
        mask_at, n_masks, mask_stride = mask.data_ptr(), mask.shape[0], mask.stride(0)
    _in_32_bits("lists", n_history, n_bias)
    params = _ADJUST.pack(
        logits.data_ptr(), out.data_ptr(), _list(history, None, i32, "history", dev),
        _list(history_starts, rows + 1, i32, "history_starts", dev),
        _list(prompt_lengths, rows, i32, "prompt_lengths", dev),
        _list(repetition, rows, f32, "repetition", dev),
        _list(frequency, rows, f32, "frequency", dev),
        _list(presence, rows, f32, "presence", dev),
        _list(bias_ids, None, i32, "bias_ids", dev),
        _list(bias_values, None, f32, "bias_values", dev),
        _list(bias_starts, rows + 1, i32, "bias_starts", dev), mask_at,
        _list(mask_rows, rows, i32, "mask_rows", dev), z0, o0, mask_stride, dtype, rows, V,
        n_history, n_bias, n_masks)
    _launch(dev, stream, lib().kvq_adjust_logits, params)
    return out


# ---------------------------------------------------------------------------
# Sampling
# ---------------------------------------------------------------------------


def sample_outputs(batch, device="cuda"):
    """The result tensors of kvq_sample."""
    return dict(token=torch.empty(batch, dtype=torch.int32, device=device),
                logprob=torch.empty(batch, dtype=torch.float32, device=device))


def _per_row(t, shape, dtype, name):
    if t is None:
        return None
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}")
    return _address(t, dtype, name)


def kvq_sample(logits, noise=None, temperature=None, top_k=None, top_p=None, min_p=None,
               outputs=None, stream=None):
    """The next token of each row of fp32 logits [batch, vocab] (rows may be
    strided) from ``noise``, fp32 uniform numbers in [0, 1) of the same shape.
    temperature, top_p, min_p (fp32) and top_k (int32) are device tensors
    [batch] or None; noise None is greedy.  Returns a dict of device tensors:
    token (int32) and logprob (fp32, may be None in ``outputs``)."""
    shape = logits.shape
    if len(shape) != 2:
        raise ValueError("logits must be [batch, vocab]")
    B, V = shape
    _in_32_bits("batch and vocab", B, V)
    f32 = torch.float32
    z = _address(logits, f32, "logits")
    u = _per_row(noise, shape, f32, "noise")
    o = _made_on(stream, sample_outputs, B, logits.device) if outputs is None else outputs
    row = shape[:1]
    _check(lib().kvq_sample(
        z, logits.stride(0), u, 0 if noise is None else noise.stride(0), B, V,
        _per_row(temperature, row, f32, "temperature"), _per_row(top_k, row, torch.int32, "top_k"),
        _per_row(top_p, row, f32, "top_p"), _per_row(min_p, row, f32, "min_p"),
        _per_row(o["token"], row, torch.int32, "token"),
        _per_row(o.get("logprob"), row, f32, "logprob"), _stream(stream)))
    return o


# ---------------------------------------------------------------------------
# DGAP epilogue
# ---------------------------------------------------------------------------


class DGAP:
    """Detector + corrector weights (device fp32) and the restore call."""

    def __init__(self, weights, K=32, tau=0.60, device="cuda"):
        self.K = int(K)
        self.tau = float(tau)
        self.w = {k: torch.as_tensor(v, dtype=torch.float32).to(device).contiguous()
                  for k, v in weights.items()}
        self.hidden = int(self.w["det_w1"].shape[0])
        nin = 5 * self.K + 8
        expect = {"det_w1": (self.hidden, 8), "det_b1": (self.hidden,),
                  "det_w2": (self.hidden,), "det_b2": (1,),
                  "cor_w1": (self.hidden, nin), "cor_b1": (self.hidden,),
                  "cor_w2": (self.K, self.hidden), "cor_b2": (self.K,)}
        for k, shp in expect.items():
            if tuple(self.w[k].shape) != shp:
                raise ValueError(f"{k} must have shape {shp}, got {tuple(self.w[k].shape)}")

    def params(self, tau=None):
        w = self.w
        return _DgapParams(self.K, self.hidden, float(self.tau if tau is None else tau),
                           *(ctypes.c_void_p(w[k].data_ptr()) for k in (
                               "det_w1", "det_b1", "det_w2", "det_b2",
                               "cor_w1", "cor_b1", "cor_w2", "cor_b2")))

    def workspace(self, batch, vocab, device="cuda"):
        p = self.params()
        n = lib().dgap_workspace_bytes(batch, vocab, ctypes.byref(p))
        if n == 0:
            raise KvqError(1, last_error())
        return torch.zeros(n, dtype=torch.uint8, device=device)

    def restore(self, logits, tau=None, outputs=None, workspace=None, features=True,
                next_token=True, stream=None):
        """Run dgap_restore on fp32 logits [batch, vocab] in place.

        Returns a dict of device tensors: topk_idx, topk_val, risk, gate,
        next_token, features (the last two may be None)."""
        if logits.dim() != 2:
            raise ValueError("logits must be [batch, vocab]")
        B, V = logits.shape
        dev = logits.device
        if outputs is None:
            outputs = dict(
                topk_idx=torch.empty(B, self.K, dtype=torch.int32, device=dev),
                topk_val=torch.empty(B, self.K, dtype=torch.float32, device=dev),
                risk=torch.empty(B, dtype=torch.float32, device=dev),
                gate=torch.empty(B, dtype=torch.uint8, device=dev),
                next_token=torch.empty(B, dtype=torch.int32, device=dev) if next_token else None,
                features=torch.empty(B, 8, dtype=torch.float32, device=dev) if features else None)
        if workspace is None:
            workspace = self.workspace(B, V, dev)
        p = self.params(tau)
        o = outputs

        def opt(t, dt, name):
            return ctypes.c_void_p(None) if t is None else _dev(t, dt, name)

        _check(lib().dgap_restore(
            ctypes.byref(p), _dev(logits, torch.float32, "logits"), B, V,
            _dev(o["topk_idx"], torch.int32, "topk_idx"),
            _dev(o["topk_val"], torch.float32, "topk_val"),
            _dev(o["risk"], torch.float32, "risk"), _dev(o["gate"], torch.uint8, "gate"),
            opt(o.get("next_token"), torch.int32, "next_token"),
            opt(o.get("features"), torch.float32, "features"),
            _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)))
        return o


def logit(tau):
    """log(tau / (1 - tau)); the gate r > tau is f > logit(tau)."""
    if tau >= 1.0:
        return math.inf
    if tau <= 0.0:
        return -math.inf
    return math.log(tau / (1.0 - tau))


# ---------------------------------------------------------------------------
# Offline drift metrics (Sec. 4.1, Sec. 4.2)
# ---------------------------------------------------------------------------

def drift_metrics(z_fp, z_q, alpha, window, k_max, eps, rho_c, outputs=None, stream=None):
    """kvq_drift_metrics on paired fp32 logits [rows, vocab].

    Returns a dict of device tensors: m_t (int32), c_t, d_loc (fp32),
    y_t (uint8) per row and cov [rows, k_max] (fp32)."""
    if z_fp.dim() != 2 or z_fp.shape != z_q.shape:
        raise ValueError("z_fp and z_q must both be [rows, vocab]")
    R, V = z_fp.shape
    dev = z_fp.device
    if outputs is None:
        outputs = dict(m_t=torch.empty(R, dtype=torch.int32, device=dev),
                       c_t=torch.empty(R, dtype=torch.float32, device=dev),
                       d_loc=torch.empty(R, dtype=torch.float32, device=dev),
                       y_t=torch.empty(R, dtype=torch.uint8, device=dev),
                       cov=torch.empty(R, k_max, dtype=torch.float32, device=dev))
    o = outputs
    p = _DriftParams(float(alpha), int(window), int(k_max), float(eps), float(rho_c))
    _check(lib().kvq_drift_metrics(
        _dev(z_fp, torch.float32, "z_fp"), _dev(z_q, torch.float32, "z_q"), R, V, ctypes.byref(p),
        _dev(o["m_t"], torch.int32, "m_t"), _dev(o["c_t"], torch.float32, "c_t"),
        _dev(o["d_loc"], torch.float32, "d_loc"), _dev(o["y_t"], torch.uint8, "y_t"),
        _dev(o["cov"], torch.float32, "cov"), _stream(stream)))
    return o


def drift_window(cov, rho_k, stream=None):
    """kvq_drift_window: (K_b as a device int32 [1], mean coverage [k_max])."""
    if cov.dim() != 2:
        raise ValueError("cov must be [rows, k_max]")
    R, K = cov.shape
    mean = torch.empty(K, dtype=torch.float32, device=cov.device)
    kb = torch.empty(1, dtype=torch.int32, device=cov.device)
    _check(lib().kvq_drift_window(_dev(cov, torch.float32, "cov"), R, K, float(rho_k),
                                  _dev(mean, torch.float32, "mean_cov"),
                                  _dev(kb, torch.int32, "k_b"), _stream(stream)))
    return kb, mean


def selftest_wait_timeout(stream=None):
    """kvq_selftest_wait_timeout: the device flag word after a bounded wait on
    a copy that never arrives ran out (KVQ_FLAG_WAIT_TIMEOUT expected)."""
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    _check(lib().kvq_selftest_wait_timeout(_dev(flag, torch.int32, "flag"), _stream(stream)))
    return flag


def selftest_block8_wait_timeout(cache: Block8Cache, q, lengths, workspace, stream=None):
    """kvq_selftest_block8_wait_timeout: kvq_block8_attn whose waits run out, as many new tokens
    for each sequence; the flag is in ``cache.flags()``."""
    n = q.shape[0]
    batch, _ = _block8_batch(cache, n, lengths, None, None)
    out = torch.empty_like(q)
    qa, q0, q1 = _rows(q, n, cache.cfg.n_q_heads, cache.cfg.dtype, "q", cache.dev)
    oa, o0, o1 = _rows(out, n, cache.cfg.n_q_heads, cache.cfg.dtype, "out", cache.dev)
    ws = _list(workspace, None, torch.uint8, "workspace", cache.dev)
    _launch(cache.dev, stream, lib().kvq_selftest_block8_wait_timeout, cache._cfg_ref,
            cache._c_ref, batch, qa, oa, _ATTN.pack(0, 0, 0.0, q0, q1, o0, o1), ws,
            workspace.numel())


def selftest_chunk_wait_timeout(role, stream=None):
    """kvq_selftest_chunk_wait_timeout: the flag word after the waits of a role
    (0 softmax, 1 loading, 2 issuing) of the chunk attention ran out."""
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    _check(lib().kvq_selftest_chunk_wait_timeout(role, _dev(flag, torch.int32, "flag"),
                                                 _stream(stream)))
    return flag
