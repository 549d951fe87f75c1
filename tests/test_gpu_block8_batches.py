"""Batches of the block-8 calls whose ranges overlap, and calls with large limits."""

import numpy as np
import pytest
import torch

from oracle import block8
from paper_2607_16248_gb300 import kvq
from test_gpu_block8 import np64
from test_gpu_block8_edges import check, filled, ints

pytestmark = pytest.mark.gpu


class Appended:
    """An append of random rows with the given starts and lengths into an empty cache."""

    def __init__(self, starts, lengths, n, max_new=None, hkv=2, rot=64):
        self.batch = len(lengths)
        self.max_len = (max(lengths) + 31) // 32 * 32
        self.cfg = kvq.Block8Config(self.batch, 2 * hkv, hkv, self.max_len)
        pages = self.batch * self.cfg.max_blocks
        self.cache = kvq.Block8Cache(self.cfg, n_pages=pages)
        self.cache.block_table.copy_(torch.arange(pages, dtype=torch.int32).view(self.batch, -1))
        g = torch.Generator().manual_seed(n)
        self.k, self.v, self.q = (torch.randn(n, h, 128, generator=g).half().cuda()
                                  for h in (hkv, hkv, 2 * hkv))
        angle = torch.arange(self.max_len)[:, None] / 100.0 ** (torch.arange(rot // 2) / rot)
        self.cos, self.sin = angle.cos(), angle.sin()
        self.out = torch.full_like(self.q, 7.0)
        kvq.kvq_block8_append(self.cache, self.k, self.v, ints(lengths), starts=ints(starts),
                              q=self.q, q_out=self.out, cos=self.cos.cuda(), sin=self.sin.cuda(),
                              max_new=max_new)
        self.starts, self.lengths = starts, lengths

    def check_appended(self, b):
        rows, L = range(self.starts[b], self.starts[b + 1]), self.lengths[b]
        pos, v = np.arange(L - len(rows), L), np64(self.v[list(rows)])
        k = block8.rotate(np64(self.k[list(rows)]), self.cos.numpy()[pos], self.sin.numpy()[pos],
                          False)
        assert L == len(rows)           # (all of the sequence is new here)
        for h in range(self.cfg.n_kv_heads):
            for i, (x, codes, ring) in enumerate((
                    (block8.to_type(k[:, h], "fp16"), self.cache.k_codes, self.cache.k_ring),
                    (v[:, h], self.cache.v_codes, self.cache.v_ring))):
                got, scales = np64(codes.float()[:, h]), np64(self.cache.scales[:, h, i])
                for j in range(L // 32):
                    page = b * self.cfg.max_blocks + j
                    c, s = block8.quantize(x[32 * j:32 * j + 32])
                    assert scales[page] == s and np.array_equal(got[page], c), (b, h, i, j)
                last = np64(ring[b, h])
                for p in range(max(0, (L // 32 - 1) * 32), L):
                    assert np.array_equal(last[p % 64], x[p]), (b, h, i, p)

    def check_alone(self, b):
        pages = slice(b * self.cfg.max_blocks, (b + 1) * self.cfg.max_blocks)
        assert (self.cache.k_codes.view(torch.uint8)[pages] == 0).all()
        assert (self.cache.v_codes.view(torch.uint8)[pages] == 0).all()
        assert (self.cache.scales[pages] == 1).all()
        assert (self.cache.k_ring[b] == 0).all() and (self.cache.v_ring[b] == 0).all()

    def check_queries(self, b, rows):
        """Rows of q go by sequence b's positions: two products and a sum in fp32, half a step."""
        pos = self.lengths[b] - self.starts[b + 1] + np.array(rows)
        x = np64(self.q[list(rows)])
        want = block8.rotate(x, self.cos.numpy()[pos], self.sin.numpy()[pos], False)
        bound = 2.0 ** -11 * np.abs(want) + 4 * 2.0 ** -24 * 2 * np.abs(x).max() + 2.0 ** -25
        assert (np.abs(np64(self.out[list(rows)]) - want) <= bound).all()


def test_overlapping_ranges_that_do_not_fit(kvq_lib):
    """Two sequences of the same 5000 rows: the second would lose most of its blocks, so it is
    left alone."""
    a = Appended([0, 5000, 0, 5000], [5000, 77, 5000], 5000)
    assert a.cache.flags() == kvq.FLAG_BAD_BATCH
    a.check_appended(0)
    a.check_alone(1)
    a.check_alone(2)
    a.check_queries(0, range(5000))


def test_overlapping_ranges_that_fit(kvq_lib):
    """Short ones that share rows are appended both; a shared row of q goes by the first."""
    a = Appended([0, 40, 20, 60], [40, 9, 40], 60)
    assert a.cache.flags() == kvq.FLAG_BAD_BATCH
    a.check_appended(0)
    a.check_alone(1)
    a.check_appended(2)
    a.check_queries(0, range(40))
    a.check_queries(2, range(40, 60))


def test_a_row_of_a_bad_range_and_a_good_one(kvq_lib):
    """Rows of a range that is too long, which a later sequence holds rightly: its queries are
    rotated."""
    a = Appended([0, 100, 20, 40], [100, 9, 20], 100, max_new=50)
    assert a.cache.flags() == kvq.FLAG_BAD_BATCH
    a.check_alone(0)
    a.check_alone(1)
    a.check_appended(2)
    a.check_queries(2, range(20, 40))
    assert (a.out[:20] == 7.0).all() and (a.out[40:] == 7.0).all()


def test_overlaps_in_a_large_batch(kvq_lib):
    """Every second sequence of 300 holds the same 64 rows: as many as fit, and whole."""
    starts = [0, 64] * 150 + [0]
    a = Appended(starts, [64] * 300, 64, max_new=64)
    assert a.cache.flags() == kvq.FLAG_BAD_BATCH
    # s = 64 sequences at most: 64 / 32 + 128 blocks, two each
    for b in range(300):
        if b % 2 == 0 and b // 2 < 65: a.check_appended(b)
        else: a.check_alone(b)
    a.check_queries(0, range(64))


@pytest.mark.parametrize("max_new", [300, 16384, 131072])
def test_long_limits(kvq_lib, max_new):
    """64 sequences of up to 131072 tokens, chunks of up to max_new: a chunk beside a token."""
    cfg, cache, seen = filled("fp16", 2, 8, [700, 333], 704, seed=40)
    big = kvq.Block8Config(64, cfg.n_q_heads, 8, 131072)
    table = torch.full((64, big.max_blocks), -1, dtype=torch.int32)
    table[:2, :cfg.max_blocks] = cache.block_table.cpu()
    tensors = {n: getattr(cache, n) for n in ("k_codes", "v_codes", "scales")}
    for n in ("k_ring", "v_ring"):
        tensors[n] = torch.zeros(64, *getattr(cache, n).shape[1:], dtype=torch.float16,
                                 device="cuda")
        tensors[n][:2] = getattr(cache, n)
    wide = kvq.Block8Cache(big, tensors=tensors, block_table=table.cuda())
    q = torch.randn(301, cfg.n_q_heads, 128,
                    generator=torch.Generator().manual_seed(41)).half().cuda()
    starts = ints([0, 300] + [301] * 63)
    out = kvq.kvq_block8_attn(wide, q, ints([700, 333] + [0] * 62), starts=starts, max_new=max_new)
    check(cfg, out, q, [700, 333], [300, 1], seen)
    assert wide.flags() == 0
