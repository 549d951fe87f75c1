"""kvq_block8_append and kvq_block8_attn against the 64-bit oracle.

Tolerances.  Codes, scales and rings are exact.  Rotated queries: two products and a sum
in fp32 (3 * 2^-24 of the magnitudes) and one rounding to the type (half a step).
Attention: a weight is rounded to fp16 (2^-11 relative, 2^-25 of the row's largest where it
is below fp16's normal range; weights carry a factor that keeps 2^-21 of it normal), a
score's fp32 error of up to 128 additions is 2^-17 relative to the largest products, and
the exponential, the sums and the quotient stay within 2^-16; with the result's own
rounding that is 2^-11 + 2^-14 of sum p |v| and half a step of the result."""

import numpy as np
import pytest
import torch

from oracle import block8
from paper_2607_16248_gb300 import kvq

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}


def np64(t):
    return t.detach().double().cpu().numpy()


class World:
    """A cache, its oracle and the bookkeeping of a caller: lengths and pages."""

    def __init__(self, batch, hq, hkv, max_len, dtype, seed=0, boost=10.0):
        self.dtype, self.rng = dtype, torch.Generator().manual_seed(seed)
        self.cfg = kvq.Block8Config(batch, hq, hkv, max_len, TYPES[dtype])
        pages = batch * self.cfg.max_blocks
        self.cache = kvq.Block8Cache(self.cfg, n_pages=pages + 3)
        self.free = (torch.randperm(pages + 3, generator=self.rng)).tolist()
        self.k = [[block8.Sequence() for _ in range(hkv)] for _ in range(batch)]
        self.v = [[block8.Sequence() for _ in range(hkv)] for _ in range(batch)]
        self.lengths = [0] * batch
        self.mapped = [set() for _ in range(batch)]
        self.boost = torch.ones(hkv, 128)
        self.boost[:, 5], self.boost[:, 77] = boost, boost

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.rng).to(TYPES[self.dtype])

    def append(self, counts, rot=128, paired=False, uniform=False, spare=0, positions=None,
               n_positions=4096, graph=False):
        cfg, hq, hkv = self.cfg, self.cfg.n_q_heads, self.cfg.n_kv_heads
        starts = np.concatenate([[0], np.cumsum(counts)])
        n = int(starts[-1]) + spare
        qkv = self.randn(n, hq + 2 * hkv, 128)
        qkv[:, hq:hq + hkv] = (qkv[:, hq:hq + hkv].float() * self.boost).to(qkv.dtype)
        for b, m in enumerate(counts):
            new = [j for j in kvq.block8_written(self.lengths[b], m) if j not in self.mapped[b]]
            if new:
                self.cache.map_blocks(b, new, [self.free.pop() for _ in new])
                self.mapped[b].update(new)
            self.lengths[b] += m
        half = rot // 2
        angle = np.arange(n_positions)[:, None] * 10000.0 ** (-np.arange(half) / max(1, half))
        cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
        dev = qkv.cuda()
        q, k, v = dev.split([hq, hkv, hkv], 1)
        lengths = torch.tensor(self.lengths, dtype=torch.int32, device="cuda")
        st = None if uniform else torch.tensor(starts, dtype=torch.int32, device="cuda")
        q_out = torch.full((n, hq, 128), 7.0, dtype=qkv.dtype, device="cuda")
        kvq.kvq_block8_append(
            self.cache, k, v, lengths, starts=st, q=q, q_out=q_out,
            cos=torch.from_numpy(cos).cuda() if rot else None,
            sin=torch.from_numpy(sin).cuda() if rot else None, paired=paired,
            positions=None if positions is None else
            torch.tensor(positions, dtype=torch.int32, device="cuda"))
        x = np64(qkv)
        pos = np.zeros(n, dtype=int)
        for b, m in enumerate(counts):
            pos[starts[b]:starts[b + 1]] = np.arange(self.lengths[b] - m, self.lengths[b])
        at = np.clip(pos if positions is None else np.array(positions), 0, n_positions - 1)
        y = block8.rotate(x[:, :hq + hkv], cos[at], sin[at], paired)
        for b, m in enumerate(counts):
            rows = slice(int(starts[b]), int(starts[b + 1]))
            for h in range(hkv):
                self.k[b][h].append(block8.to_type(y[rows, hq + h], self.dtype), self.lengths[b])
                self.v[b][h].append(x[rows, hq + hkv + h], self.lengths[b])
        real = int(starts[-1])
        if rot:
            got = np64(q_out)[:real]
            err = np.abs(got - y[:real, :hq])
            size = block8.rotate(np.abs(x[:real, :hq]), np.abs(cos[at[:real]]),
                                 -np.abs(sin[at[:real]]), paired)
            size = np.maximum(size, np.abs(x[:real, :hq]) + np.abs(y[:real, :hq]))
            assert (err <= HALF_STEP[self.dtype] * np.abs(y[:real, :hq]) + 4 * 2.0 ** -24 * size
                    + 2.0 ** -25).all()
        else:
            assert torch.equal(q_out[:real], q[:real])
        assert (q_out[real:] == 7.0).all()
        self.starts, self.counts, self.q = st, counts, q_out
        return lengths

    def check_state(self):
        table = self.cache.block_table.cpu()
        scales = np64(self.cache.scales)
        for codes, ring, seqs, i in ((self.cache.k_codes, self.cache.k_ring, self.k, 0),
                                     (self.cache.v_codes, self.cache.v_ring, self.v, 1)):
            codes, ring = np64(codes.float()), np64(ring)
            for b in range(self.cfg.batch):
                L = self.lengths[b]
                for h in range(self.cfg.n_kv_heads):
                    rows = seqs[b][h].rows
                    for j in range(L // 32):
                        c, s = block8.quantize(rows[32 * j:32 * j + 32])
                        page = int(table[b, j])
                        assert scales[page, h, i] == s, (b, h, j)
                        assert np.array_equal(codes[page, h], c), (b, h, j)
                    for p in range(max(0, (L // 32 - 1) * 32), L):
                        assert np.array_equal(ring[b, h, p % 64], rows[p]), (b, h, p)

    def check_attention(self, lengths, max_new=None, window=0, sinks=0, scale=0.0, q=None,
                        **call):
        cfg, gq = self.cfg, self.cfg.n_q_heads // self.cfg.n_kv_heads
        q = self.q if q is None else q
        out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
        kvq.kvq_block8_attn(self.cache, q, lengths, starts=self.starts, max_new=max_new,
                            window=window, sinks=sinks, softmax_scale=scale, out=out, **call)
        got, x = np64(out), np64(q)
        at = 0
        for b, n in enumerate(self.counts):
            for h in range(cfg.n_kv_heads):
                heads = slice(h * gq, (h + 1) * gq)
                want, size = block8.attend(x[at:at + n, heads], self.k[b][h].seen(),
                                           self.v[b][h].seen(), scale or None, window, sinks)
                err = np.abs(got[at:at + n, heads] - want)
                tol = (2.0 ** -11 + 2.0 ** -14) * size + HALF_STEP[self.dtype] * np.abs(want) \
                    + 2.0 ** -25
                assert (err <= tol).all(), (b, h, float((err / tol).max()))
            at += n
        assert (out[at:] == 7.0).all()
        return out


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("rot,paired", [(128, False), (128, True), (64, False), (96, True),
                                        (40, False), (8, True), (0, False)])
def test_append_rotations(kvq_lib, dtype, rot, paired):
    w = World(2, 6, 2, 256, dtype, seed=rot)
    w.append([40, 3], rot=rot, paired=paired)
    w.append([1, 31], rot=rot, paired=paired, spare=2)
    w.check_state()
    assert w.cache.flags() == 0


@pytest.mark.parametrize("steps", [[[1]], [[31], [1], [1]], [[32], [32]], [[20], [20], [70]],
                                   [[17], [100], [3], [64]], [[33], [31], [95]], [[129]],
                                   [[5], [59], [1]], [[0], [4]]])
def test_append_lengths(kvq_lib, steps):
    w = World(1, 2, 2, 320, "fp16", seed=len(steps))
    for counts in steps:
        if sum(counts):
            w.append(counts)
            w.check_state()
    assert w.cache.flags() == 0


def test_append_ragged_batch(kvq_lib):
    w = World(150, 4, 1, 96, "bf16", seed=4)
    counts = [(7 * b) % 5 for b in range(150)]
    for step in range(4):
        counts[3] = 40 if step == 1 else 1
        w.append(counts, rot=64)
    w.check_state()
    lengths = w.append([1] * 150, uniform=True)
    w.check_state()
    w.check_attention(lengths)
    assert w.cache.flags() == 0


def test_positions_and_dropped_drafts(kvq_lib):
    w = World(2, 2, 1, 256, "fp16", seed=5)
    w.append([50, 30], positions=[3 * i % 4096 for i in range(80)])
    lengths = w.append([9, 20])
    w.check_state()
    # all but two of the new tokens go: across a block's end and within one
    w.lengths = [52, 32]
    for seqs in (w.k, w.v):
        for b in (0, 1):
            seqs[b][0].rows = seqs[b][0].rows[:w.lengths[b]]
    lengths = w.append([3, 1])
    w.check_state()
    w.check_attention(lengths)
    lengths = w.append([30, 31])
    w.check_state()
    w.check_attention(lengths)
    assert w.cache.flags() == 0


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 2), (10, 2), (8, 1), (24, 2), (32, 1)])
def test_attention_heads(kvq_lib, dtype, hq, hkv):
    w = World(3, hq, hkv, 512, dtype, seed=hq)
    w.append([300, 1, 64])
    w.check_attention(w.append([1, 1, 1]), max_new=1)
    w.check_attention(w.append([3, 1, 4], spare=3), max_new=4)
    w.check_attention(w.append([40, 0, 70]), max_new=70)
    assert w.cache.flags() == 0


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (33, 4), (100, 40), (257, 128),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
def test_attention_windows(kvq_lib, window, sinks):
    w = World(2, 8, 2, 1024, "fp16", seed=window % 97)
    w.append([700, 90])
    w.check_attention(w.append([1, 1]), max_new=1, window=window, sinks=sinks)
    w.check_attention(w.append([2, 5]), max_new=5, window=window, sinks=sinks)
    w.check_attention(w.append([200, 1]), max_new=200, window=window, sinks=sinks)
    assert w.cache.flags() == 0


@pytest.mark.parametrize("L", [1, 2, 31, 32, 33, 63, 64, 65, 128, 129, 255, 256, 300])
def test_attention_prompts(kvq_lib, L):
    w = World(2, 6, 2, 320, "fp16", seed=L)
    w.check_attention(w.append([L, max(1, L // 2)]))


def test_attention_long(kvq_lib):
    w = World(2, 4, 1, 8224, "bf16", seed=9)
    w.append([8000, 4001], n_positions=8224)
    w.check_attention(w.append([1, 1], n_positions=8224), max_new=1)
    w.check_attention(w.append([150, 7], n_positions=8224), max_new=150)


def test_append_large_batch(kvq_lib):
    """So many blocks that a CTA takes several heads, some of them begun before."""
    rng = np.random.default_rng(21)
    w = World(1500, 4, 4, 128, "fp16", seed=21)
    for _ in range(2):
        counts = np.where(rng.random(1500) < 0.1, 0, rng.integers(1, 41, 1500)).tolist()
        w.append(counts, rot=32)
    w.check_state()
    assert w.cache.flags() == 0
