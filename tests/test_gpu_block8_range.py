"""Attention over the block-8 cache at the ends of its inputs' range: open blocks (16-bit
tokens in the ring) whose elements lie far apart, factors of scores that leave fp32, very large
scores.  By both kernels: up to 32 query rows a kv-head, and more, of one row tile and of two.

Tolerance: a weight is rounded to fp16, its score to fp32, as in test_gpu_block8.py: 2^-11 +
2^-14 of sum p |v| and half a step of the result (at least half of fp16's smallest, 2^-25).
An open token's elements are good to 2^-40 of its largest, values to 2^-33 (2^-25 of fp16's
smallest beside 2^15 and 2^8), far below that for the random ones here; small weights to 2^-32
of the largest product of weight and value scale: L 2^-30 of the row's largest p |v| is added
where sizes are mixed."""

import numpy as np
import pytest
import torch

from oracle import block8
from paper_2607_16248_gb300 import kvq
from test_gpu_block8 import HALF_STEP, TYPES, np64
from test_gpu_block8_edges import ints, table_of

pytestmark = pytest.mark.gpu

# query heads a kv-head, new tokens, sequences (so many that a warp has several blocks)
KINDS = {"rows8": (4, 2, 1), "rows16": (4, 3, 1), "rows24": (8, 3, 1), "rows32": (8, 4, 1),
         "many8": (4, 2, 160), "many24": (8, 3, 160), "many32": (8, 4, 160),
         "chunk64": (32, 2, 1), "chunk80": (4, 20, 1), "chunk280": (4, 70, 1),
         "many64": (32, 2, 160)}


def rounded(x, dtype):
    """The finite elements in the 16-bit type."""
    return np.where(np.isfinite(x), block8.to_type(np.where(np.isfinite(x), x, 0.0), dtype), x)


class Case:
    """Keys and values (fp64 [L, 128]) of one kv-head put in by hand, for each of a number of
    sequences."""

    def __init__(self, dtype, gq, k, v, batch=1):
        self.dtype, L, blocks = dtype, len(k), len(k) // 32
        self.cfg = kvq.Block8Config(batch, gq, 1, (L + 31) // 32 * 32, TYPES[dtype])
        self.cache = kvq.Block8Cache(self.cfg, n_pages=max(1, blocks),
                                     block_table=table_of(self.cfg, [list(range(blocks))] * batch))
        self.seen = []
        for i, (x, pool, slots) in enumerate(((k, self.cache.k_codes, self.cache.k_ring),
                                              (v, self.cache.v_codes, self.cache.v_ring))):
            rows = rounded(x, dtype)
            out, codes = rows.copy(), np.zeros((max(1, blocks), 1, 32, 128))
            scales, ring = np.ones(max(1, blocks)), np.zeros((64, 128))
            for j in range(blocks):
                codes[j, 0], scales[j] = block8.quantize(rows[32 * j:32 * j + 32])
                out[32 * j:32 * j + 32] = codes[j, 0] * scales[j]
            for p in range(32 * blocks, L):
                ring[p % 64] = rows[p]
            pool.copy_(torch.tensor(codes).to(torch.float8_e4m3fn))
            self.cache.scales[:, 0, i] = torch.tensor(scales).float().cuda()
            slots[:, 0] = torch.tensor(ring).to(TYPES[dtype]).cuda()
            self.seen.append(out)
        self.L = L

    def attend(self, q, window=0, sinks=0, scale=0.0, mixed=False, unseen=()):
        """q fp64 [n, gq, 128]; rows of queries that see none of `unseen` are compared."""
        n, L = len(q), self.L
        q, batch = torch.tensor(q).to(TYPES[self.dtype]), self.cfg.batch
        out = kvq.kvq_block8_attn(self.cache, q.cuda().repeat(batch, 1, 1), ints([L] * batch),
                                  max_new=n, window=window, sinks=sinks, softmax_scale=scale)
        k, v = (x.copy() for x in self.seen)
        k[list(unseen)] = 0.0
        want, size = block8.attend(np64(q), k, v, float(np.float32(scale)) or None, window, sinks)
        rows = [t for t in range(n) if all(self.hidden(L - n + t, j, window, sinks)
                                           for j in unseen)]
        got = np64(out).reshape(batch, n, *out.shape[1:])[:, rows]
        want, size = want[rows], size[rows]
        tol = (2.0 ** -11 + 2.0 ** -14) * size + HALF_STEP[self.dtype] * np.abs(want)
        if self.dtype == "fp16":
            tol = tol + 2.0 ** -25
        if mixed:
            tol = tol + L * 2.0 ** -30 * size.max(-1, keepdims=True)
        err = np.abs(got - want)
        assert len(rows) and np.isfinite(got).all()
        assert (err <= tol).all(), float((err / tol).max())
        assert self.cache.flags() == 0
        return out

    @staticmethod
    def hidden(p, j, window, sinks):
        return j > p or bool(window and j <= p - window and j >= sinks)


def randn(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 2.0 ** 60, 2.0 ** 127])
@pytest.mark.parametrize("where", ["later", "behind"])
def test_unseen_keys_of_the_open_block(kvq_lib, kind, bad, where):
    """A key in the ring that is later than a query, or behind every query's window."""
    gq, n, batch = KINDS[kind]
    if where == "behind" and n > 4:
        n = 9
    L, window = (32 * 20 + 13, 0) if where == "later" else (32 * 20 + 29, 11)
    k, v, q = randn(1, L, 128), randn(2, L, 128), randn(3, n, gq, 128)
    at = [L - 1] if where == "later" else [32 * 20, 32 * 20 + 3]
    k[at] = bad
    Case("bf16", gq, k, v, batch).attend(q, window=window, unseen=at)


@pytest.mark.parametrize("kind", list(KINDS))
def test_keys_of_the_open_block_far_apart(kvq_lib, kind):
    """Seen keys of 2^-60 to 2^30 in one open block (the large ones in channels in which the
    queries hold nothing, so that no score is large)."""
    gq, n, batch = KINDS[kind]
    L = 32 * 20 + 27
    k, v, q = randn(4, L, 128), randn(5, L, 128), randn(6, n, gq, 128)
    k[-20:] *= 2.0 ** np.linspace(-60, 0, 20)[:, None]
    k[-25, 100:] *= 2.0 ** 30
    q[..., 100:] = 0.0
    Case("bf16", gq, k, v, batch).attend(q)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("dtype,big", [("bf16", 2.0 ** 60), ("bf16", 2.0 ** 120),
                                       ("fp16", 2.0 ** 13)])
def test_a_later_value_of_the_open_block_is_large(kvq_lib, kind, dtype, big):
    """Finite values that a query does not see, or that count for little, leave what it does
    see as it is."""
    gq, n, batch = KINDS[kind]
    small = 1.0 if dtype == "bf16" else 2.0 ** -10
    L = 32 * 20 + 17
    k, v, q = randn(7, L, 128), small * randn(8, L, 128), randn(9, n, gq, 128)
    v[-1] = big * randn(10, 128)
    case = Case(dtype, gq, k, v, batch)
    case.attend(q, unseen=[L - 1])
    case.attend(q, mixed=True)
    case.attend(q[-1:], window=1)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("L", [1, 17, 50, 32 * 20 + 1, 32 * 20 + 31])
@pytest.mark.parametrize("dtype,size", [("bf16", 2.0 ** -40), ("bf16", 2.0 ** 40),
                                        ("fp16", 2.0 ** -14), ("fp16", 2.0 ** -18)])
def test_values_of_one_size_beside_an_open_block(kvq_lib, kind, L, dtype, size):
    gq, n, batch = KINDS[kind]
    n = min(n, L)
    k, v, q = 2.0 * randn(11, L, 128), size * randn(12, L, 128), randn(13, n, gq, 128)
    Case(dtype, gq, k, v, batch).attend(q)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("L", [32 * 20, 32 * 20 + 20])
@pytest.mark.parametrize("dtype,size", [("bf16", 2.0 ** -40), ("bf16", 1.0), ("bf16", 2.0 ** 40),
                                        ("fp16", 2.0 ** -14), ("fp16", 1.0)])
def test_blocks_and_tokens_of_no_value(kvq_lib, kind, L, dtype, size):
    """A block whose values are all zero has scale 1; its weights count all the same."""
    gq, n, batch = KINDS[kind]
    k, v, q = 2.0 * randn(14, L, 128), size * randn(15, L, 128), randn(16, n, gq, 128)
    v[32:64] = 0.0
    v[-7:-3] = 0.0
    Case(dtype, gq, k, v, batch).attend(q)
    # a block of scale 1 that does hold something
    v[64:96] *= 448.0 / np.abs(v[64:96]).max() if size == 1.0 else 1.0
    v[64, 3] = 448.0 if size == 1.0 else v[64, 3]
    Case(dtype, gq, k, v, batch).attend(q, mixed=True)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("q_size,k_size", [(-85, -40), (-90, -55), (-100, -100), (-30, -110),
                                           (60, -120)])
@pytest.mark.parametrize("window", [0, 40])
def test_factors_below_fp32(kvq_lib, kind, q_size, k_size, window):
    """Scores of nothing: every visible token counts the same, masked ones not at all."""
    gq, n, batch = KINDS[kind]
    L = 32 * 20 + 21
    k, v, q = randn(17, L, 128), randn(18, L, 128), randn(19, n, gq, 128)
    Case("bf16", gq, k * 2.0 ** k_size, v, batch).attend(q * 2.0 ** q_size, window=window)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("scale", [1e-38, 1e-44])
def test_the_smallest_softmax_scales(kvq_lib, kind, dtype, scale):
    gq, n, batch = KINDS[kind]
    L = 32 * 20 + 21
    Case(dtype, gq, 0.01 * randn(20, L, 128), randn(21, L, 128), batch).attend(
        randn(22, n, gq, 128), scale=scale)


# Keys are 448 times a power of two in every channel, so that codes, scales and the sum
# over the channels are exact and tokens of one kind have the same score to the bit.
LARGE = {"fp16": ((8.0, 4096.0, 0.0), (128.0, 65504.0, 0.0), (8.0, 4096.0, 1000.0)),
         "bf16": ((8.0, 4096.0, 0.0), (2.0 ** 50, 2.0 ** 50, 0.0), (2.0 ** 40, 2.0 ** 55, 1e3))}


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("dtype,i", [(t, i) for t in LARGE for i in range(3)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("L", [32 * 5, 32 * 20 + 14, 32 * 70 + 9])
def test_large_scores(kvq_lib, kind, dtype, i, sign, L):
    """Scores of 2^28 and far beyond: equal ones share the weight, the largest takes it all."""
    gq, n, batch = KINDS[kind]
    step, q_size, scale = LARGE[dtype][i]
    q = np.full((n, gq, 128), sign * q_size)
    v = randn(23, L, 128)
    k = np.full((L, 128), 448.0 * step)
    Case(dtype, gq, k, v, batch).attend(q, scale=scale)                      # all equal
    Case(dtype, gq, -k, v, batch).attend(q, scale=scale, window=70, sinks=2)
    half = np.arange(L) % 64 < 32
    if sign > 0:
        # the blocks' scales differ, and so do the values'
        k[half] *= 0.5
        v[~half] *= 8.0
        Case(dtype, gq, k, v, batch).attend(q, scale=scale)
        # one token above all others, in a block and in the open one
        for at in (40, L - n - 1):
            k = np.full((L, 128), 224.0 * step)
            k[at] = 448.0 * step
            Case(dtype, gq, k, v, batch).attend(q, scale=scale)
    # some queries' scores are large, the others' are not
    q = q.copy()
    q[::2, ::2] = 2.0 ** -6 / step
    Case(dtype, gq, np.full((L, 128), 448.0 * step), v, batch).attend(q, scale=scale)


@pytest.mark.parametrize("kind", list(KINDS))
def test_scores_grow_along_the_text(kvq_lib, kind):
    """The reference moves from ordinary scores to very large ones, block by block."""
    gq, n, batch = KINDS[kind]
    L = 32 * 40 + 9
    k = 7.0 * 2.0 ** (np.arange(L) // 64)[:, None] * np.ones((L, 128))
    v, q = randn(24, L, 128), np.ones((n, gq, 128))
    v *= 2.0 ** (np.arange(L) // 32 % 3 * 4)[:, None]
    Case("bf16", gq, k, v, batch).attend(q, mixed=True)
    Case("bf16", gq, k[::-1].copy(), v, batch).attend(q, mixed=True)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("L", [32 * 20, 32 * 20 + 14])
def test_scores_far_below_zero(kvq_lib, kind, L):
    """Queries that see nothing of the open block or of a step, all scores about -300."""
    gq, n, batch = KINDS[kind]
    k, v, q = -27.0 + randn(25, L, 128), randn(26, L, 128), np.ones((n, gq, 128))
    for dtype in ("fp16", "bf16"):
        case = Case(dtype, gq, k, v, batch)
        case.attend(q)
        case.attend(q, window=33, sinks=3)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("L", [32 * 20, 32 * 20 + 14])
@pytest.mark.parametrize("ks,vs", [(90, 90), (-90, -90), (90, -90), (0, -90), (-90, 0)])
def test_scales_that_a_caller_chose(kvq_lib, kind, L, ks, vs):
    """Blocks that somebody else filled may have scales of 2^-90 to 2^90."""
    gq, n, batch = KINDS[kind]
    ks, vs, blocks = 2.0 ** ks, 2.0 ** vs, L // 32
    k, v, q = randn(27, L, 128), randn(28, L, 128), randn(29, n, gq, 128)
    k[32 * blocks:] *= 128.0 * ks       # (about what the blocks hold)
    v[32 * blocks:] *= 128.0 * vs
    case = Case("bf16", gq, k, v, batch)
    for i, to in ((0, ks), (1, vs)):
        by = to / np64(case.cache.scales[:, 0, i])
        case.cache.scales[:, 0, i] = to
        case.seen[i][:32 * blocks] *= by.repeat(32)[:, None]
    case.attend(2.0 * q / (128.0 * ks))


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("L", [32 * 20, 32 * 20 + 18, 32 * 20 + 31])
@pytest.mark.parametrize("dtype,size", [("fp16", 2.0 ** 12), ("fp16", 1.0), ("bf16", 1.0),
                                        ("bf16", 2.0 ** -30)])
def test_first_token_without_value(kvq_lib, kind, L, dtype, size):
    """A first token with all but 1e-5 of the weight and no value, in a block with values like
    the others': the result is the newest tokens, open ones among them, to the bits that
    weights keep down to 2^-21 of the largest."""
    gq, n, batch = KINDS[kind]
    u = np.sign(randn(30, 128))
    k, v = randn(31, L, 128), size * randn(32, L, 128)
    k -= (k @ u)[:, None] * u / 128
    k[0], v[0] = 13.0 * np.sqrt(128) / 128 * u, 0.0
    q = u + 0.3 * randn(33, n, gq, 128)
    case = Case(dtype, gq, k, v, batch)
    case.attend(q, window=17, sinks=1)
    case.attend(q, window=300, sinks=1)
