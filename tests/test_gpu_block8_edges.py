"""The block-8 cache where it can go wrong: strides, streams, graphs, bad pages and batches,
masked places, scales and queries of any size, far pages.  Tolerances as in
test_gpu_block8.py; where a case adds a term it is derived there."""

import numpy as np
import pytest
import torch

from oracle import block8
from paper_2607_16248_gb300 import kvq
from test_gpu_block8 import HALF_STEP, TYPES, World, np64

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def table_of(cfg, pages):
    """int32 [batch, max_blocks] from lists of pages, -1 behind them."""
    t = torch.full((cfg.batch, cfg.max_blocks), -1, dtype=torch.int32)
    for b, p in enumerate(pages):
        t[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    return t.cuda()


def filled(dtype, batch, hkv, lengths, max_len, gq=4, seed=0, k_size=1.0, v_size=None):
    """A cache with random contents put in by hand, and its keys and values as attention
    sees them: fp64 [batch][hkv][L, 128].  v_size: a factor per block."""
    g = torch.Generator().manual_seed(seed)
    cfg = kvq.Block8Config(batch, gq * hkv, hkv, max_len, TYPES[dtype])
    pages = [[b * cfg.max_blocks + j for j in range(L // 32)] for b, L in enumerate(lengths)]
    cache = kvq.Block8Cache(cfg, n_pages=batch * cfg.max_blocks, block_table=table_of(cfg, pages))
    seen = [[[None, None] for _ in range(hkv)] for _ in range(batch)]
    for b, L in enumerate(lengths):
        for h in range(hkv):
            for i, (codes, ring) in enumerate(((cache.k_codes, cache.k_ring),
                                               (cache.v_codes, cache.v_ring))):
                rows = torch.randn(L, 128, generator=g).double() * (k_size if i == 0 else 1.0)
                if i and v_size is not None:
                    for j in range((L + 31) // 32):
                        rows[32 * j:32 * j + 32] *= v_size[j % len(v_size)]
                rows = block8.to_type(rows.numpy(), dtype)
                out = rows.copy()
                for j in range(L // 32):
                    c, s = block8.quantize(rows[32 * j:32 * j + 32])
                    out[32 * j:32 * j + 32] = c * s
                    codes[pages[b][j], h] = torch.tensor(c).to(torch.float8_e4m3fn).cuda()
                    cache.scales[pages[b][j], h, i] = s
                for p in range(L // 32 * 32, L):
                    ring[b, h, p % 64] = torch.tensor(rows[p]).to(TYPES[dtype]).cuda()
                seen[b][h][i] = out
    return cfg, cache, seen


def check(cfg, out, q, lengths, counts, seen, window=0, sinks=0, scale=None, extra=0.0):
    gq, at = cfg.n_q_heads // cfg.n_kv_heads, 0
    dtype = "fp16" if cfg.dtype == torch.float16 else "bf16"
    got, x = np64(out), np64(q)
    for b, n in enumerate(counts):
        for h in range(cfg.n_kv_heads):
            hs = slice(h * gq, (h + 1) * gq)
            want, size = block8.attend(x[at:at + n, hs], *seen[b][h], scale, window, sinks)
            err = np.abs(got[at:at + n, hs] - want)
            tol = (2.0 ** -11 + 2.0 ** -14) * size + HALF_STEP[dtype] * np.abs(want) + 2.0 ** -25 \
                + extra * size.max(-1, keepdims=True)
            assert (err <= tol).all(), (b, h, float((err / tol).max()))
        at += n


def test_strides_and_in_place(kvq_lib):
    """q, k, v and the outputs as views of wider arrays, q rotated in place."""
    w = World(2, 4, 2, 128, "fp16", seed=1)
    cfg, n = w.cfg, 70
    wide = w.randn(n, 12, 256).cuda()
    q, k, v = wide[:, :4, :128], wide[:, 4:8:2, 128:], wide[:, 5:9:2, 128:]
    angle = torch.arange(64)[:, None] * torch.rand(64, generator=w.rng)
    cos, sin = angle.cos().cuda(), angle.sin().cuda()
    lengths = ints([35, 35])
    w.cache.map_blocks(0, [0], [2])
    w.cache.map_blocks(1, [0], [0])
    q0, rest = q.clone(), wide.clone()
    want = kvq.kvq_block8_append(w.cache, k, v, lengths, q=q, cos=cos, sin=sin)
    state = [t.clone() for t in (w.cache.k_codes.view(torch.uint8), w.cache.v_codes.view(
        torch.uint8), w.cache.scales, w.cache.k_ring, w.cache.v_ring)]
    assert torch.equal(wide, rest) and want.is_contiguous()
    same = kvq.kvq_block8_append(w.cache, k.contiguous(), v.contiguous(), lengths, q=q, q_out=q,
                                 cos=cos, sin=sin)
    assert same is q and torch.equal(q, want) and not torch.equal(q, q0)
    rest[:, :4, :128] = q
    assert torch.equal(wide, rest)
    for a, b in zip(state, (w.cache.k_codes.view(torch.uint8), w.cache.v_codes.view(torch.uint8),
                            w.cache.scales, w.cache.k_ring, w.cache.v_ring)):
        assert torch.equal(a, b)
    out = torch.full((n, 9, 256), 3.0, dtype=torch.float16, device="cuda")
    kvq.kvq_block8_attn(w.cache, q, lengths, out=out[:, 1:9:2, 128:])
    assert torch.equal(out[:, 1:9:2, 128:], kvq.kvq_block8_attn(w.cache, want, lengths))
    out[:, 1:9:2, 128:] = 3.0
    assert (out == 3.0).all() and w.cache.flags() == 0
    assert cfg.n_q_heads == 4


def test_append_without_queries_and_shared_tables(kvq_lib):
    """Two layers' caches on one block table; a call without q."""
    cfg = kvq.Block8Config(1, 2, 1, 64)
    table = ints([[1, 0]])
    g = torch.Generator().manual_seed(3)
    k, v = torch.randn(2, 64, 1, 128, generator=g).half().cuda()
    caches = [kvq.Block8Cache(cfg, n_pages=2, block_table=table) for _ in range(2)]
    for cache in caches:
        assert kvq.kvq_block8_append(cache, k, v, ints([64])) is None
    assert torch.equal(caches[0].k_codes.view(torch.uint8), caches[1].k_codes.view(torch.uint8))
    for j in (0, 1):
        c, s = block8.quantize(np64(k[32 * j:32 * j + 32, 0]))
        assert np.array_equal(np64(caches[0].k_codes[1 - j, 0].float()), c)
        assert float(caches[0].scales[1 - j, 0, 0]) == s


def test_other_stream_and_graph_with_other_lengths(kvq_lib):
    w = World(2, 8, 2, 512, "fp16", seed=2)
    w.append([200, 90])
    lengths = w.append([1, 1])
    ws = kvq.block8_workspace(w.cfg, 1)
    q = w.q.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = kvq.kvq_block8_attn(w.cache, q, lengths, workspace=ws)
    torch.cuda.synchronize()
    got = kvq.kvq_block8_attn(w.cache, q, lengths, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(got, out)
    # a captured step of both operators, replayed as the text grows; two graphs, one workspace
    k, v = torch.zeros(2, 2, 2, 128, dtype=torch.float16, device="cuda")
    qin, outs = torch.zeros_like(q), [torch.zeros_like(q) for _ in range(2)]
    graphs = []
    w.cache.map_blocks(0, range(16), range(16))
    w.cache.map_blocks(1, range(16), range(16, 32))
    fresh = kvq.Block8Cache(w.cfg, tensors={n: getattr(w.cache, n).clone() for n in (
        "k_codes", "v_codes", "scales", "k_ring", "v_ring")}, block_table=w.cache.block_table)
    base = lengths.clone()
    for o in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lengths.add_(1)
            kvq.kvq_block8_append(w.cache, k, v, lengths)
            kvq.kvq_block8_attn(w.cache, qin, lengths, out=o, workspace=ws)
        graphs.append(graph)
    lengths.copy_(base)
    for t in ("k_codes", "v_codes", "scales", "k_ring", "v_ring"):
        getattr(w.cache, t).view(torch.uint8).copy_(getattr(fresh, t).view(torch.uint8))
    other = kvq.block8_workspace(w.cfg, 1)
    for step in range(40):
        k.copy_(w.randn(2, 2, 128))
        v.copy_(w.randn(2, 2, 128))
        qin.copy_(w.randn(*qin.shape))
        graphs[step % 2].replay()
        base.add_(1)
        kvq.kvq_block8_append(fresh, k, v, base)
        want = kvq.kvq_block8_attn(fresh, qin, base, workspace=other)
        assert torch.equal(outs[step % 2], want), step
    assert lengths.tolist() == base.tolist() and w.cache.flags() == 0


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("counts", [[1, 1, 1], [5, 8, 3], [60, 2, 100]])
def test_values_of_any_scale(kvq_lib, dtype, counts):
    """Blocks of values 2^-12 to 2^12 apart (fp16: 2^-6 to 2^6).  A weight times its scale is
    good to 2^-32 of the row's largest such product, and a block's values are at most 448
    scales: n_tokens * 448 / 448 * 2^-32 of the largest weighted magnitude is added."""
    e = 12 if dtype == "bf16" else 6
    sizes = [2.0 ** x for x in (0, e, -e, 3, -3)]
    lengths = [290, 161, 331]
    cfg, cache, seen = filled(dtype, 3, 2, lengths, 352, seed=5, v_size=sizes)
    g = torch.Generator().manual_seed(6)
    q = torch.randn(sum(counts), cfg.n_q_heads, 128, generator=g).to(cfg.dtype).cuda()
    starts = ints(np.concatenate([[0], np.cumsum(counts)]))
    out = kvq.kvq_block8_attn(cache, q, ints(lengths), starts=starts, max_new=max(counts))
    check(cfg, out, q, lengths, counts, seen, extra=331 * 2.0 ** -30)
    assert cache.flags() == 0


@pytest.mark.parametrize("counts", [[1, 1], [9, 40]])
def test_bf16_queries_and_keys_of_any_size(kvq_lib, counts):
    """Queries of 2^40, keys of 2^-45: each within bf16, far outside fp16."""
    lengths = [100, 75]
    cfg, cache, seen = filled("bf16", 2, 1, lengths, 128, seed=7, k_size=2.0 ** -45)
    g = torch.Generator().manual_seed(8)
    q = (torch.randn(sum(counts), cfg.n_q_heads, 128, generator=g) * 2.0 ** 40).bfloat16().cuda()
    starts = ints(np.concatenate([[0], np.cumsum(counts)]))
    scale = 2.0 ** 5 / np.sqrt(128)
    out = kvq.kvq_block8_attn(cache, q, ints(lengths), starts=starts, max_new=max(counts),
                              softmax_scale=scale)
    check(cfg, out, q, lengths, counts, seen, scale=float(np.float32(scale)))


@pytest.mark.parametrize("max_new", [4, 64])
def test_blocks_behind_the_window_need_no_page(kvq_lib, max_new):
    lengths, counts = [500, 330], [4, 2]
    cfg, cache, seen = filled("fp16", 2, 2, lengths, 512, seed=9)
    q = torch.randn(6, cfg.n_q_heads, 128, generator=torch.Generator().manual_seed(1)).half().cuda()
    args = dict(starts=ints([0, 4, 6]), max_new=max_new, window=70, sinks=33)
    want = kvq.kvq_block8_attn(cache, q, ints(lengths), **args)
    check(cfg, want, q, lengths, counts, seen, 70, 33)
    for b, (L, n) in enumerate(zip(lengths, counts)):
        gone = list(range(2, (L - n - 70 + 1) // 32))
        assert len(gone) > 3
        cache.map_blocks(b, gone, [-1] * len(gone))
    assert torch.equal(kvq.kvq_block8_attn(cache, q, ints(lengths), **args), want)
    assert cache.flags() == 0


@pytest.mark.parametrize("counts", [[1, 1], [70, 40]])
def test_keys_that_nobody_sees_may_be_anything(kvq_lib, counts):
    """NaN in keys behind the window, NaN in all ring slots behind the sequence's end."""
    lengths = [300, 290]
    cfg, cache, seen = filled("fp16", 2, 1, lengths, 320, seed=11)
    q = torch.randn(sum(counts), cfg.n_q_heads, 128,
                    generator=torch.Generator().manual_seed(2)).half().cuda()
    starts = ints(np.concatenate([[0], np.cumsum(counts)]))
    args = dict(starts=starts, max_new=max(counts), window=40)
    want = kvq.kvq_block8_attn(cache, q, ints(lengths), **args)
    check(cfg, want, q, lengths, counts, seen, 40)
    for b, (L, n) in enumerate(zip(lengths, counts)):
        last = L - n - 40            # the newest token behind every window
        for t in range(last // 32 * 32, last + 1):
            cache.k_codes.view(torch.uint8)[b * cfg.max_blocks + t // 32, 0, t % 32] = 0x7f
        used = [p % 64 for p in range(L // 32 * 32, L)]
        for ring in (cache.k_ring, cache.v_ring):
            free = [s for s in range(64) if s not in used]
            ring[b, 0, free] = float("nan")
    assert torch.equal(kvq.kvq_block8_attn(cache, q, ints(lengths), **args), want)


@pytest.mark.parametrize("max_new", [1, 40])
def test_bad_pages_are_skipped_and_flagged(kvq_lib, max_new):
    cfg, cache, seen = filled("fp16", 1, 1, [200], 256, seed=12)
    q = torch.randn(max_new, cfg.n_q_heads, 128,
                    generator=torch.Generator().manual_seed(3)).half().cuda()
    for page in (-1, 8, 2 ** 31 - 1, -2 ** 31):
        cache.map_blocks(0, [2], [page])
        cache.clear_flags()
        out = kvq.kvq_block8_attn(cache, q, ints([200]))
        assert cache.flags() == kvq.FLAG_BAD_PAGE
        short = [x.copy() for x in seen[0][0]]
        short = [np.concatenate([x[:64], x[96:]]) for x in short]     # as if it were not there
        check(cfg, out, q, [168], [max_new], [[short]])
    k = torch.randn(56, 1, 128).half().cuda()
    before = cache.k_codes.view(torch.uint8).clone()
    cache.map_blocks(0, [6, 7], [-5, 8])
    cache.clear_flags()
    kvq.kvq_block8_append(cache, k, k, ints([256]))
    assert cache.flags() == kvq.FLAG_BAD_PAGE
    assert torch.equal(cache.k_codes.view(torch.uint8), before)


@pytest.mark.parametrize("starts,lengths,flag", [
    ([0, 3, 2, 5], [10, 10, 10], kvq.FLAG_BAD_BATCH),
    ([-1, 1, 3, 5], [10, 10, 10], kvq.FLAG_BAD_BATCH),
    ([0, 2, 3, 6], [10, 10, 10], kvq.FLAG_BAD_BATCH),
    ([0, 2, 3, 5], [10, 97, 10], kvq.FLAG_OVERFLOW),
    ([0, 2, 3, 5], [10, 10, -3], kvq.FLAG_BAD_BATCH),
    ([0, 2, 3, 5], [10, 0, 10], kvq.FLAG_BAD_BATCH)])
def test_bad_batches_are_left_alone(kvq_lib, starts, lengths, flag):
    """A sequence whose sizes do not hold: its rows and its cache stay, the others' do not."""
    cfg = kvq.Block8Config(3, 2, 1, 96)
    cache = kvq.Block8Cache(cfg, n_pages=9)
    cache.block_table.copy_(torch.arange(9, dtype=torch.int32).view(3, 3))
    g = torch.Generator().manual_seed(4)
    k, v, q = (torch.randn(5, h, 128, generator=g).half().cuda() for h in (1, 1, 2))
    marks = [t.view(torch.uint8).clone() for t in (cache.k_codes, cache.v_codes)]
    rows = torch.full((5, 2, 128), 7.0, dtype=torch.float16, device="cuda")
    kvq.kvq_block8_append(cache, k, v, ints(lengths), starts=ints(starts), q=q, q_out=rows)
    assert cache.flags() == flag
    out = torch.full_like(rows, 7.0)
    kvq.kvq_block8_attn(cache, q, ints(lengths), starts=ints(starts), out=out)
    ok = [b for b in range(3) if 0 <= starts[b] <= starts[b + 1] <= 5 and 0 <= lengths[b] <= 96]
    touched = set()
    for b in ok:
        mine = range(starts[b], starts[b + 1])
        touched.update(mine)
        if lengths[b] < len(mine):      # ahead of the first token: zero
            assert (out[list(mine)] == 0).all() and (rows[list(mine)] == 7.0).all()
        else:
            assert torch.equal(rows[list(mine)], q[list(mine)])
            assert torch.equal(cache.v_ring[b, 0, [p % 64 for p in range(
                lengths[b] - len(mine), lengths[b])]], v[list(mine), 0])
    left = [r for r in range(5) if r not in touched]
    assert (rows[left] == 7.0).all() and (out[left] == 7.0).all()
    for b in set(range(3)) - set(ok):
        assert (cache.v_ring[b] == 0).all()
    assert all(torch.equal(a, t.view(torch.uint8)) for a, t in zip(
        marks, (cache.k_codes, cache.v_codes)))


def test_queries_ahead_of_the_first_token(kvq_lib):
    cfg, cache, seen = filled("fp16", 2, 1, [3, 0], 64, seed=13)
    q = torch.randn(80, cfg.n_q_heads, 128,
                    generator=torch.Generator().manual_seed(5)).half().cuda()
    for starts, max_new in (([0, 5, 10], 8), ([0, 40, 80], 40)):
        n = [starts[1], starts[2] - starts[1]]
        out = kvq.kvq_block8_attn(cache, q[:starts[2]], ints([3, 0]), starts=ints(starts),
                                  max_new=max_new)
        assert (out[:n[0] - 3] == 0).all() and (out[n[0]:] == 0).all()
        check(cfg, out[n[0] - 3:n[0]], q[n[0] - 3:n[0]], [3], [3], seen)
    assert cache.flags() == 0


def test_pages_beyond_two_gigabytes(kvq_lib):
    """The last pages of pools of 4.3 GB each."""
    cfg = kvq.Block8Config(1, 8, 2, 256)
    pages = (1 << 19) + 5
    cache = kvq.Block8Cache(cfg, n_pages=pages)
    g = torch.Generator().manual_seed(14)
    rows = torch.randn(2, 250, 2, 128, generator=g).half()
    cache.map_blocks(0, range(8), [pages - 1 - j * (1 << 16) for j in range(8)])
    k, v = rows.cuda()
    for n in (1, 40):
        kvq.kvq_block8_append(cache, k, v, ints([250]))
        q = torch.randn(n, 8, 128, generator=g).half().cuda()
        out = kvq.kvq_block8_attn(cache, q, ints([250]))
        seen = []
        for h in range(2):
            pair = []
            for i in (0, 1):
                s = block8.Sequence()
                s.append(np64(rows[i][:, h]), 250)
                pair.append(s.seen())
            seen.append(pair)
        check(cfg, out, q, [250], [n], [seen])
    assert cache.flags() == 0


def test_many_sequences_of_one_token(kvq_lib):
    """2000 sequences, one token each (more items than threads): its value comes back."""
    cfg = kvq.Block8Config(2000, 2, 1, 32, torch.bfloat16)
    cache = kvq.Block8Cache(cfg, n_pages=1)
    g = torch.Generator().manual_seed(15)
    k, v, q = (torch.randn(2000, h, 128, generator=g).bfloat16().cuda() for h in (1, 1, 2))
    lengths = ints([1] * 2000)
    kvq.kvq_block8_append(cache, k, v, lengths)
    out = kvq.kvq_block8_attn(cache, q, lengths)
    # one weight, 2^7 in fp16 exactly, over its own sum
    assert torch.equal(out, v.expand(2000, 2, 128)) and cache.flags() == 0


def test_more_new_tokens_than_said(kvq_lib):
    cfg = kvq.Block8Config(2, 2, 1, 96)
    cache = kvq.Block8Cache(cfg, n_pages=1)
    k, v, q = (torch.randn(6, h, 128).half().cuda() for h in (1, 1, 2))
    args = dict(starts=ints([0, 2, 6]), max_new=3)
    kvq.kvq_block8_append(cache, k, v, ints([2, 4]), **args)
    assert cache.flags() == kvq.FLAG_BAD_BATCH and (cache.k_ring[1] == 0).all()
    assert torch.equal(cache.v_ring[0, 0, :2], v[:2, 0])
    cache.clear_flags()
    out = torch.full((6, 2, 128), 7.0, dtype=torch.float16, device="cuda")
    kvq.kvq_block8_attn(cache, q, ints([2, 4]), out=out, **args)
    assert cache.flags() == kvq.FLAG_BAD_BATCH
    assert (out[2:] == 7.0).all() and not (out[:2] == 7.0).any()


@pytest.mark.parametrize("counts", [[1], [20], [90]])
def test_the_largest_cache(kvq_lib, counts):
    """2^31 - 32 tokens of which a window is seen."""
    top, n = 2 ** 31 - 32, counts[0]
    cfg = kvq.Block8Config(1, 4, 1, top)
    cache = kvq.Block8Cache(cfg, n_pages=16)
    for L in (top, top - 5):
        first = (L - 256) // 32
        blocks = list(range(first, L // 32))
        cache.map_blocks(0, blocks, range(len(blocks)))
        g = torch.Generator().manual_seed(16)
        start = 32 * first
        rows = torch.randn(2, L - start, 1, 128, generator=g).half()
        k, v = rows.cuda()
        kvq.kvq_block8_append(cache, k, v, ints([L]), starts=ints([0, L - start]))
        q = torch.randn(n, 4, 128, generator=g).half().cuda()
        out = kvq.kvq_block8_attn(cache, q, ints([L]), max_new=n, window=100)
        seen = []
        for i in (0, 1):
            s = block8.Sequence()
            s.append(np64(rows[i][:, 0]), L - start)
            seen.append(s.seen())
        check(cfg, out, q, [L - start], counts, [[seen]], 100)
        assert cache.flags() == 0


def test_short_and_long_sequences_of_every_size(kvq_lib):
    """One call with sequences of each row group count and longer ones; twice the same bits."""
    counts = [1, 2, 3, 5, 6, 8, 9, 33, 70, 4, 7, 128]
    lengths = [64 + 37 * i for i in range(len(counts))]
    lengths[-1] = 500
    cfg, cache, seen = filled("fp16", len(counts), 1, lengths, 512, seed=17)
    q = torch.randn(sum(counts), cfg.n_q_heads, 128,
                    generator=torch.Generator().manual_seed(18)).half().cuda()
    starts = ints(np.concatenate([[0], np.cumsum(counts)]))
    outs = [kvq.kvq_block8_attn(cache, q, ints(lengths), starts=starts, max_new=128)
            for _ in range(3)]
    check(cfg, outs[0], q, lengths, counts, seen)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    short = [b for b, n in enumerate(counts) if n <= 8]
    few = [counts[b] if b in short else 0 for b in range(len(counts))]
    rows = torch.cat([q[sum(counts[:b]):sum(counts[:b + 1])] for b in short])
    starts = ints(np.concatenate([[0], np.cumsum(few)]))
    out = kvq.kvq_block8_attn(cache, rows, ints(lengths), starts=starts, max_new=8)
    check(cfg, out, rows, lengths, few, seen)
    assert cache.flags() == 0


@pytest.mark.parametrize("batch,hkv,L,n", [(1, 1, 2100, 1), (1, 2, 1030, 3), (1, 8, 333, 1),
                                           (3, 2, 512, 2), (4, 1, 95, 1), (2, 3, 700, 8)])
def test_items_of_one_size(kvq_lib, batch, hkv, L, n):
    """Sequences of equal length, each item divided among as many CTAs."""
    cfg, cache, seen = filled("fp16", batch, hkv, [L] * batch, (L + 31) // 32 * 32, seed=L)
    q = torch.randn(batch * n, cfg.n_q_heads, 128,
                    generator=torch.Generator().manual_seed(L)).half().cuda()
    ws = kvq.block8_workspace(cfg, n)
    outs = [kvq.kvq_block8_attn(cache, q, ints([L] * batch), workspace=ws) for _ in range(3)]
    check(cfg, outs[0], q, [L] * batch, [n] * batch, seen)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    out = kvq.kvq_block8_attn(cache, q, ints([L] * batch), workspace=ws, window=65, sinks=3)
    check(cfg, out, q, [L] * batch, [n] * batch, seen, 65, 3)
    assert (ws[:4 * 152] == 0).all() and cache.flags() == 0


def test_positions_outside_the_tables(kvq_lib):
    """They take the nearest row, and the flag says so."""
    w = World(1, 4, 2, 128, "fp16", seed=22)
    w.append([60], n_positions=64)
    assert w.cache.flags() == 0
    w.append([20], n_positions=64)
    w.check_state()
    assert w.cache.flags() == kvq.FLAG_BAD_BATCH
    w.cache.clear_flags()
    w.append([3], positions=[-1, 5, 2 ** 31 - 1], n_positions=64)
    w.check_state()
    assert w.cache.flags() == kvq.FLAG_BAD_BATCH


def test_two_calls_at_once(kvq_lib):
    """Two layers on two streams, workspaces of their own: single tokens beside a chunk."""
    made = [filled("fp16", 2, 2, [900, 700], 928, seed=30 + i) for i in range(2)]
    g = torch.Generator().manual_seed(31)
    counts = ([1, 1], [120, 90])
    args, want = [], []
    for (cfg, cache, _), n in zip(made, counts):
        q = torch.randn(sum(n), cfg.n_q_heads, 128, generator=g).half().cuda()
        kw = dict(starts=ints([0, n[0], sum(n)]), max_new=max(n),
                  workspace=kvq.block8_workspace(cfg, max(n)))
        args.append((cache, q, ints([900, 700]), kw))
        want.append(kvq.kvq_block8_attn(*args[-1][:3], **kw))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        got = [kvq.kvq_block8_attn(*a[:3], stream=s, **a[3]) for a, s in zip(args, streams)]
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for (cfg, _, seen), n, out, a in zip(made, counts, want, args):
        check(cfg, out, a[1], [900, 700], n, seen)
