"""Operators of a serving loop on an 8-bit paged cache, as they are measured.

* ``append``  new keys and values of a ragged batch go to a paged cache of e4m3
              blocks (32 tokens and a head to a scale), keys and queries with the
              position rotation applied on the way;
* ``attend``  causal attention of the newest tokens of each sequence over that
              cache: single tokens, drafts, prompt chunks, mixed batches, with an
              optional sliding window and first tokens that stay visible;
* ``adjust``  penalties for repeated tokens, biases and a grammar's bit mask on
              rows of logits, ahead of sampling.

With ``own`` false the operators run as elementary torch operations in fp32; with
``own`` true they are the package's calls on the same tensors.
"""

import math

import torch

own = False

D = 128          # head size
G = 32           # tokens of a block
RING = 2 * G     # unquantized tokens kept at the end of a sequence
E4M3 = 448.0     # largest code
DEV = "cuda"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    a = dict(kind="append", paired=0, chunk=0)
    t = dict(kind="attend", window=0, sinks=0, chunk=0)
    z = dict(kind="adjust")
    return [
        # the next token of one long chat: the smallest append, latency alone
        dict(a, name="append_b1_token", type="fp16", batch=1, hq=32, hkv=8, lo=32773, ctx=32773,
             n_lo=1, n_hi=1, rot=128),
        # one to eight drafts in every sequence, half of each head rotated in pairs
        dict(a, name="append_b64_drafts_bf16", type="bf16", batch=64, hq=40, hkv=8, lo=500,
             ctx=8192, n_lo=1, n_hi=8, rot=64, paired=1),
        # 32 single tokens and a whole prompt of odd length: the largest append
        dict(a, name="append_b33_prompt8191", type="fp16", batch=33, hq=32, hkv=8, lo=2000,
             ctx=32768, n_lo=1, n_hi=1, chunk=8191, rot=128),
        # the next token of one long chat: the smallest attention, latency alone
        dict(t, name="attend_b1_token_32k", type="fp16", batch=1, hq=32, hkv=8, lo=32773,
             ctx=32773, n_lo=1, n_hi=1),
        # single tokens of a ragged batch, query groups of eight
        dict(t, name="attend_b32_token_g8_bf16", type="bf16", batch=32, hq=64, hkv=8, lo=2048,
             ctx=32768, n_lo=1, n_hi=1),
        # one to five drafts verified in every sequence of a ragged batch
        dict(t, name="attend_b16_drafts", type="fp16", batch=16, hq=32, hkv=8, lo=8192, ctx=32768,
             n_lo=1, n_hi=5),
        # single tokens with a sliding window and sinks
        dict(t, name="attend_b16_window", type="fp16", batch=16, hq=32, hkv=8, lo=8192, ctx=32768,
             n_lo=1, n_hi=1, window=4096, sinks=4),
        # a chunk of one long prompt among 31 single tokens, query groups of five
        dict(t, name="attend_b32_mixed_bf16", type="bf16", batch=32, hq=40, hkv=8, lo=4096,
             ctx=32768, n_lo=1, n_hi=1, chunk=2048),
        # whole prompts of odd length: the largest attention
        dict(t, name="attend_prompt8191_b2", type="fp16", batch=2, hq=32, hkv=8, lo=8191, ctx=8191,
             n_lo=8191, n_hi=8191),
        # one chat's row of a 128k vocabulary, penalties alone
        dict(z, name="adjust_b1_v128256", type="fp32", rows=1, vocab=128256, lo=2000, hist=2000,
             bias=0, mask=0),
        # long histories on a 32k vocabulary with a grammar
        dict(z, name="adjust_b16_v32768_fp16", type="fp16", rows=16, vocab=32768, lo=32768,
             hist=32768, bias=16, mask=1),
        # a large batch with everything, odd vocabulary: rows that are not aligned
        dict(z, name="adjust_b128_v152063_bf16", type="bf16", rows=128, vocab=152063, lo=100,
             hist=4000, bias=300, mask=1),
    ]


def _log(rng, lo, hi):
    """A whole number spread over [lo, hi] by its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "adjust", "adjust"])
    if kind == "adjust":
        hist = _log(rng, 1, 32768)
        return dict(kind=kind, type=rng.choice(["fp32", "fp16", "bf16"]), rows=_log(rng, 1, 128),
                    vocab=_log(rng, 2000, 152063), lo=rng.choice([0, hist // 4, hist]), hist=hist,
                    bias=rng.choice([0, 1, 16, 300]), mask=rng.randrange(2))
    while True:
        hkv = rng.choice([1, 2, 4, 8, 8])
        ctx = _log(rng, 40, 32768)
        n_hi = rng.choice([1, 1, 5, 8])
        case = dict(kind=kind, type=rng.choice(["fp16", "bf16"]), batch=_log(rng, 1, 64),
                    hq=hkv * rng.choice([1, 2, 4, 4, 5, 7, 8, 12]), hkv=hkv,
                    lo=rng.choice([ctx, max(8, ctx // 5)]), ctx=ctx, n_lo=1, n_hi=n_hi, chunk=0)
        if rng.random() < 0.5:
            case["chunk"] = _log(rng, 33, 8191)
        if kind == "append":
            case.update(rot=rng.choice([128, 128, 64, 32, 96, 0]), paired=rng.randrange(2))
            tokens = case["batch"] * n_hi + case["chunk"]
            if tokens * (case["hq"] + hkv) <= 8191 * 40:
                return case
            continue
        case.update(chunk=min(case["chunk"], ctx), window=0, sinks=0)
        if rng.random() < 0.4:
            case.update(window=_log(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 33, 128]))
        longest = max(case["chunk"], n_hi)
        if work(case)["flops"] <= 1e12 and case["batch"] * hkv * ctx <= 32 * 8 * 32768 \
                and longest * case["hq"] * ctx <= 2 << 30:
            return case


# ---------------------------------------------------------------------------
# Sizes and work
# ---------------------------------------------------------------------------


def _spread(lo, hi, i):
    """Evenly spread whole numbers of [lo, hi] in a scattered order."""
    return lo + int((hi - lo + 1) * ((0.5 + 0.6180339887 * i) % 1.0))


def _sizes(c):
    """(tokens before the call, new tokens) of each sequence.  A long chunk
    comes last and starts at a block's first token, a prompt at 0."""
    got = []
    for b in range(c["batch"]):
        n = _spread(c["n_lo"], c["n_hi"], b + 1)
        total = max(n, _spread(c["lo"], c["ctx"], b))
        got.append((total - n, n))
    if c["chunk"]:
        n = c["chunk"]
        before = 0 if c["kind"] == "append" else (c["ctx"] - n) // G * G
        got[-1] = (before, n)
    return got


def _span(p0, p1, window, sinks):
    """Tokens that queries at positions p0 .. p1 see: [0, a) and [lo, p1]."""
    lo = max(0, p0 - window + 1) if window else 0
    return min(sinks, lo) if window else 0, lo


def work(case):
    c = case
    if c["kind"] == "adjust":
        width = 4 if c["type"] == "fp32" else 2
        tokens = sum(_history(c))
        per_row = c["vocab"] * (width + 4) + 8 * c["bias"] + 20
        if c["mask"]:
            per_row += c["vocab"] // 8
        return {"bytes": c["rows"] * per_row + 4 * tokens, "flops": 2 * c["rows"] * c["vocab"]}
    nbytes = flops = 0
    for before, n in _sizes(c):
        L = before + n
        if c["kind"] == "append":
            blocks = L // G - before // G
            nbytes += n * D * 2 * (2 * c["hkv"] + 2 * c["hq"])          # k, v, q in, q out
            nbytes += n * c["rot"] * 4                                  # cosines and sines
            nbytes += blocks * c["hkv"] * (2 * G * D + 8)               # codes and scales
            nbytes += min(n, L % G + G) * c["hkv"] * D * 4              # the newest, unquantized
            if blocks:
                nbytes += before % G * c["hkv"] * D * 4                 # the begun block's
            flops += n * (c["rot"] * 3 * (c["hq"] + c["hkv"]) + 4 * D * c["hkv"])
            continue
        nbytes += n * c["hq"] * D * 4
        a, lo = _span(before, L - 1, c["window"], c["sinks"])
        full = L // G * G
        codes = min(a, full) + max(0, full - lo)
        nbytes += c["hkv"] * (codes * 2 * D + codes // G * 8 + (a + L - lo - codes) * 4 * D)
        if c["window"]:
            for p in range(before, L):
                a, lo = _span(p, p, c["window"], c["sinks"])
                flops += 4 * D * c["hq"] * (a + p + 1 - lo)
        else:
            flops += 4 * D * c["hq"] * (n * before + n * (n + 1) // 2)
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------


def _gen(seed, part):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + part * 7919 + 29) % (1 << 62))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return _ints(at)


def _normal(shape, g, dtype):
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def _boost(hkv, g):
    """Four channels of every key head ten times as large."""
    f = torch.ones(hkv, 1, D, device=DEV)
    for h in range(hkv):
        f[h, 0, torch.randperm(D, generator=g, device=DEV)[:4]] = 10.0
    return f


def _scale_of(amax):
    """The fp32 scale of a block whose largest magnitude is amax (fp32)."""
    # (a division by a Python number would be a product with its reciprocal)
    s = torch.clamp(amax / torch.full_like(amax, E4M3), 2.0 ** -60, 2.0 ** 60)
    return torch.where(amax > 0, s, torch.ones_like(s))


def _codes(x, scale):
    return torch.clamp(x / scale, -E4M3, E4M3).to(torch.float8_e4m3fn)


def _history(c):
    return [_spread(c["lo"], c["hist"], i) for i in range(c["rows"])]


def _adjust_state(c, seed):
    g = _gen(seed, 1)
    rows, V = c["rows"], c["vocab"]
    z = _normal((rows, V), g, torch.float32).mul_(3.0).to(TYPES[c["type"]])
    counts = _history(c)
    total = sum(counts)
    # a text: a few tokens often, the others seldom; the first third is the prompt
    u = torch.rand(total, generator=g, device=DEV)
    hist = (u ** 4 * V).to(torch.int32).clamp_(max=V - 1)
    st = dict(case=c, logits=z, history=hist, history_starts=_starts(counts),
              prompt_lengths=_ints([n // 3 for n in counts]), total=total,
              repetition=torch.rand(rows, generator=g, device=DEV) * 0.4 + 1.0,
              frequency=torch.rand(rows, generator=g, device=DEV) * 0.6,
              presence=torch.rand(rows, generator=g, device=DEV) * 0.9,
              bias_ids=None, bias_values=None, bias_starts=None, mask=None)
    if c["bias"]:
        st["bias_ids"] = torch.randint(0, V, (rows * c["bias"],), generator=g, device=DEV,
                                       dtype=torch.int32)
        st["bias_values"] = torch.randn(rows * c["bias"], generator=g, device=DEV) * 5.0
        st["bias_starts"] = _starts([c["bias"]] * rows)
    if c["mask"]:
        # grammars that allow half of the tokens in runs of 32, some words mixed
        words = (V + 31) // 32
        bits = torch.randint(-2 ** 31, 2 ** 31, (rows, words), generator=g, device=DEV)
        kind = torch.randint(0, 3, (rows, words), generator=g, device=DEV)
        bits = torch.where(kind == 0, torch.zeros_like(bits), bits)
        st["mask"] = torch.where(kind == 1, torch.full_like(bits, -1), bits).to(torch.int32)
    st["out"] = torch.empty(rows, V, device=DEV)
    return st


def _cache_state(c, seed):
    """A cache's tensors and a batch's sizes."""
    B, hkv, dt = c["batch"], c["hkv"], TYPES[c["type"]]
    sizes = _sizes(c)
    lens = [before + n for before, n in sizes]
    T = sum(n for _, n in sizes)
    g = _gen(seed, 0)
    need = [range(before // G, (before + n) // G) if c["kind"] == "append"
            else range((before + n) // G) for before, n in sizes]
    pages = max(1, sum(len(r) for r in need))
    order = torch.randperm(pages, generator=g, device=DEV).tolist()
    width = max(1, (max(lens) + G - 1) // G)
    table = torch.full((B, width), -1, dtype=torch.int32)
    at = 0
    for b, r in enumerate(need):
        table[b, r.start:r.stop] = torch.tensor(order[at:at + len(r)], dtype=torch.int32)
        at += len(r)
    boost = _boost(hkv, g)
    st = dict(case=c, tokens=T, lens=lens, table=table.to(DEV), lengths=_ints(lens),
              starts=_starts([n for _, n in sizes]), max_new=max(n for _, n in sizes),
              blocks=sum(len(r) for r in need),
              k_ring=(_normal((B, hkv, RING, D), g, torch.float32) * boost).to(dt),
              v_ring=_normal((B, hkv, RING, D), g, dt))
    if c["kind"] == "append":
        for name in ("k_codes", "v_codes"):
            st[name] = torch.zeros(pages, hkv, G, D, device=DEV).to(torch.float8_e4m3fn)
        st["scales"] = torch.ones(pages, hkv, 2, device=DEV)
        # one projection holds queries, keys and values
        st["qkv"] = _normal((T, c["hq"] + 2 * hkv, D), g, torch.float32)
        st["qkv"][:, c["hq"]:c["hq"] + hkv] *= boost[:, 0]
        st["qkv"] = st["qkv"].to(dt)
        st["q_out"] = torch.zeros(T, c["hq"], D, dtype=dt, device=DEV)
        half = c["rot"] // 2
        angle = torch.arange(max(lens), dtype=torch.float64, device=DEV)[:, None] \
            * 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) / max(1, half))
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        return st
    # a cache as appending leaves it
    k = _normal((pages, hkv, G, D), g, torch.float32).mul_(boost)
    v = _normal((pages, hkv, G, D), g, torch.float32)
    sk, sv = (_scale_of(x.abs().amax((2, 3))) for x in (k, v))
    st["k_codes"], st["v_codes"] = _codes(k, sk[..., None, None]), _codes(v, sv[..., None, None])
    st["scales"] = torch.stack([sk, sv], -1)
    st["q"] = _normal((T, c["hq"], D), g, dt)
    st["out"] = torch.zeros(T, c["hq"], D, dtype=dt, device=DEV)
    return st


def prepare(case, seed):
    c = case
    if c["kind"] == "adjust":
        return _adjust_state(c, seed)
    st = _cache_state(c, seed)
    if own:
        # the handle of the same tensors, and a workspace
        from paper_2607_16248_gb300 import kvq
        cfg = kvq.Block8Config(batch=c["batch"], n_q_heads=c["hq"], n_kv_heads=c["hkv"],
                               max_len=st["table"].shape[1] * G, dtype=TYPES[c["type"]])
        st["cache"] = kvq.Block8Cache(cfg, tensors={n: st[n] for n in (
            "k_codes", "v_codes", "scales", "k_ring", "v_ring")}, block_table=st["table"])
        if c["kind"] == "attend":
            st["workspace"] = kvq.block8_workspace(cfg, st["max_new"])
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------


def _rounded(x, dtype):
    """x (fp64) to the nearest of a 16-bit type: by way of the fp32 number
    towards zero, made odd where it is not x, so that the second rounding sees
    on which side of a border x lies."""
    f = x.float()
    f = torch.where(f.double().abs() > x.abs(), torch.nextafter(f, torch.zeros_like(f)), f)
    return (f.view(torch.int32) | (f.double() != x).int()).view(torch.float32).to(dtype)


def _rotated(x, cos, sin, paired):
    """x [T, H, 128] with its first 2 * cos.shape[1] channels rotated."""
    r = cos.shape[1]
    cos, sin = cos[:, None], sin[:, None]
    if paired:
        x1, x2 = x[..., 0:2 * r:2], x[..., 1:2 * r:2]
        y = torch.stack([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1).flatten(-2)
    else:
        x1, x2 = x[..., :r], x[..., r:2 * r]
        y = torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1)
    return torch.cat([y, x[..., 2 * r:]], -1)


def _plain_append(st, c):
    hq, hkv, B, T = c["hq"], c["hkv"], c["batch"], st["tokens"]
    starts, total = st["starts"].long(), st["lengths"].long()
    n = starts[1:] - starts[:-1]
    before = total - n
    seq_of = torch.repeat_interleave(torch.arange(B, device=DEV), n, output_size=T)
    pos = torch.arange(T, device=DEV) - starts[seq_of] + before[seq_of]
    cos, sin = st["cos"][pos], st["sin"][pos]
    q, k, v = st["qkv"].split([hq, hkv, hkv], 1)
    st["q_out"].copy_(_rotated(q.float(), cos, sin, c["paired"]))
    # a key next to a border decides its block's scale and codes: in 64 bits
    k = _rounded(_rotated(k.double(), cos.double(), sin.double(), c["paired"]), k.dtype)
    heads = torch.arange(hkv, device=DEV)
    if st["blocks"]:
        # every block that the new tokens complete
        first, last = before // G, total // G
        nb = last - first
        s = torch.repeat_interleave(torch.arange(B, device=DEV), nb, output_size=st["blocks"])
        blk = torch.arange(st["blocks"], device=DEV) - (torch.cumsum(nb, 0) - nb)[s] + first[s]
        p = blk[:, None] * G + torch.arange(G, device=DEV)
        row = starts[s][:, None] + p - before[s][:, None]
        old = (p < before[s][:, None])[..., None, None]
        page = st["table"][s, blk].long()
        for name, new, ring, i in (("k_codes", k, st["k_ring"], 0), ("v_codes", v, st["v_ring"], 1)):
            kept = ring[s[:, None, None], heads[None, None], (p % RING)[:, :, None]]
            y = torch.where(old, kept, new[row.clamp(min=0)]).float().transpose(1, 2)
            scale = _scale_of(y.abs().amax((2, 3)))
            st["scales"][page, :, i] = scale
            st[name].view(torch.uint8)[page] = _codes(y, scale[..., None, None]).view(torch.uint8)
    # the newest tokens' places: those of the last two blocks
    p = ((total // G - 1) * G)[:, None] + torch.arange(RING, device=DEV)
    row = starts[:-1, None] + p - before[:, None]
    fresh = ((p >= before[:, None]) & (p < total[:, None]) & (p >= 0))[:, None, :, None]
    row = row.clamp(0, max(0, T - 1))
    at = (p % RING)[:, None, :, None].expand(B, hkv, RING, D)
    for new, ring in ((k, st["k_ring"]), (v, st["v_ring"])):
        kept = torch.gather(ring, 2, at)
        ring.scatter_(2, at, torch.where(fresh, new[row].transpose(1, 2), kept))
    return [st[x] for x in ("q_out", "k_codes", "v_codes", "scales", "k_ring", "v_ring")]


def _plain_group(st, c, which, n):
    """The sequences `which` (a list), each with n new tokens."""
    hkv, gq, B = c["hkv"], c["hq"] // c["hkv"], len(which)
    idx = torch.tensor(which, device=DEV)
    total = st["lengths"].long()[idx]
    most = max(st["lens"][b] for b in which) // G
    page = st["table"][idx, :most].long().clamp(min=0)
    cols = torch.arange((most + 1) * G, device=DEV)
    tail = (total // G * G)[:, None] + torch.arange(G, device=DEV)
    kv = []
    for name, ring, i in (("k_codes", st["k_ring"], 0), ("v_codes", st["v_ring"], 1)):
        x = torch.zeros(B, hkv, (most + 1) * G, D, device=DEV)
        y = st[name].view(torch.uint8)[page].view(torch.float8_e4m3fn).float()
        y = y * st["scales"][page][..., i, None, None]
        x[:, :, :most * G] = y.transpose(1, 2).reshape(B, hkv, most * G, D)
        newest = torch.gather(ring[idx].float(), 2,
                              (tail % RING)[:, None, :, None].expand(B, hkv, G, D))
        kv.append(x.scatter_(2, tail[:, None, :, None].expand(B, hkv, G, D), newest))
    rows = st["starts"].long()[idx][:, None] + torch.arange(n, device=DEV)
    q = st["q"][rows].float().view(B, n, hkv, gq, D).permute(0, 2, 3, 1, 4)
    sc = torch.matmul(q.reshape(B, hkv, gq * n, D), kv[0].transpose(2, 3))
    sc = sc.mul_(1.0 / math.sqrt(D)).view(B, hkv, gq, n, -1)
    pos = (total[:, None] - n + torch.arange(n, device=DEV))[..., None]
    hide = cols > pos
    if c["window"]:
        hide = hide | ((cols <= pos - c["window"]) & (cols >= c["sinks"]))
    sc.masked_fill_(hide[:, None, None], -math.inf)
    e = sc.sub_(sc.amax(-1, keepdim=True)).exp_()
    # what lies behind a sequence's end is masked, whatever it holds
    o = torch.matmul(e.view(B, hkv, gq * n, -1), kv[1]).view(B, hkv, gq, n, D)
    o = o / e.sum(-1, keepdim=True)
    st["out"][rows] = o.permute(0, 3, 1, 2, 4).reshape(B, n, c["hq"], D).to(st["out"].dtype)


def _plain_attend(st, c):
    """Sequences of as many new tokens go together."""
    counts = [n for _, n in _sizes(c)]
    for n in sorted(set(counts)):
        _plain_group(st, c, [b for b, m in enumerate(counts) if m == n], n)
    return st["out"]


def _plain_adjust(st, c):
    rows, V, T = c["rows"], c["vocab"], st["total"]
    z = st["logits"].float()
    hs = st["history_starts"].long()
    row = torch.repeat_interleave(torch.arange(rows, device=DEV), hs[1:] - hs[:-1], output_size=T)
    at = row * V + st["history"]
    answer = torch.arange(T, device=DEV) - hs[row] >= st["prompt_lengths"][row]
    zero = torch.zeros(rows * V, dtype=torch.int32, device=DEV)
    count = zero.index_add(0, at, answer.int()).view(rows, V)
    seen = zero.index_add(0, at, torch.ones_like(row, dtype=torch.int32)).view(rows, V) > 0
    rep = st["repetition"][:, None]
    z = torch.where(seen, torch.where(z > 0, z / rep, z * rep), z)
    z = torch.where(count > 0, z - st["frequency"][:, None] * count - st["presence"][:, None], z)
    if c["bias"]:
        bs = st["bias_starts"].long()
        row = torch.repeat_interleave(torch.arange(rows, device=DEV), bs[1:] - bs[:-1],
                                      output_size=rows * c["bias"])
        number = torch.arange(1, rows * c["bias"] + 1, dtype=torch.int32, device=DEV)
        slot = zero.scatter_reduce(0, row * V + st["bias_ids"], number, "amax").view(rows, V)
        # of an id that is there twice, the later counts
        z = torch.where(slot > 0, z + st["bias_values"][(slot - 1).clamp(min=0)], z)
    if c["mask"]:
        v = torch.arange(V, device=DEV)
        allowed = (st["mask"][:, v // 32] >> (v % 32)) & 1
        z = torch.where(allowed > 0, z, torch.full_like(z, -math.inf))
    st["out"].copy_(z)
    return st["out"]


def run(state):
    st, c = state, state["case"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "adjust": _plain_adjust}[
            c["kind"]](st, c)
    from paper_2607_16248_gb300 import kvq
    if c["kind"] == "adjust":
        return kvq.kvq_adjust_logits(
            st["logits"], out=st["out"], history=st["history"],
            history_starts=st["history_starts"], prompt_lengths=st["prompt_lengths"],
            repetition=st["repetition"], frequency=st["frequency"], presence=st["presence"],
            bias_ids=st["bias_ids"], bias_values=st["bias_values"],
            bias_starts=st["bias_starts"], mask=st["mask"])
    if c["kind"] == "attend":
        return kvq.kvq_block8_attn(st["cache"], st["q"], st["lengths"], starts=st["starts"],
                             max_new=st["max_new"], window=c["window"], sinks=c["sinks"],
                             out=st["out"], workspace=st["workspace"])
    q, k, v = st["qkv"].split([c["hq"], c["hkv"], c["hkv"]], 1)
    kvq.kvq_block8_append(st["cache"], k, v, st["lengths"], starts=st["starts"], q=q,
                    q_out=st["q_out"], cos=st["cos"], sin=st["sin"], paired=bool(c["paired"]))
    return [st[x] for x in ("q_out", "k_codes", "v_codes", "scales", "k_ring", "v_ring")]


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------


def _to_bits(x, bits, least):
    """x (fp64) to the nearest of `bits` significant bits, ties to even, steps
    of at least 2^least."""
    _, e = torch.frexp(x)
    # 2^q from its bits: a power function need not be exact
    step = ((torch.clamp(e.long() - bits, min=least) + 1023) << 52).view(torch.float64)
    return torch.round(x / step) * step


def _exact_append(c, seed):
    """The state after the call, sequence by sequence and token by token range."""
    st = _cache_state(c, seed)
    hq, hkv = c["hq"], c["hkv"]
    bits, least = (11, -24) if c["type"] == "fp16" else (8, -133)
    x = st["qkv"].double()
    cos, sin = st["cos"].double(), st["sin"].double()
    r = c["rot"] // 2
    i = torch.arange(r, device=DEV)
    one, two = (2 * i, 2 * i + 1) if c["paired"] else (i, i + r)
    codes = [st["k_codes"].double(), st["v_codes"].double()]
    scales, rings = st["scales"].double(), [st["k_ring"].double(), st["v_ring"].double()]
    row = 0
    for b, (before, n) in enumerate(_sizes(c)):
        here = x[row:row + n, :hq + hkv]
        z = torch.complex(here[..., one], here[..., two]) * torch.complex(
            cos[before:before + n], sin[before:before + n])[:, None]
        here[..., one], here[..., two] = z.real, z.imag
        x[row:row + n, hq:hq + hkv] = _to_bits(here[:, hq:], bits, least)
        total = before + n
        for which in (0, 1):
            y = x[row:row + n, hq + hkv * which:hq + hkv * (which + 1)].transpose(0, 1)
            begun = before % G
            if begun:
                slots = [p % RING for p in range(before - begun, before)]
                y = torch.cat([rings[which][b][:, slots], y], 1)
            done = total // G - before // G
            full = y[:, :done * G].reshape(hkv, done, G, D)
            amax = full.abs().amax((2, 3))
            s = _to_bits(torch.clamp(amax / E4M3, 2.0 ** -60, 2.0 ** 60), 24, -149)
            s = torch.where(amax > 0, s, torch.ones_like(s))
            page = st["table"][b, before // G:total // G].long()
            scales[page, :, which] = s.T
            quotient = _to_bits(full / s[..., None, None], 24, -149)
            codes[which][page] = _to_bits(quotient, 4, -9).clamp(-E4M3, E4M3).transpose(0, 1)
            keep = range(max(before, (total // G - 1) * G), total)
            rings[which][b][:, [p % RING for p in keep]] = y[:, y.shape[1] - len(keep):]
        row += n
    return [x[:, :hq].contiguous(), codes[0], codes[1], scales, rings[0], rings[1]]


def _exact_attend(c, seed):
    if work(c)["flops"] > 4e12:
        return None
    st = _cache_state(c, seed)
    gq = c["hq"] // c["hkv"]
    out = torch.zeros(st["tokens"], c["hq"], D, dtype=torch.float64, device=DEV)
    row = 0
    for b, (before, n) in enumerate(_sizes(c)):
        L = before + n
        page = st["table"][b, :L // G].long()
        rest = [p % RING for p in range(L // G * G, L)]
        for h in range(c["hkv"]):
            kv = []
            for i, name in enumerate(("k_codes", "v_codes")):
                x = st[name].view(torch.uint8)[page, h].view(torch.float8_e4m3fn).double()
                x = (x * st["scales"][page, h, i].double()[:, None, None]).reshape(-1, D)
                ring = st["k_ring" if i == 0 else "v_ring"]
                kv.append(torch.cat([x, ring[b, h, rest].double()]))
            for t0 in range(0, n, 512):
                t1 = min(n, t0 + 512)
                pos = torch.arange(before + t0, before + t1, device=DEV)
                end = before + t1
                begin = max(0, before + t0 + 1 - c["window"]) if c["window"] else 0
                cols = torch.arange(end, device=DEV)
                cols = cols[(cols >= begin) | (cols < c["sinks"])]
                seen = cols <= pos[:, None]
                if c["window"]:
                    seen &= (cols > pos[:, None] - c["window"]) | (cols < c["sinks"])
                q = st["q"][row + t0:row + t1, h * gq:(h + 1) * gq].double()
                s = torch.einsum("tgd,cd->tgc", q, kv[0][cols]) / math.sqrt(D)
                w = torch.softmax(s.masked_fill(~seen[:, None], -math.inf), -1)
                out[row + t0:row + t1, h * gq:(h + 1) * gq] = torch.einsum(
                    "tgc,cd->tgd", w, kv[1][cols])
        row += n
    return out


def _exact_adjust(c, seed):
    st = _adjust_state(c, seed)
    hist, hs = st["history"].long(), st["history_starts"].tolist()
    prompts = st["prompt_lengths"].tolist()
    out = st["logits"].double()
    for b in range(c["rows"]):
        z = out[b]
        text = hist[hs[b]:hs[b + 1]]
        rep, freq, pres = (float(st[x][b]) for x in ("repetition", "frequency", "presence"))
        met = torch.unique(text)
        z[met] = torch.where(z[met] > 0, z[met] / rep, z[met] * rep)
        said, times = torch.unique(text[prompts[b]:], return_counts=True)
        z[said] -= freq * times.double() + pres
        if c["bias"]:
            ids = st["bias_ids"][b * c["bias"]:(b + 1) * c["bias"]].tolist()
            last = dict(zip(ids, st["bias_values"][b * c["bias"]:(b + 1) * c["bias"]].tolist()))
            at = torch.tensor(list(last), device=DEV)
            z[at] += torch.tensor(list(last.values()), dtype=torch.float64, device=DEV)
        if c["mask"]:
            bits = (st["mask"][b][:, None] >> torch.arange(32, device=DEV)) & 1
            z[bits.flatten()[:c["vocab"]] == 0] = -math.inf
    return out


def exact(case, seed):
    return {"append": _exact_append, "attend": _exact_attend, "adjust": _exact_adjust}[
        case["kind"]](case, seed)
