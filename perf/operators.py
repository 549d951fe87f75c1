"""Operators of a serving loop around the low-bit cache, as they are measured.

* ``chunk``   attention of the ``n_q`` newest tokens of each sequence over its
              KbVb cache (contiguous or paged), causal, for prompts that arrive
              in chunks and for draft tokens that are verified;
* ``window``  the same with a sliding window of ``window`` tokens and ``sinks``
              first tokens that stay visible, for chunks and for single tokens;
* ``sample``  the next token of each row of logits by temperature, top-k, top-p
              and min-p from given random numbers.

With ``own`` false the operators run as elementary torch operations in fp32 on
plainly stored codes, scales and zero points; with ``own`` true they are the
package's calls on its own cache.
"""

import math

import torch

own = False

D = 128        # head size
G = 32         # tokens (keys) or channels (values) of a quantization group
R = 128        # fp16 tokens kept at the end of a sequence
DEV = "cuda"


def listed():
    c = dict(kind="chunk", window=0, sinks=0, paged=False)
    w = dict(c, kind="window")
    return [
        # five draft tokens verified over one long chat, one-bit cache
        dict(c, name="verify_b1_32k_k1v1", batch=1, hq=32, hkv=8, bk=1, bv=1, ctx=32773, lo=32773,
             n_q=5),
        # four draft tokens in every sequence of a ragged batch on paged blocks
        dict(c, name="verify_b16_ragged_k2v2_paged", batch=16, hq=32, hkv=8, bk=2, bv=2,
             ctx=32768, lo=8192, n_q=4, paged=True),
        # the second chunk of a short prompt
        dict(c, name="chunk512_b1_4k_k2v2", batch=1, hq=32, hkv=8, bk=2, bv=2, ctx=4099, lo=4099,
             n_q=512),
        # a chunk of a long document, query groups of five, paged: the largest
        dict(c, name="chunk2048_b1_64k_k1v1_g5_paged", batch=1, hq=40, hkv=8, bk=1, bv=1,
             ctx=65536, lo=65536, n_q=2048, paged=True),
        # whole prompts of odd length from an empty cache, four-bit cache
        dict(c, name="prompt8191_b2_k4v4", batch=2, hq=32, hkv=8, bk=4, bv=4, ctx=8191, lo=8191,
             n_q=8191),
        # single tokens of a batch with a window and sinks, paged
        dict(w, name="token_b16_w4096_k2v2_paged", batch=16, hq=32, hkv=8, bk=2, bv=2, ctx=32768,
             lo=8192, n_q=1, window=4096, sinks=4, paged=True),
        # one token of one sequence: the smallest call, latency alone
        dict(w, name="token_b1_w1024_k1v1", batch=1, hq=32, hkv=8, bk=1, bv=1, ctx=32768,
             lo=32768, n_q=1, window=1024, sinks=4),
        # a chunk of a long stream with an odd window, eight-bit keys
        dict(w, name="chunk4096_b1_w1023_k8v4_g8", batch=1, hq=64, hkv=8, bk=8, bv=4, ctx=20001,
             lo=20001, n_q=4096, window=1023, sinks=33),
        # one row of a 128k vocabulary, usual settings: a decode step's tail
        dict(kind="sample", name="sample_b1_v128256", batch=1, vocab=128256, mixed=0,
             temperature=0.8, top_k=50, top_p=0.95, min_p=0.0),
        # rows that ask for different settings, 32k vocabulary
        dict(kind="sample", name="sample_b16_v32768_mixed", batch=16, vocab=32768, mixed=1,
             temperature=0.7, top_k=40, top_p=0.9, min_p=0.02),
        # a large batch by nucleus alone, odd vocabulary: rows not 16-byte aligned
        dict(kind="sample", name="sample_b128_v152063_topp", batch=128, vocab=152063, mixed=0,
             temperature=1.0, top_k=0, top_p=0.9, min_p=0.0),
        # a large batch of mixed settings
        dict(kind="sample", name="sample_b64_v152064_mixed", batch=64, vocab=152064, mixed=1,
             temperature=1.0, top_k=200, top_p=0.8, min_p=0.05),
    ]


def _log(rng, lo, hi):
    """A whole number spread over [lo, hi] by its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["chunk", "chunk", "window", "window", "sample"])
    if kind == "sample":
        return dict(kind=kind, batch=_log(rng, 1, 128), vocab=_log(rng, 2000, 152064),
                    mixed=rng.randrange(2), temperature=rng.uniform(0.5, 1.3),
                    top_k=rng.choice([0, 1, 20, 50, 64, 300]),
                    top_p=rng.choice([1.0, 0.99, 0.95, 0.9, 0.7]),
                    min_p=rng.choice([0.0, 0.0, 0.02, 0.1]))
    while True:
        hkv = rng.choice([1, 2, 4, 8, 8])
        batch = _log(rng, 1, 16)
        ctx = _log(rng, 200, 65536)
        bk = rng.choice([1, 2, 4, 8])
        case = dict(kind=kind, batch=batch, hq=hkv * rng.choice([1, 2, 4, 4, 5, 7, 8]), hkv=hkv,
                    bk=bk, bv=bk if rng.random() < 0.7 else rng.choice([1, 2, 4, 8]), ctx=ctx,
                    lo=ctx if rng.random() < 0.5 else max(1, ctx // 4),
                    n_q=_log(rng, 1, min(ctx, 8192)), window=0, sinks=0,
                    paged=rng.random() < 0.4)
        if kind == "window":
            case.update(window=_log(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 33, 128]),
                        n_q=1 if rng.random() < 0.4 else case["n_q"])
        if work(case)["flops"] <= 1e12 and batch * hkv * ctx <= 16 * 8 * 32768:
            return case


# ---------------------------------------------------------------------------
# Work
# ---------------------------------------------------------------------------


def _lengths(c):
    """Sequence lengths in [lo, ctx], spread evenly in a scattered order."""
    if c["lo"] >= c["ctx"] or c["batch"] == 1:
        return [c["ctx"]] * c["batch"]
    return [c["lo"] + int((c["ctx"] - c["lo"]) * ((0.5 + 0.6180339887 * i) % 1.0))
            for i in range(c["batch"])]


def _packed(L):
    return G * (max(L - R, 0) // G)


def _ranges(p0, p1, window, sinks):
    """Tokens that queries at positions p0 .. p1 can see: [0, a) and [lo, p1]."""
    lo = max(0, p0 - window + 1) if window else 0
    return min(sinks, lo), lo


def work(case):
    c = case
    if c["kind"] == "sample":
        # the logits, the random numbers of what stays, a token and a float a row
        keep = c["top_k"] if c["top_k"] > 0 and not c["mixed"] else 0
        return {"bytes": c["batch"] * (4 * c["vocab"] + 4 * keep + 24),
                "flops": 3 * c["batch"] * c["vocab"]}
    tokens = 0
    nbytes = c["batch"] * c["n_q"] * c["hq"] * D * 4       # queries and results
    for L in _lengths(c):
        n = min(c["n_q"], L)
        a, lo = _ranges(L - n, L - 1, c["window"], c["sinks"])
        lq = _packed(L)
        packed = min(a, lq) + max(0, lq - lo)
        fp16 = (a + L - lo) - packed
        nbytes += c["hkv"] * (packed * (16 * (c["bk"] + c["bv"]) + 32) + fp16 * 4 * D)
        for p in (range(L - n, L) if c["window"] else ()):
            a, lo = _ranges(p, p, c["window"], c["sinks"])
            tokens += a + p + 1 - lo
        if not c["window"]:
            tokens += n * (L - n) + n * (n + 1) // 2
    return {"bytes": nbytes, "flops": 4 * D * c["hq"] * tokens}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------


def _gen(seed, part):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + part * 7919 + 17) % (1 << 62))
    return g


def _kv(c, L, g):
    """Keys and values fp16 [hkv, L, 128]: normal, with four channels of every
    key head ten times as large (what makes low-bit keys hard)."""
    k = torch.randn(c["hkv"], L, D, generator=g, device=DEV)
    v = torch.randn(c["hkv"], L, D, generator=g, device=DEV)
    boost = torch.ones(c["hkv"], 1, D, device=DEV)
    for h in range(c["hkv"]):
        boost[h, 0, torch.randperm(D, generator=g, device=DEV)[:4]] = 10.0
    return (k * boost).half(), v.half()


def _round_up32(x):
    """The least fp32 number >= x (fp64, >= 0)."""
    f = x.float()
    return torch.where(f.double() < x, torch.nextafter(f, torch.full_like(f, math.inf)), f)


def _round_up16(x):
    """The least fp16 number >= x (fp32, >= 0)."""
    h = x.half()
    up = (h.view(torch.int16) + 1).view(torch.float16)
    return torch.where(h.float() < x, up, h)


def _quantize(x, bits):
    """Codes uint8, scale and zero fp16 of groups x [..., 32]: zero the
    minimum, the scale rounded up, codes to the nearest."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    span = _round_up32(hi.double() - lo.double())
    scale = _round_up16(_round_up32(span.double() / (2 ** bits - 1)))
    q = torch.round((x.float() - lo.float()) / scale.float())
    codes = torch.where(scale > 0, q.clamp(0, 2 ** bits - 1), torch.zeros_like(q))
    return codes.to(torch.uint8), scale.squeeze(-1), lo.squeeze(-1)


def _store(c, k, v):
    """One sequence's cache, plainly stored."""
    L = k.shape[1]
    lq = _packed(L)
    kc, ks, kz = _quantize(k[:, :lq].reshape(c["hkv"], lq // G, G, D).transpose(2, 3), c["bk"])
    vc, vs, vz = _quantize(v[:, :lq].reshape(c["hkv"], lq, D // G, G), c["bv"])
    return dict(kc=kc, ks=ks, kz=kz, vc=vc, vs=vs, vz=vz, k=k[:, lq:].clone(), v=v[:, lq:].clone())


def _settings(c):
    """Per-row settings: those of the case, or a mix around them."""
    B = c["batch"]
    t, k, p, m = ([c[n]] * B for n in ("temperature", "top_k", "top_p", "min_p"))
    if c["mixed"]:
        t = [0.0 if i % 8 == 5 else c["temperature"] * (0.8 + 0.1 * (i % 5)) for i in range(B)]
        k = [c["top_k"] if i % 3 != 1 else 0 for i in range(B)]
        p = [c["top_p"] if i % 4 != 2 else 1.0 for i in range(B)]
        m = [c["min_p"] if i % 5 == 3 else 0.0 for i in range(B)]
    return (torch.tensor(t, dtype=torch.float32, device=DEV),
            torch.tensor(k, dtype=torch.int32, device=DEV),
            torch.tensor(p, dtype=torch.float32, device=DEV),
            torch.tensor(m, dtype=torch.float32, device=DEV))


def _sample_inputs(c, seed):
    """Logits normal with deviation 3, a few tokens of every row forbidden
    (-inf); random numbers uniform in [0, 1)."""
    g = _gen(seed, 1)
    z = torch.randn(c["batch"], c["vocab"], generator=g, device=DEV) * 3.0
    z[torch.rand(z.shape, generator=g, device=DEV) < 0.01] = -math.inf
    u = torch.rand(z.shape, generator=g, device=DEV)
    return z, u


def prepare(case, seed):
    c = case
    if c["kind"] == "sample":
        z, u = _sample_inputs(c, seed)
        t, k, p, m = _settings(c)
        st = dict(case=c, logits=z, noise=u, temperature=t, top_k=k, top_p=p, min_p=m)
        if own:
            from paper_2607_16248_gb300 import kvq
            st["outputs"] = kvq.sample_outputs(c["batch"])
        return st
    lens = _lengths(c)
    q = torch.randn(c["batch"], c["n_q"], c["hq"], D, generator=_gen(seed, 0), device=DEV).half()
    st = dict(case=c, lens=lens, q=q)
    if not own:
        st["seqs"] = [_store(c, *_kv(c, L, _gen(seed, 2 + b))) for b, L in enumerate(lens)]
        return st
    from paper_2607_16248_gb300 import kvq
    cfg = kvq.CacheConfig(batch=c["batch"], n_q_heads=c["hq"], n_kv_heads=c["hkv"],
                          bits_k=c["bk"], bits_v=c["bv"], max_len=(max(lens) + 31) // 32 * 32)
    need = [_packed(L) // G for L in lens]
    cache = kvq.QuantKVCache(cfg, n_pages=max(1, sum(need)) if c["paged"] else None)
    if c["paged"]:
        order = torch.randperm(max(1, sum(need)), generator=_gen(seed, 1), device=DEV).tolist()
        for b, n in enumerate(need):
            cache.map_blocks(b, range(n), order[sum(need[:b]):sum(need[:b]) + n])
    for b, L in enumerate(lens):
        k, v = _kv(c, L, _gen(seed, 2 + b))
        kvq.kvq_pack(cache, k[None], v[None], batch_begin=b)
    st.update(cache=cache, out=torch.empty_like(q),
              workspace=kvq.chunk_workspace(cfg, c["n_q"], c["batch"]))
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------


def _plain_sequence(c, s, q):
    """fp16 [n_q, hq, 128] of one sequence."""
    hkv, n_q, gq = c["hkv"], q.shape[0], c["hq"] // c["hkv"]
    k = s["kc"].float() * s["ks"].float()[..., None] + s["kz"].float()[..., None]
    k = torch.cat([k.transpose(2, 3).reshape(hkv, -1, D), s["k"].float()], 1)
    v = s["vc"].float() * s["vs"].float()[..., None] + s["vz"].float()[..., None]
    v = torch.cat([v.reshape(hkv, -1, D), s["v"].float()], 1)
    L = k.shape[1]
    out = torch.zeros(n_q, c["hq"], D, dtype=torch.float16, device=DEV)
    first = max(0, n_q - L)                  # queries ahead of the first token see nothing
    span = min(L, c["window"] + c["sinks"] + 512) if c["window"] else L
    step = max(1, (1 << 28) // (c["hq"] * span))
    for t0 in range(first, n_q, step):
        t1 = min(n_q, t0 + step)
        p0, p1 = L - n_q + t0, L - n_q + t1 - 1
        a, lo = _ranges(p0, p1, c["window"], c["sinks"])
        kk, vv = k[:, lo:p1 + 1], v[:, lo:p1 + 1]
        pos = torch.arange(lo, p1 + 1, device=DEV)
        if a:
            kk, vv = torch.cat([k[:, :a], kk], 1), torch.cat([v[:, :a], vv], 1)
            pos = torch.cat([torch.arange(a, device=DEV), pos])
        qq = q[t0:t1].float().reshape(t1 - t0, hkv, gq, D).permute(1, 2, 0, 3)
        sc = torch.matmul(qq.reshape(hkv, -1, D), kk.transpose(1, 2)) * (1.0 / math.sqrt(D))
        sc = sc.view(hkv, gq, t1 - t0, -1)
        row = torch.arange(p0, p1 + 1, device=DEV)[:, None]
        hide = pos[None] > row
        if c["window"]:
            hide = hide | ((pos[None] <= row - c["window"]) & (pos[None] >= c["sinks"]))
        sc = sc.masked_fill(hide, -math.inf)
        e = torch.exp(sc - sc.amax(-1, keepdim=True))
        o = torch.matmul(e.view(hkv, -1, e.shape[-1]), vv).view(hkv, gq, t1 - t0, D)
        o = o / e.sum(-1, keepdim=True)
        out[t0:t1] = o.permute(2, 0, 1, 3).reshape(t1 - t0, c["hq"], D).half()
    return out


def _plain_sample(z, u, t, top_k, top_p, min_p):
    """(token int32, logprob fp32) of each row."""
    B, V = z.shape
    greedy = ~(t > 0)
    zmax = z.amax(-1, keepdim=True)
    empty = zmax[:, 0] == -math.inf
    d = (z - torch.where(empty[:, None], torch.zeros_like(zmax), zmax)) \
        / torch.where(greedy, torch.ones_like(t), t)[:, None]
    val, idx = torch.sort(z, dim=-1, descending=True, stable=True)
    e = torch.exp(torch.gather(d, 1, idx))
    rank = torch.arange(V, device=DEV)[None]
    keep = rank < torch.where(top_k > 0, top_k, torch.full_like(top_k, V))[:, None]
    e_k = torch.where(keep, e, torch.zeros_like(e))
    before = torch.cumsum(e_k, -1) - e_k
    goal = top_p * e_k.sum(-1)
    keep &= ((before < goal[:, None]) & (top_p > 0)[:, None]) | (top_p >= 1)[:, None]
    keep &= e >= min_p[:, None]
    keep[:, 0] = True
    keep &= rank < torch.where(greedy, torch.ones_like(top_k), torch.full_like(top_k, V))[:, None]
    keep &= val > -math.inf
    kept = torch.zeros_like(keep).scatter_(1, idx, keep)
    key = torch.where(kept, d - torch.log(-torch.log(u)), torch.full_like(d, -math.inf))
    best = key.amax(-1, keepdim=True)
    ids = torch.arange(V, device=DEV)[None].expand(B, V)
    token = torch.where(kept & (key == best), ids, torch.full_like(ids, V)).amin(-1)
    token = torch.where(empty, torch.full_like(token, -1), token)
    lse = torch.log(torch.exp(d).sum(-1))
    logprob = torch.gather(d, 1, token.clamp(min=0)[:, None])[:, 0] - lse
    return token.int(), torch.where(empty, torch.full_like(logprob, -math.inf), logprob)


def run(state):
    st, c = state, state["case"]
    if c["kind"] == "sample":
        if own:
            from paper_2607_16248_gb300 import kvq
            o = kvq.kvq_sample(st["logits"], st["noise"], st["temperature"], st["top_k"],
                               st["top_p"], st["min_p"], outputs=st["outputs"])
            return [o["token"], o["logprob"]]
        return list(_plain_sample(st["logits"], st["noise"], st["temperature"], st["top_k"],
                                  st["top_p"], st["min_p"]))
    if own:
        from paper_2607_16248_gb300 import kvq
        return kvq.kvq_chunk_attn(st["cache"], st["q"], out=st["out"], window=c["window"],
                                  sinks=c["sinks"], workspace=st["workspace"])
    return torch.stack([_plain_sequence(c, s, st["q"][b]) for b, s in enumerate(st["seqs"])])


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------


def _ceil_to(x, bits, least):
    """x >= 0 (fp64) rounded up to `bits` significant bits, quantum >= 2^least."""
    _, e = torch.frexp(x)
    q = torch.clamp(e.to(torch.int64) - bits, min=least)
    step = ((q + 1023) << 52).view(torch.float64)      # 2^q
    return torch.ceil(x / step) * step


def _restored(x, bits, dim):
    """The values that a quantized tensor stands for, groups of 32 along dim."""
    y = x.double().unflatten(dim, (-1, G))
    g = dim + 1
    lo, hi = y.amin(g, keepdim=True), y.amax(g, keepdim=True)
    scale = _ceil_to(_ceil_to(_ceil_to(hi - lo, 24, -149) / (2 ** bits - 1), 24, -149), 11, -24)
    ratio = ((y - lo).float().double() / torch.where(scale > 0, scale, torch.ones_like(scale)))
    code = torch.clamp(torch.round(ratio.float().double()), 0, 2 ** bits - 1)
    return (lo + torch.where(scale > 0, scale * code, torch.zeros_like(code))).flatten(dim, g)


def _exact_sequence(c, k, v, q):
    L, n_q = k.shape[1], q.shape[0]
    lq = _packed(L)
    out = torch.zeros(n_q, c["hq"], D, dtype=torch.float64, device=DEV)
    for h in range(c["hq"]):
        hk = h // (c["hq"] // c["hkv"])
        if h % (c["hq"] // c["hkv"]) == 0:
            kk = torch.cat([_restored(k[hk, :lq], c["bk"], 0), k[hk, lq:].double()])
            vv = torch.cat([_restored(v[hk, :lq], c["bv"], 1), v[hk, lq:].double()])
        for t0 in range(max(0, n_q - L), n_q, 1024):
            t1 = min(n_q, t0 + 1024)
            row = torch.arange(L - n_q + t0, L - n_q + t1, device=DEV)
            end = int(row[-1]) + 1
            begin = max(0, int(row[0]) + 1 - c["window"]) if c["window"] else 0
            cols = torch.arange(end, device=DEV)
            cols = cols[(cols >= begin) | (cols < c["sinks"])]
            seen = cols[None] <= row[:, None]
            if c["window"]:
                seen &= (cols[None] > row[:, None] - c["window"]) | (cols[None] < c["sinks"])
            s = q[t0:t1, h].double() @ kk[cols].T / math.sqrt(D)
            w = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
            out[t0:t1, h] = w @ vv[cols]
    return out


def exact(case, seed):
    c = case
    if c["kind"] == "sample":
        z, u = _sample_inputs(c, seed)
        t, top_k, top_p, min_p = (x.double() for x in _settings(c))
        tokens, logs = [], []
        for b in range(c["batch"]):
            row = z[b].double()
            m = row.max()
            T = float(t[b]) if t[b] > 0 else 1.0
            y = (row - m) / T
            logp = y - torch.logsumexp(y, 0)
            order = torch.argsort(row, descending=True, stable=True)
            if not t[b] > 0:
                order = order[:1]
            if top_k[b] > 0:
                order = order[:int(top_k[b])]
            if top_p[b] < 1:
                p = torch.exp(y[order])
                n = int((torch.cumsum(p, 0) - p < top_p[b] * p.sum()).sum()) if top_p[b] > 0 else 1
                order = order[:max(1, n)]
            order = order[(torch.exp(y[order]) >= min_p[b]) & (row[order] > -math.inf)]
            order = torch.sort(order)[0]
            key = y[order] - torch.log(-torch.log(u[b].double()[order]))
            tok = int(order[torch.nonzero(key == key.max())[0, 0]])
            tokens.append(tok)
            logs.append(float(logp[tok]))
        return [torch.tensor(tokens, dtype=torch.int32), torch.tensor(logs, dtype=torch.float64)]
    q = torch.randn(c["batch"], c["n_q"], c["hq"], D, generator=_gen(seed, 0), device=DEV).half()
    if work(c)["flops"] > 6e12:
        return None
    return torch.stack([_exact_sequence(c, *_kv(c, L, _gen(seed, 2 + b)), q[b])
                        for b, L in enumerate(_lengths(c))])
