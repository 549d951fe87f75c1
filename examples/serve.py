"""A serving loop on the low-bit cache: a prompt that arrives in chunks, then
single tokens, with a sliding window, sinks and sampled tokens.

Per layer of a chunk: ``kvq_pack`` appends its keys and values, ``kvq_chunk_attn``
attends.  Per step after the prompt: the same for one token (the window keeps a
step's cost constant as the text grows, and pages behind the window are handed
back), then ``DGAP.restore`` corrects the step's logits and ``kvq_sample`` draws
the token.  Queries, keys, values and logits are seeded random numbers (no model
weights ship with this package); everything else is what a model's loop does.

    python examples/serve.py [--prompt 5000] [--chunk 1024] [--steps 64] [--window 2048]
"""

import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))

from paper_2607_16248_gb300 import kvq, synth  # noqa: E402


class Pages:
    """Page sets of one shared pool, handed out and back."""

    def __init__(self, n):
        self.free = list(range(n))

    def take(self, n):
        if n > len(self.free):
            raise RuntimeError("the page pool is empty")
        taken, self.free = self.free[:n], self.free[n:]
        return taken

    def give(self, sets):
        self.free.extend(sets)


class Layer:
    """One attention layer's cache of a single sequence, with the window rule of
    its pages: blocks that no later query can see are unmapped."""

    def __init__(self, cfg, pool_pages, window, sinks):
        self.cfg, self.window, self.sinks = cfg, window, sinks
        self.cache = kvq.QuantKVCache(cfg, n_pages=pool_pages)
        self.pages = Pages(pool_pages)
        self.mapped = {}
        self.length = 0

    def step(self, q, k, v, workspace):
        """Append k, v [1, n_kv_heads, n, 128], attend with q [1, n, n_q_heads, 128]."""
        n = k.shape[2]
        new = list(kvq.blocks_written(self.length, n, self.cfg.residual))
        if new:
            sets = self.pages.take(len(new))
            self.cache.map_blocks(0, new, sets)
            self.mapped.update(zip(new, sets))
        kvq.kvq_pack(self.cache, k, v)
        self.length += n
        out = kvq.kvq_chunk_attn(self.cache, q, window=self.window, sinks=self.sinks,
                                 workspace=workspace)
        if self.window:
            first = max(0, self.length + 1 - self.window) // 32      # of the next query's window
            sink_blocks = (self.sinks + 31) // 32
            gone = [b for b in self.mapped if sink_blocks <= b < first]
            if gone:
                self.cache.map_blocks(0, gone, [-1] * len(gone))
                self.pages.give(self.mapped.pop(b) for b in gone)
        return out


def serve(prompt=5000, chunk=1024, steps=64, window=2048, sinks=4, layers=2, vocab=32000, bits=2,
          seed=1, temperature=0.8, top_k=50, top_p=0.95):
    """Token ids (int32 [steps], on the CPU) and the layers after the last step."""
    dev = "cuda"
    n_q_heads, n_kv_heads = 32, 8
    cfg = kvq.CacheConfig(batch=1, n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, bits_k=bits,
                          bits_v=bits, max_len=(prompt + steps + 31) // 32 * 32)
    # a chunk's blocks come before those it pushes out of the window go
    pool = cfg.max_blocks if not window else min(
        cfg.max_blocks, (window + 2 * chunk + sinks) // 32 + 8)
    stack = [Layer(cfg, pool, window, sinks) for _ in range(layers)]
    workspaces = {n: kvq.chunk_workspace(cfg, n) for n in {min(chunk, prompt), prompt % chunk, 1}
                  if n}
    dgap = kvq.DGAP(synth.dgap_weights(seed, K=32), K=32, tau=0.6)
    dgap_ws = dgap.workspace(1, vocab)
    g = synth.generator(seed, dev)

    def projections(n):
        q = torch.randn(1, n, n_q_heads, 128, generator=g, device=dev).half()
        kv = torch.randn(2, 1, n_kv_heads, n, 128, generator=g, device=dev).half()
        return q, kv[0], kv[1]

    def one(value, dtype=torch.float32):
        return torch.full((1,), value, dtype=dtype, device=dev)

    settings = (one(temperature), one(top_k, torch.int32), one(top_p))
    done = 0
    while done < prompt:
        n = min(chunk, prompt - done)
        for layer in stack:
            layer.step(*projections(n), workspaces[n])
        done += n
    tokens = torch.empty(steps, dtype=torch.int32, device=dev)
    for i in range(steps):
        for layer in stack:
            layer.step(*projections(1), workspaces[1])
        logits = torch.randn(1, vocab, generator=g, device=dev) * 3.0
        dgap.restore(logits, workspace=dgap_ws)
        noise = torch.rand(1, vocab, generator=g, device=dev)
        kvq.kvq_sample(logits, noise, *settings,
                       outputs=dict(token=tokens[i:i + 1], logprob=None))
    return tokens.cpu(), stack


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("prompt", 5000), ("chunk", 1024), ("steps", 64), ("window", 2048)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    ids, stack = serve(a.prompt, a.chunk, a.steps, a.window)
    used = len(stack[0].mapped)
    print(f"{a.prompt} prompt tokens in chunks of {a.chunk}, {a.steps} sampled tokens; "
          f"{used} pages a layer in use for {stack[0].length} tokens")
    print("tokens:", ids.tolist()[:16], "...")
