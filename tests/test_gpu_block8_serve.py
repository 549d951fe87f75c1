"""The operators together, as a serving loop uses them: a ragged batch of prompts in chunks and
single tokens on two layers' caches that share one block table, adjusted logits, sampled
tokens; then drafts, some of which are dropped."""

import numpy as np
import pytest
import torch

from oracle import block8
from paper_2607_16248_gb300 import kvq, synth

pytestmark = pytest.mark.gpu

HQ, HKV, V = 8, 2, 3001


class Loop:
    def __init__(self, seed):
        self.g = torch.Generator().manual_seed(seed)
        self.cfg = kvq.Block8Config(3, HQ, HKV, 512, torch.bfloat16)
        self.table = torch.full((3, 16), -1, dtype=torch.int32, device="cuda")
        self.layers = [kvq.Block8Cache(self.cfg, n_pages=48, block_table=self.table)
                       for _ in range(2)]
        self.free = torch.randperm(48, generator=self.g).tolist()
        self.mapped, self.lengths = [0, 0, 0], [0, 0, 0]
        self.text, self.prompt = [[], [], []], [0, 0, 0]
        self.seqs = [[[[block8.Sequence() for _ in range(2)] for _ in range(HKV)]
                      for _ in range(3)] for _ in range(2)]
        angle = torch.arange(512)[:, None] / 10000.0 ** (torch.arange(64) / 64)
        self.cos, self.sin = angle.cos(), angle.sin()
        self.ws = kvq.block8_workspace(self.cfg, 200)

    def step(self, counts, max_new, compare):
        """One forward of counts[b] new tokens; the last layer's outputs."""
        dev = dict(dtype=torch.int32, device="cuda")
        for b, n in enumerate(counts):
            self.lengths[b] += n
            need = self.lengths[b] // 32
            if need > self.mapped[b]:
                self.layers[0].map_blocks(b, range(self.mapped[b], need),
                                          [self.free.pop() for _ in range(need - self.mapped[b])])
                self.mapped[b] = need
        at = np.concatenate([[0], np.cumsum(counts)])
        starts, lengths = torch.tensor(at, **dev), torch.tensor(self.lengths, **dev)
        for i, cache in enumerate(self.layers):
            qkv = torch.randn(int(at[-1]), HQ + 2 * HKV, 128, generator=self.g).bfloat16()
            q, k, v = qkv.cuda().split([HQ, HKV, HKV], 1)
            q = kvq.kvq_block8_append(cache, k, v, lengths, starts=starts, q=q,
                                      cos=self.cos.cuda(), sin=self.sin.cuda())
            out = kvq.kvq_block8_attn(cache, q, lengths, starts=starts, max_new=max_new,
                                      workspace=self.ws)
            if compare:
                self.compare(i, qkv, q, out, at, counts)
        return out

    def compare(self, i, qkv, q, out, at, counts):
        x, got, qr = (t.detach().double().cpu().numpy() for t in (qkv, out, q))
        gq = HQ // HKV
        for b, n in enumerate(counts):
            rows = slice(int(at[b]), int(at[b + 1]))
            pos = np.arange(self.lengths[b] - n, self.lengths[b])
            keys = block8.rotate(x[rows, HQ:HQ + HKV], self.cos.numpy()[pos],
                                 self.sin.numpy()[pos], False)
            for h in range(HKV):
                k, v = self.seqs[i][b][h]
                k.append(block8.to_type(keys[:, h], "bf16"), self.lengths[b])
                v.append(x[rows, HQ + HKV + h], self.lengths[b])
                heads = slice(h * gq, (h + 1) * gq)
                want, size = block8.attend(qr[rows, heads], k.seen(), v.seen())
                tol = (2.0 ** -11 + 2.0 ** -14) * size + 2.0 ** -8 * np.abs(want) + 2.0 ** -25
                assert (np.abs(got[rows, heads] - want) <= tol).all(), (i, b, h)

    def sample(self, out):
        """The next token of each sequence from its last row's outputs (a fixed projection)."""
        g = torch.Generator().manual_seed(99)
        head = torch.randn(HQ * 128, V, generator=g).bfloat16().cuda() * 0.2
        logits = out.reshape(3, -1) @ head
        hist = [t for text in self.text for t in text]
        counts = np.concatenate([[0], np.cumsum([len(t) for t in self.text])])
        dev = dict(dtype=torch.int32, device="cuda")
        mask = torch.full((1, (V + 31) // 32), 0x55555555, **dev)     # even tokens alone
        z = kvq.kvq_adjust_logits(
            logits, history=torch.tensor(hist, **dev), history_starts=torch.tensor(counts, **dev),
            prompt_lengths=torch.tensor(self.prompt, **dev),
            repetition=torch.full((3,), 1.2, device="cuda"),
            presence=torch.full((3,), 0.5, device="cuda"), mask=mask,
            mask_rows=torch.tensor([0, -1, 0], **dev))
        for b in range(3):
            allowed = np.arange(V) % 2 == 0 if b != 1 else None
            want = block8.adjust(logits[b].double().cpu().numpy(), self.text[b], self.prompt[b],
                                 np.float32(1.2), 0.0, 0.5, allowed=allowed)
            got = z[b].double().cpu().numpy()
            assert np.array_equal(np.isinf(got), np.isinf(want))
            ok = np.isfinite(want)
            bound = 6 * 2.0 ** -24 * (np.abs(want[ok]).max() + 1)
            assert (np.abs(got[ok] - want[ok]) <= bound).all()
        u = torch.rand(3, V, generator=self.g).cuda()
        token = kvq.kvq_sample(z, u, torch.full((3,), 0.9, device="cuda"))["token"].tolist()
        assert token[0] % 2 == 0 and token[2] % 2 == 0
        for b in range(3):
            self.text[b].append(token[b])
        return token


def run(compare):
    loop = Loop(5)
    tokens = []
    for b in range(3):
        loop.text[b] = torch.randint(0, V, (40,), generator=loop.g).tolist()
        loop.prompt[b] = 40
    # prompts of different lengths, chunks beside single tokens
    for counts in ([130, 0, 20], [1, 170, 1], [1, 33, 1]):
        out = loop.step(counts, 200, compare)
    for _ in range(12):
        out = loop.step([1, 1, 1], 1, compare)
        tokens.append(loop.sample(out))
    # four drafts each, of which one, none and three are kept
    before = list(loop.lengths)
    loop.step([4, 4, 4], 4, compare)
    for b, kept in enumerate((1, 0, 3)):
        loop.lengths[b] = before[b] + kept
    out = loop.step([1, 1, 1], 1, compare)
    tokens.append(loop.sample(out))
    assert all(cache.flags() == 0 for cache in loop.layers)
    return tokens, out


def test_serving_loop(kvq_lib):
    tokens, out = run(True)
    again, other = run(False)
    assert tokens == again and torch.equal(out, other)
    assert synth.HEAD_DIM == 128
