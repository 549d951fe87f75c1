"""kvq_adjust_logits against the 64-bit oracle.  Every part is one or two fp32 operations
on a logit, a penalty or a bias: six roundings of 2^-24 of the largest magnitude met."""

import numpy as np
import pytest
import torch

from oracle import block8
from paper_2607_16248_gb300 import kvq

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def starts(lists):
    return torch.tensor(np.concatenate([[0], np.cumsum([len(x) for x in lists])]),
                        dtype=torch.int32, device="cuda")


def flat(lists, dtype=torch.int32):
    return torch.tensor([x for y in lists for x in y], dtype=dtype, device="cuda")


def packed(allowed):
    """bool [n, V] -> int32 [n, ceil(V / 32)]."""
    n, V = allowed.shape
    bits = np.zeros((n, (V + 31) // 32 * 32), dtype=np.uint64)
    bits[:, :V] = allowed
    words = (bits.reshape(n, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1)
    return torch.from_numpy(words.astype(np.uint32).view(np.int32)).cuda()


def check(got, want, size):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    ok = np.isfinite(want)
    assert (np.abs(got[ok] - want[ok]) <= 6 * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 31), (2, 1000), (5, 8193), (2, 20011)])
def test_everything(kvq_lib, dtype, rows, V):
    rng = np.random.default_rng(rows * V)
    z = torch.tensor(rng.normal(0, 3, (rows, V + 3)), device="cuda").to(TYPES[dtype])[:, :V]
    hist = [rng.integers(-1, V + 2, rng.integers(0, 400)).tolist() for _ in range(rows)]
    prompt = [int(rng.integers(0, len(h) + 2)) for h in hist]
    bias = [[(int(i), float(np.float32(x))) for i, x in zip(
        rng.integers(-1, V + 1, 40), rng.normal(0, 5, 40))] for _ in range(rows)]
    rep = np.float32(rng.uniform(0.7, 1.6, rows))
    freq, pres = np.float32(rng.normal(0, 1, rows)), np.float32(rng.normal(0, 1, rows))
    allowed = rng.random((rows + 1, V)) < 0.6
    which = rng.integers(-1, rows + 1, rows)
    which[0] = -1

    def dev(x, dt=torch.float32):
        return torch.tensor(x, dtype=dt, device="cuda")

    got = kvq.kvq_adjust_logits(
        z, history=flat(hist), history_starts=starts(hist), prompt_lengths=dev(prompt, torch.int32),
        repetition=dev(rep), frequency=dev(freq), presence=dev(pres),
        bias_ids=flat([[i for i, _ in x] for x in bias]),
        bias_values=flat([[v for _, v in x] for x in bias], torch.float32),
        bias_starts=starts(bias), mask=packed(allowed), mask_rows=dev(which, torch.int32))
    zz = z.double().cpu().numpy()
    want = np.stack([block8.adjust(zz[b], hist[b], prompt[b], rep[b], freq[b], pres[b], bias[b],
                                   allowed[which[b]] if which[b] >= 0 else None)
                     for b in range(rows)])
    check(got, want, np.abs(zz).max() * 1.6 + 400 * np.abs(freq).max() + 25)


def test_parts_alone_and_in_place(kvq_lib):
    rng = np.random.default_rng(3)
    V = 9000
    z = torch.tensor(rng.normal(0, 3, (2, V)), dtype=torch.float32, device="cuda")
    hist = [[5, 5, 8999], []]
    out = kvq.kvq_adjust_logits(z, history=flat(hist), history_starts=starts(hist),
                                presence=torch.ones(2, device="cuda"))
    want = z.clone()
    want[0, 5] -= 1
    want[0, 8999] -= 1
    assert torch.equal(out, want)
    allowed = np.ones((1, V), dtype=bool)
    allowed[0, ::7] = False
    same = kvq.kvq_adjust_logits(out, out=out, mask=packed(allowed),
                                 mask_rows=torch.tensor([0, 0], dtype=torch.int32, device="cuda"))
    assert same is out
    want[:, ::7] = -np.inf
    assert torch.equal(out, want)
    # an empty history, a row of nothing
    nothing = packed(np.zeros((2, V), dtype=bool))
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    got = kvq.kvq_adjust_logits(z, history=empty, mask=nothing,
                                history_starts=torch.zeros(3, dtype=torch.int32, device="cuda"),
                                repetition=torch.full((2,), 1.3, device="cuda"))
    assert torch.isneginf(got).all()
    assert kvq.kvq_sample(got)["token"].tolist() == [-1, -1]


def test_infinities_and_bad_lists(kvq_lib):
    z = torch.tensor([[float("inf"), float("-inf"), float("nan"), 2.0, -2.0, 1.0]], device="cuda")
    hist = [[0, 1, 2, 3, 4]]
    got = kvq.kvq_adjust_logits(z, history=flat(hist), history_starts=starts(hist),
                                repetition=torch.tensor([2.0], device="cuda"))[0].tolist()
    assert got[0] == float("inf") and got[1] == float("-inf") and got[2] != got[2]
    assert got[3:] == [1.0, -4.0, 1.0]
    for bad in ([3, 1], [-1, 4], [0, 6]):
        got = kvq.kvq_adjust_logits(z, history=flat(hist), presence=torch.ones(1, device="cuda"),
                                    history_starts=torch.tensor(bad, dtype=torch.int32,
                                                                device="cuda"))
        assert torch.equal(got[:, 3:], z[:, 3:])
    for rep in (0.0, -1.0, float("nan")):
        got = kvq.kvq_adjust_logits(z, history=flat(hist), history_starts=starts(hist),
                                    repetition=torch.tensor([rep], device="cuda"))
        assert torch.equal(got[:, 3:], z[:, 3:])


@pytest.mark.parametrize("dtype,V,pad", [("bf16", 140001, 0), ("fp16", 140003, 5), ("fp32", 140002, 1)])
def test_large_calls(kvq_lib, dtype, V, pad):
    """More than 2^23 logits with short lists: streamed, then patched.  One row names more
    tokens than are counted at a time, one none, one every token of a stretch."""
    rows, rng = 61, np.random.default_rng(V)
    z = torch.randn(rows, V + pad, device="cuda",
                    generator=torch.Generator("cuda").manual_seed(V)).to(TYPES[dtype])[:, :V]
    hist = [rng.integers(0, V, 100).tolist() for _ in range(rows)]
    hist[3] = (rng.random(20000) ** 3 * V).astype(int).tolist()
    hist[4] = []
    hist[5] = list(range(100, 5300)) * 2 + [V - 1, 0]
    prompt = [len(h) // 2 for h in hist]
    bias = [[(int(i), float(np.float32(x))) for i, x in zip(rng.integers(0, V, 30),
                                                            rng.normal(0, 5, 30))]
            for _ in range(rows)]
    bias[4] = [(7, 1.0), (7, 2.0), (V - 1, 3.0)]
    allowed = rng.random((2, V)) < 0.5
    which = [-1, 0, 1] + [i % 2 for i in range(rows - 3)]
    args = dict(history=flat(hist), history_starts=starts(hist),
                prompt_lengths=torch.tensor(prompt, dtype=torch.int32, device="cuda"),
                repetition=torch.full((rows,), 1.25, device="cuda"),
                frequency=torch.full((rows,), 0.5, device="cuda"),
                presence=torch.full((rows,), 0.25, device="cuda"),
                bias_ids=flat([[i for i, _ in x] for x in bias]),
                bias_values=flat([[v for _, v in x] for x in bias], torch.float32),
                bias_starts=starts(bias))
    masked = dict(args, mask=packed(allowed),
                  mask_rows=torch.tensor(which, dtype=torch.int32, device="cuda"))
    out = torch.full((rows, V + 2), 7.0, device="cuda")
    got = kvq.kvq_adjust_logits(z, out=out[:, 1:V + 1], **masked)
    zz = z.double().cpu().numpy()
    want = np.stack([block8.adjust(zz[b], hist[b], prompt[b], 1.25, 0.5, 0.25, bias[b],
                                   allowed[which[b]] if which[b] >= 0 else None)
                     for b in range(rows)])
    check(got, want, np.abs(zz).max() * 1.6 + 20 + 0.5 * 400)
    assert (out[:, 0] == 7.0).all() and (out[:, V + 1] == 7.0).all()
    assert torch.equal(got, kvq.kvq_adjust_logits(z, **masked))
    if dtype == "fp32":     # in its place: with a mask, and with nothing to stream
        for kw in (masked, args):
            want = kvq.kvq_adjust_logits(z, **kw)
            same = z.clone()
            kvq.kvq_adjust_logits(same, out=same, **kw)
            assert torch.equal(same, want)


def test_a_vocabulary_of_several_slices(kvq_lib):
    rng = np.random.default_rng(8)
    V = (1 << 23) + 12345
    z = torch.randn(1, V, device="cuda", generator=torch.Generator("cuda").manual_seed(8))
    hist = [rng.integers(0, V, 3000).tolist() + [0, V - 1]]
    got = kvq.kvq_adjust_logits(z, history=flat(hist), history_starts=starts(hist),
                                presence=torch.ones(1, device="cuda"))
    want = z.clone()
    ids = torch.tensor(sorted(set(hist[0])), device="cuda")
    want[0, ids] -= 1.0
    assert torch.equal(got, want)


def test_small_in_place_without_a_mask(kvq_lib):
    z = torch.randn(3, 500, device="cuda")
    hist = [[1, 2, 2], [499], []]
    args = dict(history=flat(hist), history_starts=starts(hist),
                frequency=torch.ones(3, device="cuda"))
    want = kvq.kvq_adjust_logits(z, **args)
    kvq.kvq_adjust_logits(z, out=z, **args)
    assert torch.equal(z, want)
