"""Sampling where much of what may be drawn lies in very many tokens of very small weight: one likely token and a flat tail far below it.

Bound.  A weight w is off by at most (1 + |log2 w|) 2^-23 of itself, and by half a unit: units are 2^-45 up to 2^19 - 1 tokens, 2^-(63 - floor(log2 vocab)) from there on.  A
token's interval of u is a quotient of two sums of weights, the lower at most the upper, so both its ends are off by at most twice the sum of all these errors over the sum of the
weights.  The token that is drawn is one whose interval, by so much larger, holds u.  With top-p the place where it ends is off by as much again, and by the token there.
"""
import numpy as np
import pytest
import torch

import synth
import paper_2602_05367_amd as rb

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
INF = float("inf")


def unit(vocab):
    return 2.0 ** -min(45, 63 - (vocab.bit_length() - 1))


def check(x, tokens, u, top_p=1.0):
    """Rows x on the host in 64 bits."""
    for row, (logits, got, number) in enumerate(zip(x, tokens.tolist(), u)):
        w = np.exp(logits - logits.max())
        with np.errstate(divide="ignore"):
            error = (w * (1 + np.abs(np.log2(w))) * 2.0 ** -23 + unit(w.size) / 2).sum()
        total, off = w.sum(), 2 * error / w.sum()
        kept = w
        if top_p < 1:
            order = np.argsort(-logits, kind="stable")
            before = np.cumsum(w[order]) - w[order]
            assert before[order == got] < (top_p + off) * total, (row, "behind top-p", got)
            n = int((before < top_p * total).sum())
            kept = np.where(np.isin(np.arange(w.size), order[:n]), w, 0.0)
            off = 2 * off + w[order[n - 1]] / total
        ends = np.cumsum(kept)
        ends, low = ends / ends[-1], (ends - kept) / ends[-1]
        assert low[got] - off <= number <= ends[got] + off, (row, got, low[got], ends[got], number, off)


def rows_of(vocab, gaps, at, dtype):
    """One likely token at place `at`, all others `gap` below it; the values that dtype has."""
    x = torch.zeros((len(gaps), vocab), dtype=torch.float32, device="cuda")
    for row, gap in enumerate(gaps):
        x[row, at % vocab] = gap
    return x.to(dtype)


U = [0.25, 0.9, 0.999, 0.9999, 0.99999, 0.999999, 1 - 2.0 ** -23, 1 - 2.0 ** -24]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("vocab,many", [(9, 1), (5003, 1), (32000, 1), (32000, 40), (131071, 1), (131071, 40), (262147, 1), (262147, 40)])
def test_a_flat_tail_far_below(vocab, many, dtype):
    """As one row that several workgroups share, and as many of one workgroup each."""
    gaps = [8.0, 12.5, 16.0, 20.0, 21.25, 21.5, 21.625, 22.0, 23.5, 26.0, 29.0, 31.0, 33.5]
    rng = synth.child_rng(660, vocab)
    for at in (0, vocab // 2, vocab - 1):
        u = np.array([U[i % len(U)] if i % 3 else rng.random() for i in range(len(gaps) * 2)], dtype=np.float32)
        x = rows_of(vocab, [gaps[i // 2] for i in range(len(u))], at, dtype)
        print(vocab, many, dtype, at, flush=True)
        host = x.double().cpu().numpy()
        for part in range(0, len(u), len(u) if many > 1 else 1):
            rows = slice(part, part + (len(u) if many > 1 else 1))
            n = rows.stop - rows.start
            repeat = 7 if many > 1 else 1      # (more rows than half the compute units: one workgroup each)
            got = rb.rb_sample(x[rows].repeat(repeat, 1), torch.from_numpy(np.tile(u[rows], repeat)).cuda())
            torch.cuda.synchronize()
            got = got.view(repeat, n)
            assert (got == got[0]).all()
            check(host[rows], got[0], u[rows].astype(np.float64))


@pytest.mark.parametrize("vocab", [1 << 20, 1 << 22])
def test_the_largest_vocabularies(vocab):
    gaps = [20.0, 21.25, 21.5, 21.625, 23.0, 27.0]
    u = np.array([0.999, 0.9999, 0.999, 0.9975, 0.9999, 0.999999], dtype=np.float32)
    x = rows_of(vocab, gaps, 12345, F32)
    got = [rb.rb_sample(x[i:i + 1], torch.from_numpy(u[i:i + 1]).cuda()) for i in range(len(u))]
    torch.cuda.synchronize()
    check(x.double().cpu().numpy(), torch.cat(got), u.astype(np.float64))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("top_p", [0.999, 0.9999, 0.99999])
def test_a_nucleus_that_ends_in_the_tail(top_p, dtype):
    """The tail's tokens are equal, so those that are left are its first ones."""
    top_p = float(np.float32(top_p))
    for vocab, repeat in ((131071, 1), (131071, 40), (1 << 22, 1)):
        gaps = [float(torch.tensor(g).to(dtype)) for g in (13.0, 17.0, 20.0, 21.5)]
        u = np.array([0.99, 0.999, 0.99995, 1 - 2.0 ** -24], dtype=np.float32)
        x = rows_of(vocab, gaps, 0, dtype)
        print(vocab, repeat, dtype, top_p, flush=True)
        for rows in ([slice(0, 4)] if repeat > 1 else [slice(i, i + 1) for i in range(4)]):
            n = rows.stop - rows.start
            p = torch.full((n * repeat,), top_p, device="cuda")
            got = rb.rb_sample(x[rows].repeat(repeat, 1), torch.from_numpy(np.tile(u[rows], repeat)).cuda(), top_p=p)
            torch.cuda.synchronize()
            check(x[rows].double().cpu().numpy(), got[:n], u[rows].astype(np.float64), top_p)


def test_slopes():
    """Tails that fall off slowly, over all magnitudes that have a weight and beyond them, with the random numbers spread over what lies in the tail."""
    rng = synth.child_rng(661)
    for vocab in (60000, 131071, 400000):
        x = torch.from_numpy(np.linspace(-18.0, -40.0, vocab)[rng.permutation(vocab)].astype(np.float32))[None].cuda()
        x[0, 7] = 0.0
        host = x.double().cpu().numpy()
        w = np.exp(host[0] - host[0].max())
        tail = 1 - 1 / w.sum()
        u = (1 - tail * rng.random(8)).astype(np.float32)
        u = np.minimum(u, np.float32(1 - 2.0 ** -24))
        for number in u:
            got = rb.rb_sample(x, torch.tensor([float(number)], device="cuda"))
            torch.cuda.synchronize()
            check(host, got, [float(number)])


@pytest.mark.parametrize("vocab", [(1 << 19) - 1, 1 << 19, (1 << 22) - 1, 1 << 22])
def test_the_largest_sums(vocab):
    """All logits alike: every sum of weights is as large as it can be, and a whole number of the largest weight, so the token is known exactly."""
    x = torch.full((1, vocab), 3.25, device="cuda")
    for number in (0.0, 0.3, 0.5, 0.99999, 1 - 2.0 ** -24):
        u = torch.tensor([number], device="cuda")
        number = float(np.float32(number))
        for top_k, top_p, temperature in ((0, 1.0, 1.0), (vocab - 5, 1.0, 0.01), (0, 0.75, INF), (vocab // 2, 0.999, 1.0), (7, 1.0, 1.0), (0, 1 - 2.0 ** -24, 1.0)):
            given = {"temperature": torch.tensor([temperature], device="cuda")}
            if top_k:
                given["top_k"] = torch.tensor([top_k], dtype=torch.int32, device="cuda")
            if top_p < 1:
                given["top_p"] = torch.tensor([top_p], device="cuda")
            left = top_k or vocab
            left = -(-int(float(np.float32(top_p)) * 2 ** 24) * left // 2 ** 24) if top_p < 1 else left      # (fp32 numbers from 1/2 on are multiples of 2^-24)
            got = rb.rb_sample(x, u, **given)
            assert int(got) == int(number * 2 ** 149) * left // 2 ** 149, (vocab, number, top_k, top_p, temperature)
