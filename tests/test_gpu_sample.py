"""Sampling against the fp64 oracle, token by token.

Tokens are whole numbers: they are equal or wrong.  The kernel's weights are off by some 2^-22 of themselves, so u would have to lie that near to the edge of a token's
interval for another one to come out; the inputs are seeded, and none of them has such a u.
"""
import numpy as np
import pytest
import torch

import oracle
import synth
import paper_2602_05367_amd as rb

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
INF = float("inf")


def _f32(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.float32).cuda()


def _i32(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def check(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, label=""):
    """Parameters: None, or one per row."""
    u, t, p, m = _f32(u), _f32(temperature), _f32(top_p), _f32(min_p)
    got = rb.rb_sample(logits, u, temperature=t, top_k=_i32(top_k), top_p=p, min_p=m)
    torch.cuda.synchronize()
    x, got = logits.double().cpu().numpy(), got.cpu().numpy()
    of = lambda v, i, default: default if v is None else float(v[i])
    want = [oracle.next_token(x[i], float(u[i]), of(t, i, 1.0), int(of(top_k, i, 0)), of(p, i, 1.0), of(m, i, 0.0)) for i in range(len(x))]
    assert got.tolist() == want, (label, [(i, a, b) for i, (a, b) in enumerate(zip(got.tolist(), want)) if a != b][:5])
    return got


def _logits(rng, rows, vocab, dtype, gain=2.5):
    x = gain * rng.standard_normal((rows, vocab)) + 4 * rng.random((rows, vocab)) ** 8
    return torch.from_numpy(x.astype(np.float32)).to(dtype).cuda()


VOCABS = [1, 2, 7, 63, 64, 65, 511, 513, 1000, 4096, 8191, 32000, 50001, 131071]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("filters", ["none", "temperature", "top_k", "top_p", "min_p", "all"])
def test_against_the_oracle(filters, dtype):
    for vocab in VOCABS:
        rng = synth.child_rng(630, vocab, len(filters))
        rows = 9 if vocab < 40000 else 4
        print(filters, dtype, vocab, flush=True)
        x = _logits(rng, rows, vocab, dtype)
        given = {"temperature": rng.choice([0.2, 0.7, 1.0, 1.7, 20.0], rows), "top_k": rng.choice([1, 2, 3, 40, 300, 5000, 0, 1 << 30], rows),
                 "top_p": rng.choice([0.01, 0.5, 0.9, 0.99, 0.9999, 1.0], rows), "min_p": rng.choice([0.001, 0.02, 0.3, 0.9, 1.0], rows)}
        given = {n: v for n, v in given.items() if filters in (n, "all")}
        check(x, rng.random(rows), **given, label=(filters, dtype, vocab))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_rows_at_any_place(dtype):
    """Rows of a wider tensor, beginning at every element of 16 bytes, with infinities around them."""
    rng = synth.child_rng(631)
    for offset in range(9):
        for vocab in (700, 1023):
            x = torch.full((5, vocab + 17), INF, dtype=dtype, device="cuda")
            x[:, offset:offset + vocab] = _logits(rng, 5, vocab, dtype)
            check(x[:, offset:offset + vocab], rng.random(5), top_p=[0.9] * 5, label=(offset, vocab))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_ties(dtype):
    """Equal logits: the lowest indexes come first, at the borders of top-k and top-p and in greedy rows; more of them than a list holds, too."""
    rng = synth.child_rng(632)
    for vocab in (10, 1000, 5003, 40000):
        rows = 8
        check(torch.zeros((rows, vocab), dtype=dtype, device="cuda"), rng.random(rows), top_k=[1, 2, 3, 7, 0, 9, 5, 8], top_p=[1, 1, 0.5, 0.3, 0.25, 0.9, 1, 0.01],
              temperature=[1, 0.5, 1, 2, 1, 1, 0, 1], label=("all", vocab))
        few = torch.from_numpy(rng.integers(-3, 3, (rows, vocab)).astype(np.float32)).to(dtype).cuda()
        check(few, rng.random(rows), top_k=rng.integers(0, vocab + 2, rows), top_p=rng.choice([0.2, 0.6, 0.95, 1.0], rows), min_p=rng.choice([0.0, 0.04, 0.2], rows), label=("few", vocab))
        signs = few * 0
        signs[:, ::2] = -0.0      # zeros of both signs are equal
        check(signs, rng.random(rows), top_k=[3] * rows, label=("zeros", vocab))


def test_close_logits_in_one_bin():
    """Thousands of different logits that a histogram's bin does not tell apart."""
    rng = synth.child_rng(633)
    for vocab in (900, 3000, 30000):
        x = torch.from_numpy((5 + 1e-3 * rng.standard_normal((6, vocab))).astype(np.float32)).cuda()
        check(x, rng.random(6), top_k=[10, 1, 500, 0, 700, 0], top_p=[1, 1, 1, 0.5, 0.3, 0.9], label=vocab)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_masks_infinities_and_nan(dtype):
    rng = synth.child_rng(634)
    rows, vocab = 12, 3000
    x = _logits(rng, rows, vocab, dtype)
    lowest = float(torch.finfo(dtype).min)
    x[0] = -INF                                   # nothing left
    x[1] = -INF
    x[1, 2999] = -3.0                             # one left, the last
    x[2] = float("nan")
    x[3, ::2], x[3, 1::3] = -INF, float("nan")
    x[4] = lowest
    x[5, 100:] = lowest
    x[6, 7], x[6, 2000] = INF, INF                # the infinite ones alone
    x[7] = INF
    x[8, :] = -INF
    x[8, 5], x[8, 6] = lowest, float("nan")
    x[9, 17] = float(torch.finfo(dtype).max)
    x[10, ::5] = -0.0
    x[11, 0] = -INF
    u = rng.random(rows)
    got = check(x, u)
    assert got[0] == -1 and got[1] == 2999 and got[2] == -1 and got[8] == 5
    check(x, u, top_k=[3] * rows, top_p=[0.8] * rows, min_p=[0.1] * rows, temperature=[0.7] * rows)
    check(x, u, top_p=[0.99] * rows)
    check(x, u, temperature=[0.0] * rows)


def test_random_numbers_and_parameters_at_and_beyond_their_ends():
    rng = synth.child_rng(635)
    x = _logits(rng, 1, 5000, F32).repeat(16, 1)
    u = [0.0, -1.0, float("nan"), 1.0, 2.0, INF, -INF, 1 - 2.0 ** -24, 2.0 ** -149, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5]
    got = rb.rb_sample(x, _f32(u), top_k=_i32([50] * 16))
    row = x[0].double().cpu().numpy()
    kept = np.sort(np.argsort(-row, kind="stable")[:50])
    torch.cuda.synchronize()
    got = got.tolist()
    assert got[:3] == [kept[0]] * 3 and got[3:6] == [kept[-1]] * 3 and got[6] == kept[0] and got[7] == kept[-1] and got[8] == kept[0]
    half = got[9]
    nan = float("nan")
    # NaN: 0 in temperature and min_p, 1 in top_p; top_k outside 1 .. vocab: all; top_p of 0 and less: one; min_p above 1: the largest
    t = rb.rb_sample(x[:8].contiguous(), _f32([0.5] * 8), temperature=_f32([nan, -1, 0, -0.0, 1, 1, 1, 1]), top_k=_i32([50] * 8), top_p=_f32([1, 1, 1, 1, 0, -2, nan, 1]),
                     min_p=_f32([0, 0, 0, 0, 0, 0, nan, 7.0]))
    torch.cuda.synchronize()
    best = int(row.argmax())
    assert t.tolist() == [best] * 6 + [half, best]
    everything = rb.rb_sample(x[:4].contiguous(), _f32([0.5] * 4), top_k=_i32([0, -5, 5000, 5001]))
    torch.cuda.synchronize()
    assert everything.tolist() == [oracle.next_token(row, 0.5)] * 4


def test_temperatures_from_tiny_to_infinite():
    rng = synth.child_rng(636)
    x = _logits(rng, 7, 2000, F32)
    x[6] = torch.linspace(-3e38, 3e38, 2000)
    u = rng.random(7)
    got = rb.rb_sample(x, _f32(u), temperature=_f32([1e-45, 1e-30, 1e-3, 1e4, 3e38, INF, 1e38]))
    torch.cuda.synchronize()
    X, got = x.double().cpu().numpy(), got.tolist()
    assert got[:2] == [int(X[0].argmax()), int(X[1].argmax())] and got[2] == oracle.next_token(X[2], float(np.float32(u[2])), 1e-3)
    low = x[:4].clone()      # logits of the type's lowest value beside others, at temperatures where what lies between overflows in every way
    low[:, ::2] = torch.finfo(F32).min
    cold = [1e-45, 1e-30, 1e-20, 1.0]
    got_low = rb.rb_sample(low, _f32(u[:4]), temperature=_f32(cold))
    torch.cuda.synchronize()
    assert got_low.tolist()[:3] == [int(r.argmax()) for r in low[:3].cpu()] and got_low.tolist()[3] == oracle.next_token(low[3].cpu().numpy(), float(np.float32(u[3])))
    for i in (3, 4, 5):      # all alike, to 1e-3: the token's number is u's share of them
        assert abs(got[i] - u[i] * 2000) < 3
    assert got[6] == oracle.next_token(X[6], float(np.float32(u[6])), float(np.float32(1e38)))


def test_largest_vocabulary_and_long_strides():
    rng = synth.child_rng(637)
    x = torch.from_numpy(rng.standard_normal((2, 1 << 22), dtype=np.float32)).cuda()
    for given in (dict(), dict(top_k=[1000, 100000]), dict(top_p=[0.3, 0.999])):
        check(x, rng.random(2), **given)
    wide = torch.zeros((3, 1 << 30), dtype=F16, device="cuda")[:, :50]      # rows 2 GiB apart
    wide.copy_(_logits(rng, 3, 50, F16))
    check(wide, rng.random(3))


def test_frequencies():
    """Many rows of one distribution: each token comes out as often as its weight says, to five standard deviations."""
    rng = synth.child_rng(638)
    p = np.array([0.5, 0.25, 0.125, 0.0625, 0.0625])
    n = 20000
    x = torch.from_numpy(np.log(p).astype(np.float32)).cuda().repeat(n, 1)
    got = rb.rb_sample(x, _f32(rng.random(n)))
    torch.cuda.synchronize()
    counts = np.bincount(got.cpu().numpy(), minlength=5)
    assert (np.abs(counts - n * p) < 5 * np.sqrt(n * p * (1 - p))).all(), counts


def test_in_a_graph_and_on_another_stream():
    rng = synth.child_rng(639)
    x, u, t = _logits(rng, 6, 32000, BF16), _f32(rng.random(6)), _f32([0.7] * 6)
    k, p = _i32([40, 0, 7, 0, 100, 1]), _f32([0.9, 0.95, 1.0, 0.5, 0.3, 1.0])
    tokens = torch.zeros(6, dtype=torch.int32, device="cuda")
    rb.rb_sample(x, u, temperature=t, top_k=k, top_p=p)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        rb.rb_sample(x, u, temperature=t, top_k=k, top_p=p, tokens=tokens)
    for _ in range(4):
        x.copy_(_logits(rng, 6, 32000, BF16))
        u.copy_(_f32(rng.random(6)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = check(x, u.cpu().numpy(), temperature=[0.7] * 6, top_k=k.tolist(), top_p=p.cpu().numpy())
        assert tokens.tolist() == want.tolist()
