"""The gradient of attention over packed prompts against the fp64 oracle and against differences.

Bounds, derived from what is rounded (u: the unit of the stored type, 2^-11 or 2^-8): every weight and every score
gradient ds once before the product that uses it, o before it enters delta = do.o, and the result.  With the oracle's
sums over magnitudes, which hold |ds| widened by what a rounded o moves it by, an element is off by at most u |g| + u wide; held to
twice u of both, which leaves room for fp32 sums and exponentials.
"""
import numpy as np
import pytest
import torch

import oracle
import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import BF16, F16, UNIT, _f64, _rand, _sees, _starts

pytestmark = pytest.mark.gpu


def _grad(go, q, k, v, lens_q, lens_k, causal, scale):
    first, first_k = _starts(lens_q), None if list(lens_q) == list(lens_k) else _starts(lens_k)
    o, lse = rb.rb_attn_prompt(q, k, v, first, first_k=first_k, causal=causal, scale=scale, want_lse=True)
    got = rb.rb_attn_prompt_grad(go, q, k, v, o, lse, first, first_k=first_k, causal=causal, scale=scale)
    torch.cuda.synchronize()
    return got


def _reference(go, q, k, v, lens_q, lens_k, causal, scale):
    g = q.shape[1] // k.shape[1]
    GO, Q, K, V = (_f64(x) for x in (go, q, k, v))
    ref, wide = ([np.zeros(x.shape) for x in (q, k, v)] for _ in range(2))
    q0 = k0 = 0
    for n, m in zip(lens_q, lens_k):
        a, b = slice(q0, q0 + n), slice(k0, k0 + m)
        for h in range(q.shape[1] if n and m else 0):
            grads, wides = oracle.attention_grad(GO[a, h], Q[a, h], K[b, h // g], V[b, h // g], _sees(n, m, causal), scale)
            for to, x in ((ref, grads), (wide, wides)):
                to[0][a, h] = x[0]
                to[1][b, h // g] += x[1]
                to[2][b, h // g] += x[2]
        q0, k0 = q0 + n, k0 + m
    return ref, wide


def check(go, q, k, v, lens_q, lens_k, causal, scale=None, label=""):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    got = _grad(go, q, k, v, lens_q, lens_k, causal, scale)
    ref, wide = _reference(go, q, k, v, lens_q, lens_k, causal, scale)
    u = UNIT[q.dtype]
    for name, x, r, w in zip(("dq", "dk", "dv"), got, ref, wide):
        off = np.abs(_f64(x) - r) - (2 * u * (np.abs(r) + w) + 2.0 ** -24)
        assert np.isfinite(_f64(x)).all() and (off.size == 0 or off.max() <= 0), (label, name, float(off.max()), float(np.abs(r).max()))
    return got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv,dim", [(2, 2, 128), (6, 2, 64), (5, 1, 96), (4, 4, 8), (14, 2, 80)])
def test_packed_prompts(heads, kv, dim, causal, dtype):
    for n, lens in enumerate([[1], [2, 1, 3], [63, 64, 65], [0, 127, 0, 128, 129, 0], [300]]):
        rng = synth.child_rng(340, heads, dim, n, causal)
        print(heads, kv, dim, causal, dtype, lens, flush=True)
        t = sum(lens)
        q, k, v, go = (_rand(rng, t, x, dim, dtype=dtype, gain=g) for x, g in ((heads, 2.0), (kv, 1.0), (kv, 1.0), (heads, 0.01)))
        check(go, q, k, v, lens, lens, causal, label=(heads, kv, dim, causal, dtype, lens))


@pytest.mark.parametrize("causal", [True, False])
def test_more_or_fewer_keys_than_queries_and_rows_that_see_nothing(causal):
    rng = synth.child_rng(341, causal)
    lens_q, lens_k = [5, 70, 0, 40, 9, 130], [200, 3, 17, 0, 9, 129]
    q, go, k, v = _rand(rng, sum(lens_q), 4, 64, gain=2.0), _rand(rng, sum(lens_q), 4, 64), _rand(rng, sum(lens_k), 2, 64), _rand(rng, sum(lens_k), 2, 64)
    dq, dk, dv = check(go, q, k, v, lens_q, lens_k, causal)
    assert not dq[75:115].any() and not dk[203:220].any() and not dv[203:220].any()      # no keys; no queries


def test_strided_operands():
    rng = synth.child_rng(342)
    lens, dim = [70, 131], 64
    t = sum(lens)
    x = torch.full((t, 9, dim + 8), float("nan"), dtype=F16, device="cuda")
    x[:, :8, :dim] = _rand(rng, t, 8, dim)
    q, k, v, go = x[:, :4, :dim], x[:, 4:6, :dim], x[:, 6:8, :dim], _rand(rng, t, 4, dim)
    check(go, q, k, v, lens, lens, True)
    check(go, q.transpose(0, 1).contiguous().transpose(0, 1), k[:, :1].expand(-1, 2, -1), v, lens, lens, True)


@pytest.mark.parametrize("gain", [1e-6, 1e-4, 1e3])
def test_small_and_large_gradients_keep_their_bits(gain):
    """fp16 do near the bottom and the top of its range: dk, dq and dv relative to themselves, where they can be stored at all."""
    rng = synth.child_rng(343)
    n, d = 260, 128
    q, k, v = _rand(rng, n, 4, d), _rand(rng, n, 2, d), _rand(rng, n, 2, d)
    go = _rand(rng, n, 4, d, gain=gain)
    check(go, q, k, v, [n], [n], True)
    # rows of very different size: the small ones' dq is no worse
    go = _rand(rng, n, 4, d)
    go[::2] *= 2.0 ** -12
    check(go, q, k, v, [n], [n], False)
    check(go, q, k, (v * 1000).half(), [n], [n], False)


def test_gradient_against_differences():
    """Along random directions: the loss of the 64-bit forward changes by what the gradient says."""
    rng = synth.child_rng(344)
    n, heads, kv, d, scale = 90, 4, 2, 64, 0.11
    q, k, v, go = _rand(rng, n, heads, d), _rand(rng, n, kv, d), _rand(rng, n, kv, d), _rand(rng, n, heads, d)
    got = _grad(go, q, k, v, [n], [n], True, scale)
    base, GO, e = [_f64(x) for x in (q, k, v)], _f64(go), 1e-5

    def loss(x):
        return sum((oracle.attention(x[0][:, h], x[1][:, h // 2], x[2][:, h // 2], _sees(n, n, True), scale)[0] * GO[:, h]).sum() for h in range(heads))

    for i in range(3):
        step = [rng.standard_normal(b.shape) if i == j else np.zeros(b.shape) for j, b in enumerate(base)]
        slope = (loss([b + e * s for b, s in zip(base, step)]) - loss([b - e * s for b, s in zip(base, step)])) / (2 * e)
        # a random sum over many elements, each off by some u of its size
        g = _f64(got[i])
        assert abs(slope - (g * step[i]).sum()) <= 8 * UNIT[F16] * np.sqrt(((g * step[i]) ** 2).sum()), i


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_does_not_take_part_has_no_influence(dim, dtype):
    """Another sequence full of NaN; infinities and NaN in later keys, values and gradients: rows before them stay as they are."""
    rng = synth.child_rng(345, dim)
    lens = [150, 90, 33]
    q, k, v, go = (_rand(rng, sum(lens), h, dim, dtype=dtype) for h in (4, 2, 2, 4))
    clean = _grad(go, q, k, v, lens, lens, True, 0.1)
    bad = [x.clone() for x in (go, q, k, v)]
    for x in bad:
        x[150:240] = float("nan")
    got = _grad(*bad, lens, lens, True, 0.1)
    for g, c in zip(got, clean):
        assert torch.equal(g[:150], c[:150]) and torch.equal(g[240:], c[240:])
    # key and value 145 are seen by rows 145 ..: earlier rows' dq does not know them
    bad_k, bad_v = k.clone(), v.clone()
    bad_k[145], bad_v[145] = float("nan"), float("inf")
    got = _grad(go, q, bad_k, bad_v, lens, lens, True, 0.1)
    assert torch.equal(got[0][:145], clean[0][:145]) and torch.isnan(got[0][145:150]).all()
    # row 20's gradient and query reach the keys up to 20 only
    bad_go, bad_q = go.clone(), q.clone()
    bad_go[20, :, 5] = float("inf")
    got = _grad(bad_go, q, k, v, lens, lens, True, 0.1)
    assert torch.equal(got[2][21:], clean[2][21:]) and torch.equal(got[1][21:], clean[1][21:])
    assert torch.isposinf(got[2][:21, :, 5]).all() and torch.equal(got[2][:21, :, 6:], clean[2][:21, :, 6:]) and not torch.isfinite(got[1][:21]).any()
    bad_q[20] = float("nan")
    got = _grad(go, bad_q, k, v, lens, lens, True, 0.1)
    assert torch.equal(got[2][21:], clean[2][21:]) and torch.equal(got[1][21:], clean[1][21:]) and torch.isnan(got[1][:21]).all()


def test_same_bits_again_and_on_another_stream():
    rng = synth.child_rng(346)
    lens = [400, 77]
    q, k, v, go = (_rand(rng, 477, h, 128) for h in (8, 2, 2, 8))
    want = _grad(go, q, k, v, lens, lens, True, 0.1)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [_grad(go, q, k, v, lens, lens, True, 0.1) for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
