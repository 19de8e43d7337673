"""Gradients of very different size in one call, finite ones: what a row or a key does not see leaves no trace, and what it does see together with
something larger is off by no more than the bounds say (those of test_gpu_attention_grad: two units in the last place of the sums over magnitudes, which hold
only what takes part).
"""
import numpy as np
import pytest
import torch

import synth
from test_gpu_attention import BF16, F16, UNIT, _f64, _rand
from test_gpu_attention_grad import _grad, _reference, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 128), (4, 4, 64), (8, 1, 80)])
def test_large_neighbours_leave_the_bits_as_they_are(heads, kv, dim, causal, dtype):
    """Sequences before and after, in the same blocks of 64 tokens, with do and v of 6e4."""
    rng = synth.child_rng(360, heads, dim)
    lens, a, b = [70, 200, 41], 70, 270
    q, k, v, go = (_rand(rng, sum(lens), x, dim, dtype=dtype, gain=s) for x, s in ((heads, 2.0), (kv, 1.0), (kv, 1.0), (heads, 1e-4)))
    want = _grad(go, q, k, v, lens, lens, causal, dim ** -0.5)
    for name, x in (("go", go), ("v", v), ("q", q), ("k", k)):
        x[:a], x[b:] = x[:a].sign() * 6e4, x[b:].sign() * 6e4
        print(heads, kv, dim, causal, dtype, name, flush=True)
        if name in ("go", "v"):      # (scores stay what they are)
            got = _grad(go, q, k, v, lens, lens, causal, dim ** -0.5)
            assert all(torch.equal(g[a:b], w[a:b]) for g, w in zip(got, want)), name


@pytest.mark.parametrize("power", [14, 16])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_large_early_row(dtype, power):
    """Row 0 is seen by key 0 alone: every later key's gradients keep their bits, and all are within their bounds."""
    rng = synth.child_rng(361)
    n = 1000
    q, k, v, go = (_rand(rng, n, x, 128, dtype=dtype, gain=s) for x, s in ((4, 1.0), (2, 1.0), (2, 1.0), (4, 0.1)))
    want = _grad(go, q, k, v, [n], [n], True, 128 ** -0.5)
    go[0] *= 2.0 ** power
    assert torch.isfinite(go).all()
    got = check(go, q, k, v, [n], [n], True, label=(dtype, power))
    assert torch.equal(got[0][1:], want[0][1:]) and torch.equal(got[1][1:], want[1][1:]) and torch.equal(got[2][1:], want[2][1:])


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_large_last_value(dtype):
    """The last value is seen by the last row alone: all other rows' dq keep their bits."""
    rng = synth.child_rng(362)
    n = 1000
    q, k, v, go = (_rand(rng, n, x, 128, dtype=dtype, gain=s) for x, s in ((4, 1.0), (2, 1.0), (2, 1.0), (4, 0.1)))
    want = _grad(go, q, k, v, [n], [n], True, 128 ** -0.5)
    v[-1] *= 2.0 ** 13
    got = check(go, q, k, v, [n], [n], True, label=dtype)
    assert torch.equal(got[0][:-1], want[0][:-1])


@pytest.mark.parametrize("causal", [True, False])
def test_rows_and_keys_of_every_size(causal):
    """fp16: do over 2^-16 .. 2^12 and v over 2^-10 .. 2^10, in every order, growing and falling along the sequence and at random."""
    rng = synth.child_rng(363, causal)
    n, d = 300, 64
    along = torch.linspace(0, 1, n, dtype=torch.float64)
    places = [along, 1 - along, torch.from_numpy(rng.permutation(n)).double() / (n - 1)]
    q, k, v, go = (_rand(rng, n, x, d) for x in (4, 2, 2, 4))
    for i, a in enumerate(places):
        for j, b in enumerate(places):
            big_go = (go.double() * (2.0 ** (28 * a - 16).cuda())[:, None, None]).half()
            big_v = (v.double() * (2.0 ** (20 * b - 10).cuda())[:, None, None]).half()
            got = _grad(big_go, q, k, big_v, [n], [n], causal, d ** -0.5)
            ref, wide = _reference(big_go, q, k, big_v, [n], [n], causal, d ** -0.5)
            for name, x, r, w in zip(("dq", "dk", "dv"), got, ref, wide):
                x, bound = _f64(x), 2 * UNIT[F16] * (np.abs(r) + w) + 2.0 ** -24
                # some are beyond what fp16 holds: infinite where that is beyond doubt, of the right sign
                beyond, inside = np.abs(r) - bound >= 65520, np.abs(r) + bound < 65520
                assert np.array_equal(x[beyond], np.sign(r[beyond]) * np.inf), (i, j, name)
                assert np.isfinite(x[inside]).all() and (np.abs(x - r)[inside] <= bound[inside]).all(), (i, j, name)
