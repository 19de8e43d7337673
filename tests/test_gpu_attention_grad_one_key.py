"""Rows that see one key: the weight is one whatever the score, dp = delta, so ds, and with it the row's dq and its part of dk, are
zero by definition.  Held to exactly zero: the bound is no rounding, at any size of the scores.
"""
import pytest
import torch

import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import BF16, F16, UNIT, _rand, _starts
from test_gpu_attention_grad import _grad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("gain", [2.0, 60.0])
@pytest.mark.parametrize("heads,kv,dim,causal", [(32, 32, 128, True), (64, 8, 128, False), (14, 2, 80, True), (12, 4, 64, True), (2, 1, 8, False)])
def test_sequences_of_one_token(heads, kv, dim, causal, gain, dtype):
    rng = synth.child_rng(350, heads, dim)
    for lens in ([1], [1, 0, 1, 1, 0], [1] * 150):
        print(heads, kv, dim, causal, gain, dtype, len(lens), flush=True)
        t, g = sum(lens), heads // kv
        q, k, v, go = (_rand(rng, t, x, dim, dtype=dtype, gain=s) for x, s in ((heads, gain), (kv, 1.0), (kv, 1.0), (heads, 0.01)))
        dq, dk, dv = _grad(go, q, k, v, lens, lens, causal, dim ** -0.5)
        assert not dq.any() and not dk.any(), (len(lens), float(dq.abs().max()), float(dk.abs().max()))
        # dv = the sum of do over the heads that share it: one rounding of each weight, one of the result
        x = go.double().view(t, kv, g, dim)
        assert ((dv.double() - x.sum(2)).abs() <= 2 * UNIT[dtype] * x.abs().sum(2) + 2.0 ** -24).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_first_rows_and_single_keys(dtype):
    """First rows of causal sequences; queries that share a single key; rows at the end of the queries, where keys are fewer."""
    rng = synth.child_rng(351)
    lens = [300, 1, 77, 0, 130, 2]
    q, k, v, go = (_rand(rng, sum(lens), x, 128, dtype=dtype, gain=s) for x, s in ((8, 2.0), (2, 1.0), (2, 1.0), (8, 0.01)))
    dq, _, _ = _grad(go, q, k, v, lens, lens, True, 0.1)
    firsts = [sum(lens[:i]) for i, n in enumerate(lens) if n]
    assert not dq[firsts].any() and all(dq[i + 1].any() for i in firsts if i != 300)
    lens_q, lens_k = [200, 3, 65], [1, 1, 1]
    q, go, k, v = (_rand(rng, n, x, 64, dtype=dtype) for n, x in ((268, 4), (268, 4), (3, 2), (3, 2)))
    for causal in (True, False):
        dq, dk, dv = _grad(go, q, k, v, lens_q, lens_k, causal, 0.1)
        assert not dq.any() and not dk.any() and dv.any()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_not_finite_comes_through(dtype):
    """0 * inf: an infinite value makes dp - delta, and with it both gradients, NaN."""
    rng = synth.child_rng(352)
    q, k, v, go = (_rand(rng, 3, x, 64, dtype=dtype) for x in (2, 2, 2, 2))
    v[1, 0, 5] = float("inf")
    dq, dk, _ = _grad(go, q, k, v, [1, 1, 1], [1, 1, 1], True, 0.1)
    assert torch.isnan(dq[1, 0]).all() and torch.isnan(dk[1, 0]).all()
    dq[1, 0], dk[1, 0] = 0, 0
    assert not dq.any() and not dk.any()
