"""Scales at the ends of what is accepted: towards zero every visible key has the same weight, and dv is do's mean over the rows that see it; large scales with small
scores are scores like any others.
"""
import pytest
import torch

import synth
from test_gpu_attention import BF16, F16, _rand, check_prompt
from test_gpu_attention_grad import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("scale", [1e-20, 1e-37, 3e-38, 1e-38, 1e-40, 1e-44])
def test_small(scale, dtype):
    rng = synth.child_rng(390)
    lens = [70, 1, 130]
    q, k, v, go = (_rand(rng, sum(lens), x, 64, dtype=dtype) for x in (4, 2, 2, 4))
    check_prompt(q, k, v, lens, lens, True, scale=scale)
    _, _, dv = check(go, q, k, v, lens, lens, True, scale=scale, label=(scale, dtype))
    assert dv.any()


def test_large():
    """bf16 scores of some 2^-120 times a scale of 2^120 (q and k times 2^-60)."""
    rng = synth.child_rng(391)
    lens = [70, 1, 130]
    q, k, v, go = (_rand(rng, sum(lens), x, 64, dtype=BF16) for x in (4, 2, 2, 4))
    check_prompt(q * 2.0 ** -60, k * 2.0 ** -60, v, lens, lens, True, scale=2.0 ** 117)
    check(go, q * 2.0 ** -60, k * 2.0 ** -60, v, lens, lens, True, scale=2.0 ** 117)
