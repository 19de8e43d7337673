"""Attention over a cache in 8 bits for every unit that a value may have, 2^-127 among them, by the kernel for few new tokens and by the other.

Bound.  Weights and sums as in test_gpu_attention.py: one rounding of each weight to bf16, one of the result, 2^-8 of the sum of magnitudes each at most.  Where a
weight times its unit is below fp32's normal range, it is also off by half of bf16's smallest step, 2^-134, times the element, over the sum of the weights.
"""
import numpy as np
import pytest
import torch

import oracle
import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import BF16, _f64, _rand, _sees, _starts
from test_gpu_cache8 import E4M3, _ints, empty_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 40])      # rows that see three keys and more
@pytest.mark.parametrize("dim", [64, 128])
def test_every_unit_of_values(dim, new):
    rng = synth.child_rng(690, dim, new)
    length, heads = new + 2, 2
    pages = -(-length // 16)
    k = rng.standard_normal((length, dim))
    codes = torch.from_numpy(rng.integers(0, 0x7f, (length, dim)).astype(np.uint8) | (rng.integers(0, 2, (length, dim)) << 7).astype(np.uint8))
    elements = codes.view(E4M3).double().numpy()
    table, first, now = _ints([list(range(pages))]), _starts([new]), _ints([length])
    cache = empty_cache(pages, 16, 1, dim, BF16)
    at = torch.arange(length)
    held, units = oracle.held_in_8_bits(k, "bf16")
    cache.k.view(torch.uint8)[at // 16, at % 16, 0] = torch.from_numpy(held).float().to(E4M3).view(torch.uint8).cuda()
    cache.k_exp[at // 16, 0, at % 16] = torch.from_numpy(units.astype(np.uint8)).cuda()
    cache.v.view(torch.uint8)[at // 16, at % 16, 0] = codes.cuda()
    K = held * np.exp2(units - 127.0)[:, None]
    q = _rand(rng, new, heads, dim, dtype=BF16)
    for byte in (*range(0, 12), 60, 119, 127, 180, 235):
        cache.v_exp[at // 16, 0, at % 16] = byte
        got = rb.rb_attn_cache8(cache, q, first, now, table)
        torch.cuda.synchronize()
        V = elements * 2.0 ** (byte - 127)
        for h in range(heads):
            sees = _sees(new, length, True)
            ref, _, mag = oracle.attention(_f64(q)[:, h], K, V, sees, dim ** -0.5)
            seen = np.arange(length) < np.asarray(sees)[:, None]
            scores = np.where(seen, _f64(q)[:, h] @ K.T * dim ** -0.5, -np.inf)
            total = np.exp(scores - scores.max(1, keepdims=True)).sum(1)
            tiny = 2.0 ** -134 * (seen.astype(float) @ np.abs(elements)) / total[:, None] + 2.0 ** -134
            off = np.abs(_f64(got[:, h]) - ref)
            assert (off <= 2.0 ** -7 * mag + tiny).all(), (byte, h, off.max(), np.abs(ref).max())
        assert got.any(), byte
