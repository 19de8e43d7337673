"""One value for all tokens of a head (a token stride of zero), with infinities in it: every row sees them, and zero times infinity of places that are not there
does not turn them into NaN.
"""
import numpy as np
import pytest
import torch

import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import BF16, F16, UNIT, _f64, _rand, _starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
def test_infinities_in_a_broadcast_value(dim, causal, dtype):
    rng = synth.child_rng(430, dim)
    for lens in ([1], [64], [130], [1, 33, 700]):
        t = sum(lens)
        q, k, v = _rand(rng, t, 4, dim, dtype=dtype), _rand(rng, t, 2, dim, dtype=dtype), _rand(rng, 1, 2, dim, dtype=dtype)
        v[0, 0, 3], v[0, 1, dim - 1] = float("inf"), -float("inf")
        for all_of in (v.expand(t, -1, -1), v[:, :, None].expand(1, 2, t, dim)[0].transpose(0, 1)):
            print(dim, causal, dtype, lens, flush=True)
            o = _f64(rb.rb_attn_prompt(q, k, all_of, _starts(lens), causal=causal))
            want = np.broadcast_to(np.repeat(_f64(v), 2, axis=1), o.shape)      # weights add up to one: once the weights, once the result are rounded
            inf = np.isinf(want)
            assert np.array_equal(o[inf], want[inf]) and (np.abs(o[~inf] - want[~inf]) <= 4 * UNIT[dtype] * np.abs(want[~inf])).all()
