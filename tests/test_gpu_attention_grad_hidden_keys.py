"""Keys of minus infinity, which every row sees with a weight of zero: their dk and dv are zero, and the other keys' are those without them, however
many rows there are.
"""
import pytest
import torch

import synth
from test_gpu_attention import BF16, F16, UNIT, _f64, _rand
from test_gpu_attention_grad import _grad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [1, 31, 64, 70, 129])
def test_keys_without_weight(n, causal, dtype):
    rng = synth.child_rng(440, n)
    m = n + 40
    q, go = _rand(rng, n, 4, 64, dtype=dtype).abs(), _rand(rng, n, 4, 64, dtype=dtype)
    k, v = _rand(rng, m, 2, 64, dtype=dtype), _rand(rng, m, 2, 64, dtype=dtype)
    hidden = [3, 10, 39]      # (seen by every row, causal or not)
    k[hidden] = -float("inf")
    _, dk, dv = _grad(go, q, k, v, [n], [m], causal, 0.1)
    assert not dk[hidden].any() and not dv[hidden].any()
    kept = [i for i in range(m) if i not in hidden]
    _, want_k, want_v = _grad(go, q, k[kept], v[kept], [n], [m - 3], causal, 0.1)
    # (the same terms in another order, and by different lse)
    for got, want in ((dk[kept], want_k), (dv[kept], want_v)):
        assert (got.double() - want.double()).abs().max() <= 4 * UNIT[dtype] * float(want.double().abs().max())
