"""Calls without any keys, whose tensors have no memory: results and gradients of zero, a log-sum of minus infinity."""
import pytest
import torch

import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import BF16, F16, _rand, _starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 64), (2, 2, 128)])
def test_no_keys(heads, kv, dim, causal, dtype):
    rng = synth.child_rng(400, heads)
    lens = [7, 0, 300]
    q, go = (_rand(rng, sum(lens), heads, dim, dtype=dtype) for _ in range(2))
    none = _rand(rng, 5, kv, dim, dtype=dtype)
    first, first_k = _starts(lens), _starts([0, 0, 0])
    for k, v in ((none[:0], none[5:]), (torch.empty((0, kv, dim), dtype=dtype, device="cuda"),) * 2):
        o, lse = rb.rb_attn_prompt(q, k, v, first, first_k=first_k, causal=causal, want_lse=True)
        dq, dk, dv = rb.rb_attn_prompt_grad(go, q, k, v, o, lse, first, first_k=first_k, causal=causal)
        torch.cuda.synchronize()
        assert o.shape == q.shape and not o.any() and torch.isneginf(lse).all()
        assert dq.shape == q.shape and not dq.any() and dk.shape == k.shape and dv.shape == v.shape
