"""A workspace sized for the largest call of a program serves its smaller ones, and nothing behind its end is written."""
import ctypes

import pytest
import torch

import synth
import paper_2602_05367_amd as rb
from test_attention_workspace import HEADS, test_gradient as gradient_sizes, test_paged as paged_sizes
from test_gpu_attention import F16, _rand, _starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv,dim", HEADS)
def test_sizes_where_the_device_is_known(heads, kv, dim):
    paged_sizes(heads, kv, dim)
    gradient_sizes(heads, kv, dim)


def test_one_workspace_for_prompts_chunks_and_single_tokens():
    rng = synth.child_rng(380)
    heads, kv, dim, page, n, longest = 32, 8, 128, 16, 8, 600
    cache = rb.Cache(*(_rand(rng, n * 38, page, kv, dim) for _ in range(2)))
    table = torch.arange(n * 38, dtype=torch.int32).view(n, 38).cuda()
    need = rb.lib.rb_attn_paged_workspace_bytes(ctypes.byref(cache.struct()), heads, n, 4096)
    behind = 4096
    ws = torch.full((need + behind,), 0x5a, dtype=torch.uint8, device="cuda")
    for new in ([512] * 8, [1] * 8, [512, 1, 1, 1], [1], [3, 5], [100], [600]):
        lengths = torch.tensor([min(m + 70 * i, longest) for i, m in enumerate(new)], dtype=torch.int32).cuda()
        q, first = _rand(rng, sum(new), heads, dim), _starts(new)
        some = table[:len(new)].contiguous()
        print(new, flush=True)
        want = rb.rb_attn_paged(cache, q, first, lengths, some)
        got = rb.rb_attn_paged(cache, q, first, lengths, some, workspace=ws[:need])
        torch.cuda.synchronize()
        assert torch.equal(got, want) and (ws[need:] == 0x5a).all()


def test_one_workspace_for_gradients():
    rng = synth.child_rng(381)
    heads, kv, dim = 16, 1, 128
    H = rb.binding.rb_heads(heads, kv, dim, rb.RB_F16, heads * dim, dim, kv * dim, dim, kv * dim, dim)
    need = rb.lib.rb_attn_grad_workspace_bytes(ctypes.byref(H), 4096, 4096)
    ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    for n in (4096, 2000, 2048, 1025, 128, 1):
        print(n, flush=True)
        q, k, v, go, first = *(_rand(rng, n, x, dim) for x in (heads, kv, kv, heads)), _starts([n])
        o, lse = rb.rb_attn_prompt(q, k, v, first, want_lse=True)
        want = rb.rb_attn_prompt_grad(go, q, k, v, o, lse, first)
        got, p = [torch.empty_like(x) for x in (q, k, v)], lambda x: x.data_ptr()
        assert rb.lib.rb_attn_prompt_grad(ctypes.byref(H), p(go), p(q), p(k), p(v), p(o), p(lse), p(first), None, 1, n, n, 1, dim ** -0.5, *map(p, got), p(ws), need,
                                          None) == rb.RB_OK
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and (ws[need:] == 0x5a).all()
