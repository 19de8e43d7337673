"""One token or one head: the stride of an axis of length one is no stride, whatever torch keeps there (odd, huge, of another axis)."""
import pytest
import torch

import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import F16, _rand, _starts

pytestmark = pytest.mark.gpu
ODD = [3, 100, (1 << 23) + 8, 1 << 40]


def _as(x, axis, stride):
    """x with another stride where its length is one."""
    assert x.shape[axis] == 1
    return x.as_strided(x.shape, [stride if i == axis else s for i, s in enumerate(x.stride())])


@pytest.mark.parametrize("stride", ODD)
def test_one_token(stride):
    rng = synth.child_rng(420)
    q, k, v, go = _rand(rng, 1, 4, 64), _rand(rng, 1, 2, 64), _rand(rng, 1, 2, 64), _rand(rng, 1, 4, 64)
    first, cos = _starts([1]), torch.ones((9, 32), device="cuda")
    cache = rb.Cache.zeros(2, 16, 2, 64)
    table, lengths = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([5], dtype=torch.int32, device="cuda")

    def run(q, k, v):
        o, lse = rb.rb_attn_prompt(q, k, v, first, want_lse=True)
        turned = rb.rb_cache_append(cache, k, v, first, lengths, table, q=q, cos=cos, sin=cos)
        return o, lse, turned, rb.rb_attn_paged(cache, q, first, lengths, table), *rb.rb_attn_prompt_grad(go, q, k, v, o, lse, first)

    want = run(q, k, v)
    got = run(*(_as(x, 0, stride) for x in (q, k, v)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("stride", ODD)
def test_one_head(stride):
    rng = synth.child_rng(421)
    q, k, v, go = (_rand(rng, 70, 1, 64) for _ in range(4))
    first = _starts([70])

    def run(q, k, v):
        o, lse = rb.rb_attn_prompt(q, k, v, first, want_lse=True)
        return o, lse, *rb.rb_attn_prompt_grad(go, q, k, v, o, lse, first)

    assert all(torch.equal(a, b) for a, b in zip(run(*(_as(x, 1, stride) for x in (q, k, v))), run(q, k, v)))


@pytest.mark.parametrize("stride", ODD)
def test_one_page_and_head_of_a_cache(stride):
    rng = synth.child_rng(422)
    k, v, q = _rand(rng, 1, 16, 1, 64), _rand(rng, 1, 16, 1, 64), _rand(rng, 1, 1, 64)
    table, first, lengths = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), _starts([1]), torch.tensor([11], dtype=torch.int32, device="cuda")
    want = rb.rb_attn_paged(rb.Cache(k, v), q, first, lengths, table)
    odd = rb.Cache(*(_as(_as(x, 0, stride), 2, stride) for x in (k, v)))
    assert torch.equal(rb.rb_attn_paged(odd, _as(q, 1, stride), first, lengths, table), want)
    odd = rb.Cache(_as(k, 0, stride), _as(v, 2, stride))
    assert torch.equal(rb.rb_attn_paged(odd, q, first, lengths, table), want)


def test_the_last_token_of_each_of_many():
    """Rows taken out of a large tensor one by one: their strides are the large tensor's."""
    x = torch.zeros((1, 5000, 40, 128), dtype=F16, device="cuda").normal_()
    last = x[:, -1]
    assert last.stride(0) > 1 << 23
    assert torch.equal(rb.rb_attn_prompt(last, last, last, _starts([1])), last)
