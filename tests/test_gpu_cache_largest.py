"""Tokens entering a cache, and coming back out of one, as many as a call may have: more workgroups than one dimension of a launch holds threads for.

Inputs are one row that all tokens share (a stride of zero) where their content does not matter, so that what has to be in memory is the results.
"""
import pytest
import torch

import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import F16, _rand
from test_gpu_cache8 import _ints, empty_cache

pytestmark = pytest.mark.gpu
TOKENS, LAST = 1 << 24, 37      # of them the last sequence's


def _cache(in8, pages, kv, dim):
    return empty_cache(pages, 16, kv, dim, F16) if in8 else rb.Cache.zeros(pages, 16, kv, dim)


@pytest.mark.parametrize("in8", [False, True])
@pytest.mark.parametrize("kv", [1, 129])      # one workgroup a token, with queries, and three
def test_tokens_entering(kv, in8):
    """The first sequence's positions but the first 48 lie outside of the page table; the last sequence's are all stored, and every token's queries come out."""
    rng = synth.child_rng(670, kv)
    dim, pages = 16, 8
    append = rb.rb_cache8_append if in8 else rb.rb_cache_append
    q = q_out = None
    if kv == 1:
        q = torch.zeros((TOKENS, 1, dim), dtype=F16, device="cuda")
        q[:, 0, 0] = (torch.arange(TOKENS, device="cuda") % 2039).half()
        q_out = torch.full_like(q, 7.0)
    k, v = (_rand(rng, 1, kv, dim).expand(TOKENS, kv, dim) for _ in range(2))
    table = _ints([[0, 1, 2], [5, 3, 4]])
    first, lengths = _ints([0, TOKENS - LAST, TOKENS]), _ints([TOKENS - LAST, LAST])
    cache, few = _cache(in8, pages, kv, dim), _cache(in8, pages, kv, dim)
    print(kv, in8, flush=True)
    append(cache, k, v, first, lengths, table, q=q, q_out=q_out)
    # the same tokens by a call of fewer
    append(few, k[:48 + LAST].contiguous(), v[:48 + LAST].contiguous(), _ints([0, 48, 48 + LAST]), _ints([48, LAST]), table)
    torch.cuda.synchronize()
    assert q is None or torch.equal(q_out, q)
    names = ("k", "v", "k_exp", "v_exp") if in8 else ("k", "v")
    for name in names:
        a, b = (getattr(c, name).view(torch.uint8) for c in (cache, few))
        assert torch.equal(a, b), name
    del q, q_out
    torch.cuda.empty_cache()


def test_positions_coming_back():
    """193 heads of 16 elements, four wavefronts a token; keys and values are one array, and come back into one, so that it is 104 GB and not twice that."""
    kv, dim, tokens = 193, 16, TOKENS
    need = tokens * kv * dim * 2
    if torch.cuda.mem_get_info()[0] < need + (8 << 30):
        pytest.skip("other programs hold the memory")
    rng = synth.child_rng(671)
    cache = empty_cache(4, 16, kv, dim, F16)
    x = _rand(rng, 48, kv, dim)
    rb.rb_cache8_append(cache, x, x, _ints([0, 11, 48]), _ints([11, 37]), _ints([[2, 3, 0], [3, 1, 0]]))
    # a first sequence whose positions lie outside of the table but for 11, the last one's 37
    cache = rb.Cache8(cache.k, cache.k, cache.k_exp, cache.k_exp, F16)
    out = torch.empty((tokens, kv, dim), dtype=F16, device="cuda")
    out[-200:] = 7.0
    out[TOKENS // 2:TOKENS // 2 + 200] = 7.0
    print(out.shape, flush=True)
    table = _ints([[2, -1, -1], [3, 1, 0]])
    rb.rb_cache8_read(cache, _ints([0, tokens - 37, tokens]), _ints([tokens - 37, 37]), table, tokens, out, out)
    want, _ = rb.rb_cache8_read(cache, _ints([0, 37]), _ints([37]), _ints([[3, 1, 0]]), 37)
    torch.cuda.synchronize()
    assert torch.equal(out[-37:].nan_to_num(nan=9.0), want.nan_to_num(nan=9.0)) and not out[-200:-37].any() and not out[TOKENS // 2:TOKENS // 2 + 200].any()
    assert torch.isfinite(want).all() and want.any()
    del out
    torch.cuda.empty_cache()
