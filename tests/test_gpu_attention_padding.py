"""Calls of a fixed number of tokens of which the last belong to no sequence, as a captured graph has them, and page tables whose
unused entries are -1: nothing but the sequences' own positions is written, and the padding's rows stay as they are.
"""
import numpy as np
import pytest
import torch

import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import BF16, F16, _rand, _starts

pytestmark = pytest.mark.gpu
KEPT = 7.0


def _cache(rng, lengths, page, kv, dim, dtype, unused):
    """A cache of random values, with a table that has two places more than any sequence needs."""
    used = [-(-n // page) for n in lengths]
    cache = rb.Cache(*(_rand(rng, sum(used) + 2, page, kv, dim, dtype=dtype) for _ in range(2)))
    order, table = rng.permutation(sum(used) + 2), np.full((len(lengths), max(used) + 2), unused)
    for i, n in enumerate(used):
        table[i, :n] = order[sum(used[:i]):sum(used[:i + 1])]
    return cache, torch.from_numpy(table.astype(np.int32)).cuda()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n_seqs", [1, 3, 63, 64, 130])
@pytest.mark.parametrize("unused", [-1, 1 << 20, -(1 << 31)])
def test_append(n_seqs, unused, dtype):
    rng = synth.child_rng(370, n_seqs)
    page, kv, dim, heads, more = 16, 2, 64, 4, 21
    new = [1 + i % 3 for i in range(n_seqs)]
    lengths = [n + (16 - n if i % 2 else 5 * (i % 7)) for i, n in enumerate(new)]      # every other one ends with its page
    cache, table = _cache(rng, lengths, page, kv, dim, dtype, unused)
    t = sum(new)
    q, k, v = (_rand(rng, t + more, x, dim, dtype=dtype) for x in (heads, kv, kv))
    want_k, want_v, at = cache.k.clone(), cache.v.clone(), 0
    for i, n in enumerate(new):
        for j in range(n):
            p = lengths[i] - n + j
            where = int(table[i, p // page]), p % page
            want_k[where], want_v[where] = k[at + j], v[at + j]
        at += n
    q_out = torch.full_like(q, KEPT)
    got = rb.rb_cache_append(cache, k, v, _starts(new), torch.tensor(lengths, dtype=torch.int32).cuda(), table, q=q, q_out=q_out)
    torch.cuda.synchronize()
    assert torch.equal(cache.k, want_k) and torch.equal(cache.v, want_v)
    assert torch.equal(got[:t], q[:t]) and (got[t:] == KEPT).all()


def test_append_of_padding_alone():
    rng = synth.child_rng(371)
    cache, table = _cache(rng, [5, 16], 16, 2, 64, F16, -1)
    before = cache.k.clone(), cache.v.clone()
    k = _rand(rng, 40, 2, 64)
    rb.rb_cache_append(cache, k, k, _starts([0, 0]), torch.tensor([5, 16], dtype=torch.int32).cuda(), table)
    torch.cuda.synchronize()
    assert torch.equal(cache.k, before[0]) and torch.equal(cache.v, before[1])


@pytest.mark.parametrize("new", [[1, 1, 1], [1, 300, 0, 5]])
def test_attention_over_the_cache(new):
    rng = synth.child_rng(372, len(new))
    lengths = [n + p for n, p in zip(new, (33, 500, 7, 16))]
    cache, table = _cache(rng, lengths, 16, 2, 64, F16, -1)
    t, now = sum(new), torch.tensor(lengths, dtype=torch.int32).cuda()
    q = _rand(rng, t + 50, 4, 64)
    want = rb.rb_attn_paged(cache, q[:t], _starts(new), now, table)
    got = rb.rb_attn_paged(cache, q, _starts(new), now, table, o=torch.full_like(q, KEPT))
    torch.cuda.synchronize()
    # (how the work is shared out may depend on the number of tokens)
    assert (got[t:] == KEPT).all() and (got[:t].float() - want.float()).abs().max() <= 2.0 ** -8


def test_prompts_and_their_gradient():
    rng = synth.child_rng(373)
    lens, more = [130, 1, 70], 90
    t = sum(lens)
    q, k, v, go = (_rand(rng, t + more, x, 64) for x in (4, 2, 2, 4))
    for x in (q, k, v, go):
        x[t:] = float("nan")
    first = _starts(lens)
    o, lse = rb.rb_attn_prompt(q, k, v, first, want_lse=True, o=torch.full_like(q, KEPT))
    want, want_lse = rb.rb_attn_prompt(q[:t], k[:t], v[:t], first, want_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(o[:t], want) and torch.equal(lse[:t], want_lse) and (o[t:] == KEPT).all()
    H, p = rb.binding._heads(q, k, v), lambda x: x.data_ptr()
    grads = [torch.full_like(x, KEPT) for x in (q, k, v)]
    ws = torch.empty(rb.lib.rb_attn_grad_workspace_bytes(H, t + more, t + more), dtype=torch.uint8, device="cuda")
    assert rb.lib.rb_attn_prompt_grad(H, p(go), p(q), p(k), p(v), p(o), p(lse), p(first), None, len(lens), t + more, t + more, 1, 0.125, *map(p, grads), p(ws),
                                      ws.numel(), None) == rb.RB_OK
    wants = rb.rb_attn_prompt_grad(go[:t].contiguous(), q[:t], k[:t], v[:t], want, want_lse, first)
    torch.cuda.synchronize()
    for g, w in zip(grads, wants):
        assert (g[t:] == KEPT).all() and torch.isfinite(g[:t]).all() and (g[:t].float() - w.float()).abs().max() <= 2.0 ** -8 * float(w.float().abs().max())
