"""Attention and its gradient where the work is laid out in other ways: many sequences, many workgroups, contexts of very different lengths.

Bounds as in the tests of the operators themselves, whose checks these use.
"""
import numpy as np
import pytest
import torch

import synth
import paper_2602_05367_amd as rb
import test_gpu_attention_grad as grad
from test_gpu_attention import BF16, F16, _rand, _starts, build_cache, check_paged, check_prompt

pytestmark = pytest.mark.gpu


def _lengths(rng, n, most):
    return [int(x) for x in rng.integers(0, most, n - 1)] + [most]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [2, 16, 17, 70])
def test_many_packed_sequences(n, causal):
    rng = synth.child_rng(360, n, causal)
    lens = _lengths(rng, n, 300 if n < 20 else 90)
    other = [int(x) for x in rng.permutation(lens)]
    print(lens, other, flush=True)
    for lens_k in (lens, other):
        q, go = (_rand(rng, sum(lens), 4, 64, gain=g) for g in (2.0, 0.01))
        k, v = (_rand(rng, sum(lens), 2, 64) for _ in range(2))
        check_prompt(q, k, v, lens, lens_k, causal)
        grad.check(go, q, k, v, lens, lens_k, causal)


@pytest.mark.parametrize("heads,kv,dim,dtype", [(36, 36, 64, F16), (40, 40, 128, BF16)])
def test_more_workgroups_than_compute_units(heads, kv, dim, dtype):
    rng = synth.child_rng(361, heads)
    lens = [700, 1, 450, 64]
    q, k, v = (_rand(rng, sum(lens), heads, dim, dtype=dtype, gain=g) for g in (2.0, 1.0, 1.0))
    check_prompt(q, k, v, lens, lens, True)
    # what a row does not see: a value and a key of the first sequence, a whole sequence
    clean = rb.rb_attn_prompt(q, k, v, _starts(lens))
    v[600, 3, 5], k[601, 4], v[701:1151] = float("inf"), float("nan"), float("nan")
    got = rb.rb_attn_prompt(q, k, v, _starts(lens))
    torch.cuda.synchronize()
    assert torch.equal(got[:600], clean[:600]) and torch.equal(got[1151:], clean[1151:]) and torch.equal(got[:701, 5:], clean[:701, 5:])
    assert torch.isinf(got[600:700, 3, 5]).all() and torch.isnan(got[601:700, 4]).all() and torch.isnan(got[701:1151]).all()


@pytest.mark.parametrize("heads,kv,dim,page,dtype", [(8, 2, 128, 8, F16), (6, 2, 64, 64, BF16), (5, 1, 96, 16, F16)])
def test_chunks_over_contexts_of_very_different_lengths(heads, kv, dim, page, dtype):
    rng = synth.child_rng(362, heads)
    new, lengths = [300, 64, 1, 33, 0, 200, 50], [420, 3100, 2500, 33, 10, 201, 20]      # (the last: thirty that see nothing)
    cache, table, hold = build_cache(rng, lengths, page, kv, dim, dtype)
    q = _rand(rng, sum(new), heads, dim, dtype=dtype, gain=2.0)
    check_paged(q, cache, table, hold, new, lengths)
    check_paged(q[:128], cache, table[1:2], hold[1:2], [128], lengths[1:2])
    first, now = _starts(new), torch.tensor(lengths, dtype=torch.int32).cuda()
    clean = rb.rb_attn_paged(cache, q, first, now, table)
    for i in (0, 1, 5):      # the last position's key and value
        p = lengths[i] - 1
        at = int(table[i, p // page])
        cache.k[at, p % page], cache.v[at, p % page] = float("nan"), float("inf")
    got = rb.rb_attn_paged(cache, q, first, now, table)
    torch.cuda.synchronize()
    last = [int(first[i + 1]) - 1 for i in (0, 1, 5)]
    others = [i for i in range(sum(new)) if i not in last]
    assert torch.isnan(got[last]).all() and torch.equal(got[others], clean[others])


def test_chunks_of_many_sequences():
    rng = synth.child_rng(363)
    for n, new, heads, kv in ((70, 9, 8, 2), (40, 40, 32, 32)):      # workgroups that share keys; one for every block of rows
        lengths = [int(x) for x in rng.integers(new - 3, 300, n)]
        cache, table, hold = build_cache(rng, lengths, 16, kv, 64, F16)
        check_paged(_rand(rng, n * new, heads, 64, gain=2.0), cache, table, hold, [new] * n, lengths)


def test_drafts_of_many_sequences():
    rng = synth.child_rng(364)
    new = [int(x) for x in rng.integers(0, 7, 90)]
    lengths = [int(x) + n for x, n in zip(np.exp(rng.uniform(0, 7, 90)), new)]
    cache, table, hold = build_cache(rng, lengths, 32, 2, 128, BF16)
    check_paged(_rand(rng, sum(new), 8, 128, dtype=BF16, gain=2.0), cache, table, hold, new, lengths)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", [[700, 450], [64, 700, 1, 450, 0, 333, 200, 90], [130, 0, 1, 257, 33, 90, 412, 128, 77, 5, 300, 64, 18, 201, 2, 60]])
def test_sequences_whose_blocks_are_taken_heaviest_first(lens, causal):
    """More blocks than run at once, of up to sixteen sequences."""
    rng = synth.child_rng(365, len(lens), causal)
    t, other = sum(lens), [int(x) for x in rng.permutation(lens)]
    for heads, kv, lens_k in ((60, 60, lens), (42, 14, other)):
        q, go = (_rand(rng, t, heads, 64, gain=g) for g in (2.0, 0.01))
        k, v = (_rand(rng, t, kv, 64) for _ in range(2))
        check_prompt(q, k, v, lens, lens_k, causal)
        if heads == 42:
            grad.check(go, q, k, v, lens, lens_k, causal)
            grad.check(go, q, k, v, lens, lens, causal)


def test_chunks_and_gradients_in_a_graph():
    """Captured once, replayed with other lengths and other operands, each replay against the eager calls."""
    rng = synth.child_rng(366)
    new, lengths = [90, 1, 40], [1500, 300, 700]
    cache, table, _ = build_cache(rng, lengths, 16, 2, 128, F16)
    q, first, now = _rand(rng, sum(new), 8, 128), _starts(new), torch.tensor(lengths, dtype=torch.int32).cuda()
    p, go = _rand(rng, sum(new), 8, 128), _rand(rng, sum(new), 8, 128)
    k, v = _rand(rng, sum(new), 2, 128), _rand(rng, sum(new), 2, 128)

    def run():
        o, lse = rb.rb_attn_prompt(p, k, v, first, want_lse=True)
        return (rb.rb_attn_paged(cache, q, first, now, table), o, *rb.rb_attn_prompt_grad(go, p, k, v, o, lse, first))

    run()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        got = run()
    for i in range(3):
        now.copy_(torch.tensor([1500 - 400 * i, 300 - 7 * i, 700], dtype=torch.int32))
        q.copy_(_rand(rng, *q.shape))
        k.copy_(_rand(rng, *k.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
