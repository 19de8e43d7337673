"""A step of generation put together as a program has it: tokens enter a cache in 8 bits, attention over it, an output head, the next token; each part against the
fp64 oracle on what the part before it gave, eagerly and replayed from a captured graph.  And what the operators share: workspaces, streams, rows of any number.

Bounds: those of the parts by themselves (test_gpu_cache8.py, test_gpu_sample.py); whole numbers are equal.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle
import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import BF16, F16, _close, _f64, _rand, _sees, _starts
from test_gpu_cache8 import NAMES, _ints, _table, empty_cache
from test_gpu_sample import _f32, _i32, _logits, check

pytestmark = pytest.mark.gpu
INF = float("inf")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("attention_example", os.path.join(ROOT, "examples", "attention.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _head(rng, vocab, inn, dtype):
    g, h = (torch.from_numpy((0.1 * (1 + 0.2 * rng.random(s))).astype(np.float32)).half().cuda() for s in ((2, vocab), (2, inn)))
    W = torch.from_numpy(rng.standard_normal((vocab, inn)).astype(np.float32)).cuda()
    return rb.Layer(rb.rb_couple(W, g, h)[1], g, h, 2, vocab, inn)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_steps_of_a_program(dtype):
    """Prompts, a chunk beside single tokens, single tokens: every intermediate result is the next part's input and is looked at."""
    heads, kv, dim, page, vocab = 8, 2, 64, 16, 5003
    steps = [[33, 0, 100, 7], [1, 40, 1, 1], [1, 1, 1, 1], [3, 1, 0, 2]]
    rng = synth.child_rng(650)
    total = np.sum(steps, axis=0)
    host_table, pages = _table(rng, total, page)
    table, cache, head = torch.from_numpy(host_table).cuda(), empty_cache(pages, page, kv, dim, dtype), _head(rng, vocab, heads * dim, dtype)
    cos, sin = (torch.from_numpy(f(rng.random((200, dim // 2)) * 6).astype(np.float32)).cuda() for f in (np.cos, np.sin))
    lengths = np.zeros(4, dtype=int)
    for new in steps:
        print(dtype, new, flush=True)
        lengths = lengths + new
        t, first, now = sum(new), _starts(new), _ints(lengths)
        q, k, v = (_rand(rng, t, n, dim, dtype=dtype, gain=2.0) for n in (heads, kv, kv))
        turned = rb.rb_cache8_append(cache, k, v, first, now, table, q=q, cos=cos, sin=sin)
        all_k, all_v = rb.rb_cache8_read(cache, _starts(lengths), now, table, int(lengths.sum()))
        o = rb.rb_attn_cache8(cache, turned, first, now, table)
        has = [i for i, n in enumerate(new) if n]
        last = o.view(t, -1)[[int(np.cumsum(new)[i]) - 1 for i in has]].contiguous()
        logits = rb.rb_linear_gemm(head, last, out_dtype=torch.float32)
        torch.cuda.synchronize()
        ends = np.cumsum(lengths)
        for i in range(4):
            K, V, at = (_f64(x)[ends[i] - lengths[i]:ends[i]] for x in (all_k, all_v, all_k))
            mine = slice(sum(new[:i]), sum(new[:i + 1]))
            values, units = oracle.held_in_8_bits(_f64(v)[mine], NAMES[dtype])      # (v is not turned: held as it came)
            assert np.array_equal(V[lengths[i] - new[i]:], values * np.exp2(units - 127.0)[..., None])
            for h in range(heads):
                ref, _, mag = oracle.attention(_f64(turned)[mine, h], K[:, h // 4], V[:, h // 4], _sees(new[i], lengths[i], True), dim ** -0.5)
                _close(o[mine, h], ref, mag, dtype, (i, h))
        n = len(has)
        check(logits, rng.random(n), temperature=rng.choice([0.0, 0.6, 1.0, 1.5], n), top_k=rng.choice([0, 1, 20, 400], n), top_p=rng.choice([0.3, 0.9, 1.0], n),
              min_p=rng.choice([0.0, 0.02], n))


def test_whole_prompts_read_back_and_over_the_cache():
    """Attention over the cache, and attention of whole prompts with the keys and values that come back out of it: both to the oracle's of those."""
    rng = synth.child_rng(651)
    heads, kv, dim, lens = 8, 2, 128, [70, 1, 130]
    host_table, pages = _table(rng, lens, 16)
    table, cache, t = torch.from_numpy(host_table).cuda(), empty_cache(pages, 16, kv, dim, F16), sum(lens)
    q, k, v = _rand(rng, t, heads, dim, gain=2.0), _rand(rng, t, kv, dim), _rand(rng, t, kv, dim)
    first, now = _starts(lens), _ints(lens)
    rb.rb_cache8_append(cache, k, v, first, now, table)
    k, v = rb.rb_cache8_read(cache, first, now, table, t)
    outs = rb.rb_attn_cache8(cache, q, first, now, table), rb.rb_attn_prompt(q, k, v, first)
    torch.cuda.synchronize()
    for got in outs:
        at = 0
        for n in lens:
            s = slice(at, at + n)
            for h in range(heads):
                ref, _, mag = oracle.attention(_f64(q)[s, h], _f64(k)[s, h // 4], _f64(v)[s, h // 4], _sees(n, n, True), dim ** -0.5)
                _close(got[s, h], ref, mag, F16, (n, h))
            at += n


def test_a_captured_step_of_generation():
    """Tokens, lengths and caches stay on the device: a graph of one step, replayed, gives the tokens and the cache of eager steps, bit for bit."""
    heads, kv, dim, page, vocab, lens = 4, 2, 64, 16, 50001, [20, 61, 5]
    rng = synth.child_rng(652)
    host_table, pages = _table(rng, [n + 12 for n in lens], page)
    table, head = torch.from_numpy(host_table).cuda(), _head(rng, vocab, heads * dim, F16)
    embedding = _rand(rng, vocab, (heads + 2 * kv) * dim)
    u = _f32(rng.random((10, 3)))
    given = dict(temperature=_f32([0.8, 1.0, 0.0]), top_k=_i32([0, 40, 0]), top_p=_f32([0.9, 1.0, 1.0]), min_p=_f32([0.0, 0.05, 0.0]))
    first = _starts([1, 1, 1])

    def step(cache, tokens, now, random, out, ws):
        x = embedding[tokens].view(3, -1, dim)
        q = rb.rb_cache8_append(cache, x[:, heads:heads + kv], x[:, heads + kv:], first, now, table, q=x[:, :heads])
        o = rb.rb_attn_cache8(cache, q, first, now, table)
        return rb.rb_sample(rb.rb_linear_gemm(head, o.view(3, -1), out_dtype=torch.float32), random, tokens=out, workspace=ws, **given)

    def prepared():
        cache = empty_cache(pages, page, kv, dim, F16)
        r = synth.child_rng(653)
        rb.rb_cache8_append(cache, _rand(r, sum(lens), kv, dim), _rand(r, sum(lens), kv, dim), _starts(lens), _ints(lens), table)
        return cache, _i32([1, 2, 3]), _ints(lens)

    # eagerly, the outputs elsewhere each time
    cache, tokens, now = prepared()
    want = []
    for i in range(10):
        now = now + 1
        tokens = step(cache, tokens, now, u[i], None, None)
        want.append(tokens.tolist())
    held = [x.view(torch.uint8).clone() for x in (cache.k, cache.v)] + [cache.k_exp.clone(), cache.v_exp.clone()]

    cache, tokens, now = prepared()
    random, ws = u[0].clone(), torch.empty(rb.lib.rb_sample_workspace_bytes(rb.RB_F32, 3, vocab), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    side, graphs = torch.cuda.Stream(), [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:      # two graphs over one workspace
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            now += 1
            step(cache, tokens, now, random, tokens, ws)
    got = []
    for i in range(10):
        random.copy_(u[i])
        ws.fill_(255 if i % 3 else 0)
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got.append(tokens.tolist())
    assert got == want
    for a, b in zip(held, [x.view(torch.uint8) for x in (cache.k, cache.v)] + [cache.k_exp, cache.v_exp]):
        assert torch.equal(a, b)


def test_the_example_generates():
    ex = _example()
    model = ex.Blocks(blocks=2, heads=8, kv_heads=2, dim=64, ffn=1376, pages=40, page_tokens=16, positions=256, seed=3, in_8_bits=True)
    gen = torch.Generator(device="cuda").manual_seed(4)
    embedding = torch.randn(3000, 512, device="cuda", generator=gen).half()
    head, norm = ex.random_layer(gen, 3000, 512, rms=4.0), torch.ones(512, device="cuda").half()
    prompts = [torch.randint(3000, (n,), device="cuda", generator=gen) for n in (90, 17, 1)]
    u = torch.rand((6, 3), device="cuda", generator=gen)
    tokens = [ex.generate(model, embedding, norm, head, prompts, 6, u, temperature=_f32([0.0, 0.7, 1.0]), top_k=_i32([0, 1, 50])) for _ in range(2)]
    torch.cuda.synchronize()
    assert tokens[0].shape == (6, 3) and bool(((tokens[0] >= 0) & (tokens[0] < 3000)).all()) and torch.equal(tokens[0], tokens[1])
    greedy = ex.generate(model, embedding, norm, head, prompts, 6, u, temperature=_f32([0.0] * 3))
    torch.cuda.synchronize()
    # top-k of one draws the same as no temperature; the other sequences' tokens do not enter a sequence's own
    assert torch.equal(greedy[:, :2], tokens[0][:, :2])


# ------------------------------------------- rows shared by several workgroups ---
@pytest.mark.parametrize("dtype", [F16, torch.float32])
@pytest.mark.parametrize("rows", [1, 5, 33, 70, 129])
def test_rows_in_any_number(rows, dtype):
    """From one row, which many workgroups share, to one workgroup a row; a workspace that holds anything."""
    vocab = 66001
    rng = synth.child_rng(654, rows)
    x = _logits(rng, rows, vocab, dtype)
    u, t, k, p = rng.random(rows), rng.choice([0.5, 1.0, 3.0, 0.0], rows), rng.choice([0, 1, 9, 200, 3000, 30000], rows), rng.choice([0.2, 0.9, 0.999, 1.0], rows)
    check(x, u, temperature=t, top_k=k, top_p=p, label=rows)
    got = []
    for filled in (0, 255, 0x7f):
        ws = torch.full((rb.lib.rb_sample_workspace_bytes(rb.binding._DTYPE_CODE[dtype], rows, vocab),), filled, dtype=torch.uint8, device="cuda")
        got.append(rb.rb_sample(x, _f32(u), temperature=_f32(t), top_k=_i32(k), top_p=_f32(p), workspace=ws))
    torch.cuda.synchronize()
    assert all(torch.equal(g, got[0]) for g in got)


def test_shared_rows_with_masks_infinities_and_ties():
    rng = synth.child_rng(655)
    rows, vocab = 11, 120001
    x = _logits(rng, rows, vocab, torch.float32)
    x[0] = -INF
    x[1], x[1, 120000] = -INF, -3.0
    x[2] = float("nan")
    x[3, ::2], x[3, 1::3] = -INF, float("nan")
    x[4, 70000:] = torch.finfo(torch.float32).min
    x[5, 7], x[5, 110000], x[5, 60000] = INF, INF, INF
    x[6] = INF
    x[7] = 0.0                                            # all alike: more candidates than any list holds
    x[8] = torch.from_numpy(rng.integers(-2, 2, vocab).astype(np.float32))
    x[9] = 5 + 1e-4 * x[9]                                # all in few bins
    x[10, :40000] = 9.0
    u = rng.random(rows)
    for given in (dict(), dict(top_k=[3, 0, 3, 1000, 5, 2, 90001, 50001, 33333, 40001, 39999]), dict(top_p=[0.9, 0.9, 0.5, 0.99, 0.8, 0.5, 0.7, 0.3, 0.6, 0.45, 0.2]),
                  dict(top_k=[50, 1, 1, 9, 700, 3, 100, 119999, 60000, 100000, 50000], top_p=[0.5] * rows, min_p=[0.0, 0.1] * 5 + [0.3]), dict(temperature=[0.0] * rows)):
        print(sorted(given), flush=True)
        check(x, u, **given, label=sorted(given))


@pytest.mark.parametrize("dtype", [F16, BF16, torch.float32])
def test_a_row_gives_the_same_token_alone_and_among_others(dtype):
    """Alone many workgroups share it, among 300 it has one; sums do not depend on who adds them."""
    rng = synth.child_rng(657)
    vocab, n = 100003, 300
    rows = _logits(rng, 4, vocab, dtype)
    for i, given in enumerate((dict(), dict(top_k=700), dict(top_k=5), dict(top_p=0.93), dict(top_k=2000, top_p=0.97, min_p=1e-4))):
        each = {name: torch.full((n,), value, dtype=torch.int32 if name == "top_k" else torch.float32, device="cuda") for name, value in given.items()}
        u = _f32(rng.random(n))
        many = rb.rb_sample(rows.repeat(n // 4, 1), u, **each)
        for j in (0, 1, 2, 3, 130, 299):
            alone = rb.rb_sample(rows[j % 4:j % 4 + 1], u[j:j + 1].clone(), **{name: x[:1].clone() for name, x in each.items()})
            assert int(alone) == int(many[j]), (dtype, i, j)


def test_two_streams_at_once():
    """Calls on two streams, each with a workspace and a cache of its own, interleaved."""
    rng = synth.child_rng(656)
    streams = [torch.cuda.Stream() for _ in range(2)]
    x, u = [_logits(rng, 3, 128000, BF16) for _ in range(2)], [_f32(rng.random(3)) for _ in range(2)]
    p = _f32([0.9] * 3)
    want = [rb.rb_sample(a, b, top_p=p).tolist() for a, b in zip(x, u)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for s, a, b, out in zip(streams, x, u, got):
            with torch.cuda.stream(s):
                out.append(rb.rb_sample(a, b, top_p=p))
    torch.cuda.synchronize()
    assert all(g.tolist() == w for out, w in zip(got, want) for g in out)
