"""Attention over packed prompts and over the paged cache, and tokens entering it, against the fp64 oracle.

Bounds, derived from what is rounded: with u the rounding unit of the stored type (2^-11 fp16, 2^-8 bf16), every softmax
weight is rounded once before it meets the values and the result once, so an element is off by at most
u |o| + u sum_j p_j |v_j|, plus what fp32 sums and exponentials leave, which for the inputs here is well below
another u of the same sum.  Held to twice u of both, and 2^-24 for fp16 results below the normal range.
"""
import numpy as np
import pytest
import torch

import oracle
import synth
import paper_2602_05367_amd as rb

pytestmark = pytest.mark.gpu

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
F16, BF16 = torch.float16, torch.bfloat16


def _f64(t):
    return t.detach().double().cpu().numpy()


def _rand(rng, *shape, dtype=F16, gain=1.0):
    return (torch.from_numpy(rng.standard_normal(shape).astype(np.float32)) * gain).to(dtype).cuda()


def _starts(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32).cuda()


def _close(got, ref, mag, dtype, label):
    got, u = _f64(got), UNIT[dtype]
    assert np.array_equal(np.isnan(got), np.isnan(ref)), label
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]), label
    fine = np.isfinite(ref)
    off = np.abs(got - np.where(fine, ref, 0.0))[fine] - (2 * u * (np.abs(ref) + np.where(fine, mag, 0.0)) + 2.0 ** -24)[fine]
    assert off.size == 0 or off.max() <= 0, (label, float(off.max()))


def _sees(n_q, n_k, causal):
    return np.clip(np.arange(n_q) + 1 + n_k - n_q, 0, n_k) if causal else np.full(n_q, n_k)


def check_prompt(q, k, v, lens_q, lens_k, causal, scale=None, label=""):
    d, g = q.shape[2], q.shape[1] // k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    first, first_k = _starts(lens_q), _starts(lens_k)
    same = list(lens_q) == list(lens_k)
    o, lse = rb.rb_attn_prompt(q, k, v, first, first_k=None if same else first_k, causal=causal, scale=scale, want_lse=True)
    torch.cuda.synchronize()
    Q, K, V, O = _f64(q), _f64(k), _f64(v), o
    q0 = k0 = 0
    for n, m in zip(lens_q, lens_k):
        for h in range(q.shape[1]):
            ref, ref_lse, mag = oracle.attention(Q[q0:q0 + n, h], K[k0:k0 + m, h // g], V[k0:k0 + m, h // g], _sees(n, m, causal), scale)
            _close(O[q0:q0 + n, h], ref, mag, q.dtype, (label, n, m, h))
            got = _f64(lse[q0:q0 + n, h])
            assert np.array_equal(np.isfinite(got), np.isfinite(ref_lse)) and np.array_equal(np.isneginf(got), np.isneginf(ref_lse))
            fine = np.isfinite(ref_lse)
            assert np.all(np.abs(got[fine] - ref_lse[fine]) <= 2.0 ** -16 * np.maximum(1.0, np.abs(ref_lse[fine]))), (label, n, m, h)
        q0, k0 = q0 + n, k0 + m
    return o


LENGTHS = [[1], [2, 1, 3], [63, 64, 65], [0, 127, 0, 128, 129, 0], [300]]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv,dim", [(2, 2, 128), (6, 2, 64), (5, 1, 96), (4, 4, 8), (14, 2, 80)])
def test_packed_prompts(heads, kv, dim, causal, dtype):
    for n, lens in enumerate(LENGTHS):
        rng = synth.child_rng(300, heads, dim, n, causal)
        print(heads, kv, dim, causal, dtype, lens, flush=True)
        t = sum(lens)
        q, k, v = (_rand(rng, t, x, dim, dtype=dtype, gain=g) for x, g in ((heads, 2.0), (kv, 1.0), (kv, 1.0)))
        check_prompt(q, k, v, lens, lens, causal, label=(heads, kv, dim, causal, dtype, lens))


@pytest.mark.parametrize("causal", [True, False])
def test_more_or_fewer_keys_than_queries_and_rows_that_see_nothing(causal):
    """Causal rows are aligned at the end: with fewer keys than queries the first rows see none."""
    rng = synth.child_rng(301, causal)
    lens_q, lens_k = [5, 70, 0, 40, 9, 130], [200, 3, 17, 0, 9, 129]
    q, k, v = _rand(rng, sum(lens_q), 4, 64, gain=2.0), _rand(rng, sum(lens_k), 2, 64), _rand(rng, sum(lens_k), 2, 64)
    o = check_prompt(q, k, v, lens_q, lens_k, causal)
    assert not o[75:115].any()      # the sequence without keys


def test_no_keys_at_all():
    q, k = _rand(synth.child_rng(302), 7, 2, 64), torch.empty((0, 2, 64), dtype=F16, device="cuda")
    anything = torch.zeros((1, 2, 64), dtype=F16, device="cuda")
    first, first_k = _starts([7]), _starts([0])
    o, lse = rb.rb_attn_prompt(q, anything[:0], anything[:0], first, first_k=first_k, want_lse=True) if anything[:0].data_ptr() else (None, None)
    if o is not None:
        assert not o.any() and torch.isneginf(lse).all()
    H = rb.binding._heads(q, anything, anything)
    o, p = torch.full_like(q, 3.0), lambda t: t.data_ptr()
    assert rb.lib.rb_attn_prompt(H, p(q), p(anything), p(anything), p(first), p(first_k), 1, 7, 0, 0, 0.125, p(o), None, None) == rb.RB_OK
    torch.cuda.synchronize()
    assert not o.any() and k.numel() == 0


@pytest.mark.parametrize("dim", [64, 128])
def test_strided_heads_and_what_lies_between_them(dim):
    """q, k and v as parts of one tensor, head-major tensors, broadcast heads, with NaN in everything that is not theirs."""
    rng = synth.child_rng(303, dim)
    lens = [70, 131]
    t = sum(lens)
    x = torch.full((t + 3, 11, dim + 8), float("nan"), dtype=F16, device="cuda")
    x[2:-1, 1:9, :dim] = _rand(rng, t, 8, dim)
    q, k, v = x[2:-1, 1:5, :dim], x[2:-1, 5:7, :dim], x[2:-1, 7:9, :dim]
    assert q.data_ptr() % 16 == 0
    check_prompt(q, k, v, lens, lens, True, label="parts of one")
    major = [y.transpose(0, 1).contiguous().transpose(0, 1) for y in (q, k, v)]
    assert major[0].stride(0) == dim
    check_prompt(*major, lens, lens, True, label="head major")
    check_prompt(q, k[:, :1].expand(-1, 2, -1), v, lens, lens, True, label="broadcast keys")
    check_prompt(q, k[:1].expand(t, -1, -1), v, lens, lens, False, label="one key for all")


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_a_row_does_not_see_is_not_there(dim, dtype):
    """Infinities and NaN in later keys and values and in other sequences leave a row as it is; where it sees them they come out."""
    rng = synth.child_rng(304, dim)
    lens, heads = [150, 90, 33], 4
    q, k, v = (_rand(rng, sum(lens), h, dim, dtype=dtype) for h in (heads, 2, 2))
    clean = rb.rb_attn_prompt(q, k, v, _starts(lens))
    bad_k, bad_v = k.clone(), v.clone()
    bad_v[100, 0, 3] = float("inf")
    bad_v[101, 1, dim - 1] = float("nan")
    bad_v[120, 0, 3] = -float("inf")
    bad_v[130, 1, 9] = -float("inf")
    bad_k[140, 0, 1] = float("nan")
    bad_k[150:240], bad_v[150:240] = float("nan"), float("inf")      # all of the second sequence
    o = check_prompt(q, k, bad_v, lens, lens, True, label="values")
    assert torch.equal(o[:100], clean[:100])
    o = rb.rb_attn_prompt(q, bad_k, bad_v, _starts(lens))
    torch.cuda.synchronize()
    assert torch.equal(o[:100], clean[:100]) and torch.equal(o[240:], clean[240:])
    assert torch.isnan(o[150:240]).all() and torch.isnan(o[140:150, :2]).all() and torch.isfinite(o[:140, 2:, 10:dim - 1]).all()
    assert torch.equal(torch.isposinf(o[100:120, :2, 3]), torch.ones(20, 2, dtype=torch.bool, device="cuda")) and torch.isnan(o[120:140, :2, 3]).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_extreme_scores(dtype):
    """Weights of one key alone, of all keys alike, and scores of thousands, rising and falling along the keys."""
    rng = synth.child_rng(305)
    n, d = 200, 64
    q, k, v = (_rand(rng, n, 2, d, dtype=dtype) for _ in range(3))
    check_prompt(q * 0, k, v, [n], [n], True, label="all alike")
    ramp = torch.linspace(-60, 60, n, device="cuda")[:, None, None]
    for sign in (1, -1):
        check_prompt((q * 0 + 8).to(dtype), (k * 0 + sign * ramp).to(dtype), v, [n], [n], True, scale=1.0, label="ramp")
    check_prompt((q * 16).to(dtype), (k * 16).to(dtype), v, [n], [n], False, scale=1.0, label="one each")
    check_prompt(q, k, v, [n], [n], True, scale=1e-6, label="tiny scale")


def test_same_bits_again_and_on_another_stream():
    rng = synth.child_rng(306)
    lens = [400, 77]
    q, k, v = _rand(rng, 477, 8, 128), _rand(rng, 477, 2, 128), _rand(rng, 477, 2, 128)
    first = _starts(lens)
    want = rb.rb_attn_prompt(q, k, v, first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [rb.rb_attn_prompt(q, k, v, first) for _ in range(5)]
    side.synchronize()
    assert all(torch.equal(g, want) for g in got)


# ------------------------------------------------------------------ cache ---
def build_cache(rng, lengths, page, kv, dim, dtype, layout="tokens", spare=3):
    """A cache with all positions of all sequences filled, NaN everywhere else; host copies of what the sequences hold."""
    used = [-(-max(n, 0) // page) for n in lengths]
    pages = sum(used) + spare
    shape = (pages, page, kv, dim)
    if layout == "heads":
        k, v = (torch.full((pages, kv, page, dim), float("nan"), dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2))
    else:
        k, v = (torch.full(shape, float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    order = rng.permutation(pages)
    table = np.full((len(lengths), max(max(used), 1) + 1), -12345, dtype=np.int32)
    hold = []
    at = 0
    for i, n in enumerate(lengths):
        table[i, :used[i]] = order[at:at + used[i]]
        at += used[i]
        K, V = _rand(rng, max(n, 0), kv, dim, dtype=dtype), _rand(rng, max(n, 0), kv, dim, dtype=dtype)
        for p in range(used[i]):
            m = min(page, n - p * page)
            k[int(table[i, p]), :m], v[int(table[i, p]), :m] = K[p * page:p * page + m], V[p * page:p * page + m]
        hold.append((K, V))
    return rb.Cache(k, v), torch.from_numpy(table).cuda(), hold


def check_paged(q, cache, table, hold, new, lengths, scale=None, label="", o=None):
    d, g = q.shape[2], q.shape[1] // cache.kv_heads
    scale = d ** -0.5 if scale is None else scale
    got = rb.rb_attn_paged(cache, q, _starts(new), torch.tensor(lengths, dtype=torch.int32).cuda(), table, scale=scale)
    torch.cuda.synchronize()
    Q, at = _f64(q), 0
    for i, n in enumerate(new):
        K, V = _f64(hold[i][0]), _f64(hold[i][1])
        for h in range(q.shape[1]):
            ref, _, mag = oracle.attention(Q[at:at + n, h], K[:, h // g], V[:, h // g], _sees(n, max(lengths[i], 0), True), scale)
            _close(got[at:at + n, h], ref, mag, q.dtype, (label, i, n, lengths[i], h))
        at += n
    return got


PAGED = [  # new tokens, lengths after them
    ([1], [1]), ([1], [700]), ([1, 1, 1, 1], [5, 64, 1300, 129]), ([3, 1, 2, 5], [3, 900, 65, 200]),
    ([40, 1, 0, 17], [300, 77, 20, 17]), ([150], [150]), ([200, 1, 1], [1111, 31, 8]),
]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads,kv,dim,page", [(4, 4, 128, 16), (16, 2, 128, 64), (6, 2, 64, 8), (12, 1, 96, 32), (40, 1, 40, 256)])
def test_paged(heads, kv, dim, page, dtype):
    for n, (new, lengths) in enumerate(PAGED):
        rng = synth.child_rng(310, heads, dim, n)
        print(heads, kv, dim, page, dtype, new, lengths, flush=True)
        cache, table, hold = build_cache(rng, lengths, page, kv, dim, dtype, layout="heads" if n % 2 else "tokens")
        q = _rand(rng, sum(new), heads, dim, dtype=dtype, gain=2.0)
        check_paged(q, cache, table, hold, new, lengths, label=(heads, kv, dim, page, dtype))


def test_paged_long_contexts_and_many_sequences():
    rng = synth.child_rng(311)
    lengths = [int(x) for x in rng.integers(1, 400, 130)] + [20000, 9000]
    cache, table, hold = build_cache(rng, lengths, 16, 2, 64, F16)
    q = _rand(rng, len(lengths), 8, 64, gain=2.0)
    check_paged(q, cache, table, hold, [1] * len(lengths), lengths)


def test_paged_rows_that_see_nothing():
    """More new tokens than positions (the first of them lie before the sequence), and sequences without any."""
    rng = synth.child_rng(312)
    new, lengths = [4, 3, 90, 2], [2, 0, 30, -5]
    cache, table, hold = build_cache(rng, lengths, 16, 2, 64, F16)
    q = _rand(rng, sum(new), 4, 64)
    got = check_paged(q, cache, table, hold, new, lengths)
    assert not got[:2].any() and not got[4:67].any() and not got[97:].any() and got[2:4].all(-1).any()


@pytest.mark.parametrize("new", [[1, 1, 1], [9, 1, 40]])
def test_paged_masked_places(new):
    """Infinities and NaN in positions behind a row's own leave it as it is."""
    rng = synth.child_rng(313, len(new))
    lengths = [140, 64, 90]
    cache, table, hold = build_cache(rng, lengths, 16, 2, 128, F16)
    q = _rand(rng, sum(new), 4, 128)
    clean = check_paged(q, cache, table, hold, new, lengths)
    for i in range(3):      # the last position's key and value
        p = lengths[i] - 1
        page = int(table[i, p // 16])
        cache.k[page, p % 16], cache.v[page, p % 16] = float("nan"), float("inf")
    got = rb.rb_attn_paged(cache, q, _starts(new), torch.tensor(lengths, dtype=torch.int32).cuda(), table)
    torch.cuda.synchronize()
    last = [sum(new[:i + 1]) - 1 for i in range(3)]
    others = [i for i in range(sum(new)) if i not in last]
    assert torch.isnan(got[last]).all() and torch.equal(got[others], clean[others])


def test_paged_offsets_beyond_32_bits():
    """A cache of more than 4 GiB per array, its first and its last pages in use."""
    rng = synth.child_rng(314)
    page, kv, dim, pages = 128, 8, 128, 17000
    k, v = (torch.empty((pages, page, kv, dim), dtype=F16, device="cuda") for _ in range(2))
    assert k.numel() * 2 > 1 << 32
    lengths, hold, rows = [300, 130], [], [[pages - 1, 0, pages - 2], [pages // 2, 16384]]
    table = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    for i, n in enumerate(lengths):
        K, V = _rand(rng, n, kv, dim), _rand(rng, n, kv, dim)
        hold.append((K, V))
        for p, at in enumerate(rows[i]):
            table[i, p] = at
            m = min(page, n - p * page)
            k[at, :m], v[at, :m] = K[p * page:p * page + m], V[p * page:p * page + m]
    cache = rb.Cache(k, v)
    for new in ([1, 1], [70, 33]):
        check_paged(_rand(rng, sum(new), 16, dim), cache, table, hold, new, lengths)
    x = _rand(rng, 2, kv, dim)
    rb.rb_cache_append(cache, x, x, _starts([1, 1]), torch.tensor(lengths, dtype=torch.int32).cuda(), table)
    torch.cuda.synchronize()
    assert torch.equal(k[pages - 2, 43], x[0]) and torch.equal(v[16384, 1], x[1])


def test_paged_in_a_graph():
    """Captured once, replayed with other lengths and other cache contents."""
    rng = synth.child_rng(315)
    lengths = [200, 777]
    cache, table, hold = build_cache(rng, lengths, 16, 2, 128, F16)
    q = _rand(rng, 2, 8, 128)
    first, now = _starts([1, 1]), torch.tensor(lengths, dtype=torch.int32).cuda()
    new_k, new_v = _rand(rng, 2, 2, 128), _rand(rng, 2, 2, 128)
    o = rb.rb_attn_paged(cache, q, first, now, table)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        rb.rb_cache_append(cache, new_k, new_v, first, now, table)
        o = rb.rb_attn_paged(cache, q, first, now, table)
    for i in range(3):
        now.copy_(torch.tensor([100 + 7 * i, 700 - 60 * i], dtype=torch.int32))
        new_k.copy_(_rand(rng, 2, 2, 128))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = rb.rb_attn_paged(cache, q, first, now, table)
        torch.cuda.synchronize()
        assert torch.equal(o, want)
        page = int(table[0, (100 + 7 * i - 1) // 16])
        assert torch.equal(cache.k[page, (100 + 7 * i - 1) % 16], new_k[0])


# ----------------------------------------------------------------- append ---
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,kv,dim,rotary,page", [(4, 4, 128, 128, 16), (8, 1, 64, 32, 8), (3, 3, 80, 80, 64), (2, 2, 72, 72, 16), (4, 2, 96, 0, 32)])
def test_append(heads, kv, dim, rotary, page, interleaved, dtype):
    rng = synth.child_rng(320, heads, dim, rotary)
    new, lengths = [1, 0, 30, 5], [1, 40, 47, 300]
    cache, table, hold = build_cache(rng, lengths, page, kv, dim, dtype)
    before = cache.k.clone(), cache.v.clone()
    t = sum(new)
    x = torch.full((t, heads + 2 * kv + 1, dim), float("nan"), dtype=dtype, device="cuda")
    x[:, :-1] = _rand(rng, t, heads + 2 * kv, dim, dtype=dtype)
    q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:-1]
    cos = sin = None
    if rotary:
        angle = rng.uniform(-4, 4, (max(lengths), rotary // 2))
        cos, sin = (torch.from_numpy(f(angle).astype(np.float32)).cuda() for f in (np.cos, np.sin))
    got = rb.rb_cache_append(cache, k, v, _starts(new), torch.tensor(lengths, dtype=torch.int32).cuda(), table, q=q, cos=cos, sin=sin,
                             interleaved=interleaved)
    torch.cuda.synchronize()
    at, u = 0, UNIT[dtype]
    for i, n in enumerate(new):
        for j in range(n):
            p = lengths[i] - n + j
            page_at = int(table[i, p // page])
            turn = (lambda y: oracle.rotary(_f64(y), _f64(cos[p]), _f64(sin[p]), interleaved)) if rotary else _f64
            for y, src in ((got[at + j], q[at + j]), (cache.k[page_at, p % page], k[at + j])):
                # one rounding; two products and their sum in fp32 before it, of operands that may cancel
                ref, most = turn(src), float(src.float().abs().max())
                assert np.all(np.abs(_f64(y) - ref) <= u * np.abs(ref) + 2.0 ** -22 * most + 2.0 ** -24)
            assert torch.equal(cache.v[page_at, p % page], v[at + j])
            before[0][page_at, p % page], before[1][page_at, p % page] = cache.k[page_at, p % page], cache.v[page_at, p % page]
        at += n
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert same(cache.k, before[0]) and same(cache.v, before[1])      # nothing else has been written


def test_append_in_place_and_without_queries():
    rng = synth.child_rng(321)
    new, lengths = [7, 2], [20, 2]
    cache, table, _ = build_cache(rng, lengths, 16, 2, 64, F16)
    q, k, v = _rand(rng, 9, 4, 64), _rand(rng, 9, 2, 64), _rand(rng, 9, 2, 64)
    angle = torch.linspace(0, 6, 20 * 32, device="cuda").view(20, 32)
    first, now, cos, sin = _starts(new), torch.tensor(lengths, dtype=torch.int32).cuda(), angle.cos(), angle.sin()
    for interleaved in (False, True):
        want = rb.rb_cache_append(cache, k, v, first, now, table, q=q, cos=cos, sin=sin, interleaved=interleaved)
        held = cache.k.clone()
        again = q.clone()
        rb.rb_cache_append(cache, k, v, first, now, table, q=again, cos=cos, sin=sin, interleaved=interleaved, q_out=again)
        assert rb.rb_cache_append(cache, k, v, first, now, table, cos=cos, sin=sin, interleaved=interleaved) is None
        torch.cuda.synchronize()
        assert torch.equal(want, again) and torch.equal(held.view(torch.int16), cache.k.view(torch.int16))


def test_append_outside_the_table_is_not_stored():
    rng = synth.child_rng(322)
    cache, table, _ = build_cache(rng, [20, 20], 16, 2, 64, F16)
    before = cache.k.clone().view(torch.int16), cache.v.clone().view(torch.int16)
    k = _rand(rng, 4, 2, 64)
    # two tokens before position 0; two behind the table's last
    lengths = torch.tensor([0, table.shape[1] * 16 + 2], dtype=torch.int32).cuda()
    rb.rb_cache_append(cache, k, k, _starts([2, 2]), lengths, table)
    torch.cuda.synchronize()
    assert torch.equal(cache.k.view(torch.int16), before[0]) and torch.equal(cache.v.view(torch.int16), before[1])


def test_appended_tokens_are_what_attention_reads():
    """A prompt in two chunks and three single tokens through the cache give what one pass over the whole gives."""
    rng = synth.child_rng(323)
    n, heads, kv, dim, page = 150, 4, 2, 64, 16
    q, k, v = _rand(rng, n, heads, dim), _rand(rng, n, kv, dim), _rand(rng, n, kv, dim)
    cache = rb.Cache.zeros(12, page, kv, dim)
    table = torch.arange(12, dtype=torch.int32).flip(0).contiguous().view(1, 12).cuda()
    out, at = [], 0
    for m in (100, 47, 1, 1, 1):
        first, now = _starts([m]), torch.tensor([at + m], dtype=torch.int32).cuda()
        rb.rb_cache_append(cache, k[at:at + m], v[at:at + m], first, now, table)
        out.append(rb.rb_attn_paged(cache, q[at:at + m], first, now, table))
        at += m
    torch.cuda.synchronize()
    got, Q, K, V = torch.cat(out), _f64(q), _f64(k), _f64(v)
    for h in range(heads):
        ref, _, mag = oracle.attention(Q[:, h], K[:, h // 2], V[:, h // 2], _sees(n, n, True), dim ** -0.5)
        _close(got[:, h], ref, mag, F16, h)
