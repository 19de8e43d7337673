"""The cache in 8 bits: what tokens become in it, what comes back, and attention over it, against the fp64 oracle.

Bounds.  A value is rounded once, from the 16-bit input or, turned, from fp32: what is held is the nearest of its e4m3 neighbours, off by at most half of
their distance, plus, turned, three fp32 roundings of its pair (3 * 2^-24 of |x cos| + |y sin|).  Attention is held to the bounds of attention over a
cache of 16 bits (test_gpu_attention.py), for the values that the cache holds: elements come out of 8 bits exactly.
"""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import BF16, F16, PAGED, _close, _f64, _rand, _sees, _starts

pytestmark = pytest.mark.gpu
NAMES = {F16: "fp16", BF16: "bf16"}
E4M3 = torch.float8_e4m3fn


def _held(elements, exponents):
    """The values that elements [..., d] and bytes [...] stand for, in 64 bits on the host."""
    return elements.double().cpu().numpy() * np.exp2(exponents.cpu().numpy().astype(np.float64) - 127.0)[..., None]


def _ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def _table(rng, lengths, page, spare=3, unused=-12345):
    used = [-(-max(n, 0) // page) for n in lengths]
    order, table = rng.permutation(sum(used) + spare), np.full((len(lengths), max(max(used), 1) + 1), unused, dtype=np.int32)
    for i, n in enumerate(used):
        table[i, :n] = order[sum(used[:i]):sum(used[:i + 1])]
    return table, sum(used) + spare


def empty_cache(pages, page, kv, dim, dtype, layout="tokens"):
    """A cache of NaN everywhere, its exponents NaN's as well."""
    shape = (pages, kv, page, dim) if layout == "heads" else (pages, page, kv, dim)
    k, v = (torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    if layout == "heads":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return rb.Cache8(k, v, *(torch.full((pages, kv, page), 255, dtype=torch.uint8, device="cuda") for _ in range(2)), dtype)


def build_cache(rng, lengths, page, kv, dim, dtype, layout="tokens", spread=0.7):
    """A cache with all positions of all sequences filled, NaN everywhere else; host copies of the values that the sequences hold."""
    table, pages = _table(rng, lengths, page)
    cache = empty_cache(pages, page, kv, dim, dtype, layout)
    # (views of bytes: elements of 8 bits are not indexed on every device)
    raw = [x.view(torch.uint8) for x in (cache.k, cache.v)]
    hold = []
    for i, n in enumerate(lengths):
        pair = []
        for at, exponents in zip(raw, (cache.k_exp, cache.v_exp)):
            x = rng.standard_normal((max(n, 0), kv, dim)) * np.exp(spread * rng.standard_normal((max(n, 0), kv, 1)))
            values, exps = oracle.held_in_8_bits(x, NAMES[dtype])
            codes = torch.from_numpy(values).float().to(E4M3).view(torch.uint8).cuda()
            for p in range(-(-max(n, 0) // page)):
                m = slice(p * page, min((p + 1) * page, n))
                at[int(table[i, p]), :m.stop - m.start] = codes[m]
                exponents[int(table[i, p]), :, :m.stop - m.start] = torch.from_numpy(exps[m].T.astype(np.uint8)).cuda()
            pair.append(values * np.exp2(exps - 127.0)[..., None])
        hold.append(pair)
    return cache, torch.from_numpy(table).cuda(), hold


# ------------------------------------------------------------- entering it ---
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,kv,dim,rotary,page", [(4, 4, 128, 128, 16), (8, 1, 64, 32, 8), (3, 3, 80, 80, 64), (2, 2, 16, 16, 16), (4, 2, 96, 0, 32), (6, 6, 112, 56, 16)])
def test_append(heads, kv, dim, rotary, page, interleaved, dtype):
    rng = synth.child_rng(610, heads, dim, rotary)
    new, lengths = [1, 0, 30, 5], [1, 40, 47, 300]
    table, pages = _table(rng, lengths, page)
    cache = empty_cache(pages, page, kv, dim, dtype, "heads" if interleaved else "tokens")
    before = [x.view(torch.uint8).clone() for x in (cache.k, cache.v)] + [cache.k_exp.clone(), cache.v_exp.clone()]
    t = sum(new)
    x = torch.full((t, heads + 2 * kv, dim + 8), float("nan"), dtype=dtype, device="cuda")
    x[:, :, :dim] = _rand(rng, t, heads + 2 * kv, dim, dtype=dtype) * torch.exp(2 * _rand(rng, t, heads + 2 * kv, 1, dtype=torch.float32)).to(dtype)
    q, k, v = x[:, :heads, :dim], x[:, heads:heads + kv, :dim], x[:, heads + kv:, :dim]
    angle = torch.from_numpy(rng.uniform(-7, 7, (300, rotary // 2))).cuda()
    cos, sin = (angle.cos().float(), angle.sin().float()) if rotary else (None, None)
    got = rb.rb_cache8_append(cache, k, v, _starts(new), _ints(lengths), torch.from_numpy(table).cuda(), q=q, cos=cos, sin=sin, interleaved=interleaved)
    torch.cuda.synchronize()
    at = 0
    written = torch.zeros((pages, page), dtype=torch.bool)
    for i, n in enumerate(new):
        for j in range(n):
            p = lengths[i] - n + j
            where = int(table[i, p // page]), p % page
            written[where] = True
            turn = (lambda y: oracle.rotary(_f64(y), _f64(cos[p]), _f64(sin[p]), interleaved)) if rotary else _f64
            # what moves a turned value: three roundings of |x cos| + |y sin|
            size = np.abs(oracle.rotary(np.abs(_f64(k[at])), np.abs(_f64(cos[p])), -np.abs(_f64(sin[p])), interleaved)) + np.abs(
                oracle.rotary(np.abs(_f64(k[at])), np.abs(_f64(cos[p])), np.abs(_f64(sin[p])), interleaved)) if rotary else np.zeros((kv, dim))
            off = 3 * 2.0 ** -24 * size
            ref, units = oracle.held_in_8_bits(_f64(v[at]), NAMES[dtype])
            assert np.array_equal(cache.v[where].double().cpu().numpy(), ref) and np.array_equal(cache.v_exp[where[0], :, where[1]].cpu().numpy(), units), (i, j)
            exact = turn(k[at])
            exps = cache.k_exp[where[0], :, where[1]].cpu().numpy().astype(np.int64)
            low, high = (oracle.held_in_8_bits(exact * f, NAMES[dtype])[1] for f in (1 - 2.0 ** -21, 1 + 2.0 ** -21))
            assert ((exps >= low) & (exps <= high)).all(), (i, j, exps, low, high)
            held = _held(cache.k[where], cache.k_exp[where[0], :, where[1]])
            step = np.exp2(np.maximum(np.frexp(np.abs(exact) + off)[1] - 1 - (exps - 127)[:, None], -6) - 3 + (exps - 127)[:, None])
            assert (np.abs(held - exact) <= step / 2 * (1 + 1e-9) + off).all(), (i, j)
            ref = turn(q[at])
            assert (np.abs(_f64(got[at]) - ref) <= {F16: 2.0 ** -11, BF16: 2.0 ** -8}[dtype] * np.abs(ref) + 2.0 ** -21 * np.abs(ref).max()).all()
            at += 1
    for now, was, per in zip((cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_exp.transpose(1, 2), cache.v_exp.transpose(1, 2)),
                             (before[0], before[1], before[2].transpose(1, 2), before[3].transpose(1, 2)), (1, 1, 1, 1)):
        assert torch.equal(now[~written], was[~written])      # nobody else's


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_append_at_the_edges_of_the_type(dtype):
    """The largest values, zeros, subnormal ones, infinities and NaN, heads whose largest lies next to where the unit changes."""
    large, least = float(torch.finfo(dtype).max), 2.0 ** (-24 if dtype == F16 else -133)
    eps = float(torch.finfo(dtype).eps)
    firsts = [large, -large, 0.0, least, -3 * least, float("inf"), float("nan"), 1.75, 1.75 * (1 + eps), 448.0, 448 * (1 + eps), 1.0, 2.0, 2 - eps, large / 2, 61440.0]
    dim = 32
    x = torch.zeros((len(firsts), 1, dim), dtype=dtype, device="cuda")
    x[:, 0, 5] = torch.tensor(firsts, dtype=torch.float64).to(dtype).cuda()
    x[:, 0, 6] = 1.0 / 3
    x[2:5, 0, 6] = least * 2
    cache = empty_cache(2, 16, 1, dim, dtype)
    first, lengths, table = _starts([len(firsts)]), _ints([len(firsts)]), _ints([[1]])
    rb.rb_cache8_append(cache, x, x, first, lengths, table)
    k, v = rb.rb_cache8_read(cache, first, lengths, table, len(firsts))
    torch.cuda.synchronize()
    values, units = oracle.held_in_8_bits(_f64(x), NAMES[dtype])
    for elements, exponents, back in ((cache.k, cache.k_exp, k), (cache.v, cache.v_exp, v)):
        got = elements[1].double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(values)) and np.array_equal(np.nan_to_num(got), np.nan_to_num(values))
        assert np.array_equal(exponents[1, 0].cpu().numpy(), units[:, 0])
        back = back[:, 0]
        assert torch.equal(torch.isfinite(back), torch.isfinite(x[:, 0]))      # what was finite is again
        ref = torch.from_numpy((np.nan_to_num(values) * np.exp2(units - 127.0)[..., None])[:, 0]).to(dtype).cuda()
        assert torch.equal(torch.nan_to_num(back, nan=0.0), ref)


@pytest.mark.parametrize("n_seqs", [1, 3, 63, 64, 130])
@pytest.mark.parametrize("unused", [-1, 1 << 20, -(1 << 31)])
def test_padding_and_bad_pages(n_seqs, unused):
    """Tokens behind the last sequence, and positions whose entry is no page: nothing is stored; read back, they are left as they are and zeros."""
    rng = synth.child_rng(611, n_seqs)
    page, kv, dim, heads, more = 16, 2, 64, 4, 21
    new = [1 + i % 3 for i in range(n_seqs)]
    lengths = [n + (16 - n if i % 2 else 5 * (i % 7)) for i, n in enumerate(new)]
    table, pages = _table(rng, lengths, page, unused=unused)
    bad = int(table[0, (lengths[0] - 1) // page])
    table[0, (lengths[0] - 1) // page] = unused      # the first sequence's last position has no page
    cache = empty_cache(pages, page, kv, dim, F16)
    t, first, now = sum(new), _starts(new), _ints(lengths)
    q, k, v = (_rand(rng, t + more, x, dim) for x in (heads, kv, kv))
    at = torch.from_numpy(table).cuda()
    q_out = rb.rb_cache8_append(cache, k, v, first, now, at, q=q, q_out=torch.full_like(q, 7.0))
    back = rb.rb_cache8_read(cache, first, now, at, t + more, *(torch.full((t + more, kv, dim), 7.0, dtype=F16, device="cuda") for _ in range(2)))
    torch.cuda.synchronize()
    assert torch.equal(q_out[:t], q[:t]) and (q_out[t:] == 7).all() and (cache.k_exp[bad] == 255).all() and torch.isnan(cache.k[bad].float()).all()
    for x, y in zip((k, v), back):
        values, units = oracle.held_in_8_bits(_f64(x[:t]), "fp16")
        ref = values * np.exp2(units - 127.0)[..., None]
        lost = [i for i in range(new[0]) if (lengths[0] - new[0] + i) // page == (lengths[0] - 1) // page]
        ref[lost] = 0
        assert np.array_equal(_f64(y[:t]), ref) and (y[t:] == 7).all()
    written = {(int(table[i, p // page]), p % page) for i, n in enumerate(new) for p in range(lengths[i] - n, lengths[i]) if table[i, p // page] != unused}
    mask = torch.zeros((pages, page), dtype=torch.bool)
    for w in written:
        mask[w] = True
    assert torch.isnan(cache.v.float().cpu()[~mask]).all() and (cache.v_exp.cpu().transpose(1, 2)[~mask] == 255).all()


# ------------------------------------------------------------- out of it ---
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("kv,dim,page,layout", [(8, 128, 16, "tokens"), (1, 64, 8, "tokens"), (3, 80, 64, "heads"), (2, 16, 128, "tokens"), (5, 96, 32, "heads"), (40, 112, 16, "tokens")])
def test_read(kv, dim, page, layout, dtype):
    rng = synth.child_rng(612, kv, dim)
    lengths = [1, 0, 77, 130, 16]
    cache, table, hold = build_cache(rng, lengths, page, kv, dim, dtype, layout, spread=3.0)
    for new in (lengths, [1, 0, 5, 70, 0]):
        k, v = rb.rb_cache8_read(cache, _starts(new), _ints(lengths), table, sum(new))
        torch.cuda.synchronize()
        for got, which in ((k, 0), (v, 1)):
            ref = torch.from_numpy(np.concatenate([hold[i][which][lengths[i] - n:] for i, n in enumerate(new)])).to(dtype)
            assert torch.equal(got.cpu(), ref), (new, which)


def test_read_every_code_in_every_unit():
    """256 codes times 256 units against 64 bits, in both types."""
    codes = torch.arange(256, dtype=torch.uint8).view(1, 1, 2, 128).repeat(4, 64, 1, 1)
    exps = torch.arange(256, dtype=torch.uint8).view(4, 1, 64).repeat(1, 2, 1)
    values = codes.view(E4M3).double() * torch.exp2(exps.double() - 127).transpose(1, 2)[..., None]
    for dtype in (F16, BF16):
        cache = rb.Cache8(*(codes.cuda().view(E4M3) for _ in range(2)), exps.cuda(), exps.cuda(), dtype)
        k, v = rb.rb_cache8_read(cache, _starts([255]), _ints([255]), _ints([[0, 1, 2, 3]]), 255)      # (byte 255: NaN)
        torch.cuda.synchronize()
        want = values.reshape(256, 2, 128)[:255].to(dtype).cuda()
        for got in (k, v):
            assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got, nan=0.0), torch.nan_to_num(want, nan=0.0))


# ------------------------------------------------------------- attention ---
def check(q, cache, table, hold, new, lengths, scale=None, label=""):
    d, g = q.shape[2], q.shape[1] // cache.kv_heads
    scale = d ** -0.5 if scale is None else scale
    got = rb.rb_attn_cache8(cache, q, _starts(new), _ints(lengths), table, scale=scale)
    torch.cuda.synchronize()
    Q, at = _f64(q), 0
    for i, n in enumerate(new):
        for h in range(q.shape[1]):
            ref, _, mag = oracle.attention(Q[at:at + n, h], hold[i][0][:, h // g], hold[i][1][:, h // g], _sees(n, max(lengths[i], 0), True), scale)
            _close(got[at:at + n, h], ref, mag, q.dtype, (label, i, n, lengths[i], h))
        at += n
    return got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads,kv,dim,page", [(4, 4, 128, 16), (16, 2, 128, 64), (6, 2, 64, 8), (12, 1, 96, 32), (10, 1, 48, 256), (2, 2, 16, 16), (3, 3, 80, 64), (12, 6, 112, 16), (5, 5, 32, 8),
                                                (16, 8, 128, 32), (40, 1, 64, 16), (7, 7, 128, 128)])
def test_attention(heads, kv, dim, page, dtype):
    for n, (new, lengths) in enumerate(PAGED):
        rng = synth.child_rng(620, heads, dim, n)
        print(heads, kv, dim, page, dtype, new, lengths, flush=True)
        cache, table, hold = build_cache(rng, lengths, page, kv, dim, dtype, layout="heads" if n % 2 else "tokens")
        check(_rand(rng, sum(new), heads, dim, dtype=dtype, gain=2.0), cache, table, hold, new, lengths, label=(heads, kv, dim, page, dtype))


def test_attention_over_long_contexts_and_many_sequences():
    rng = synth.child_rng(621)
    lengths = [int(x) for x in rng.integers(1, 400, 130)] + [20000, 9000]
    cache, table, hold = build_cache(rng, lengths, 16, 2, 64, F16)
    check(_rand(rng, len(lengths), 8, 64, gain=2.0), cache, table, hold, [1] * len(lengths), lengths)


def test_rows_that_see_nothing():
    rng = synth.child_rng(622)
    new, lengths = [4, 3, 90, 2], [2, 0, 30, -5]
    cache, table, hold = build_cache(rng, lengths, 16, 2, 64, F16)
    got = check(_rand(rng, sum(new), 4, 64), cache, table, hold, new, lengths)
    assert not got[:2].any() and not got[4:67].any() and not got[97:].any() and got[2:4].all(-1).any()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("unit", [False, True])
@pytest.mark.parametrize("new", [[1, 1, 1], [9, 1, 40]])
def test_masked_places(new, unit, dtype):
    """NaN in positions behind a row's own, in elements or by their unit's byte, leaves it as it is."""
    rng = synth.child_rng(623, len(new))
    lengths = [140, 64, 90]
    cache, table, hold = build_cache(rng, lengths, 16, 2, 128, dtype)
    q = _rand(rng, sum(new), 4, 128, dtype=dtype)
    clean = check(q, cache, table, hold, new, lengths)
    for i in range(3):      # the last position's key and value
        p = lengths[i] - 1
        page = int(table[i, p // 16])
        if unit:
            cache.k_exp[page, :, p % 16], cache.v_exp[page, :, p % 16] = 255, 255
        else:
            cache.k.view(torch.uint8)[page, p % 16, :, ::7], cache.v.view(torch.uint8)[page, p % 16] = 0x7f, 0xff
    got = rb.rb_attn_cache8(cache, q, _starts(new), _ints(lengths), table)
    torch.cuda.synchronize()
    last = [sum(new[:i + 1]) - 1 for i in range(3)]
    others = [i for i in range(sum(new)) if i not in last]
    assert torch.isnan(got[last]).all() and torch.equal(got[others], clean[others])


@pytest.mark.parametrize("new", [[1, 2], [70, 33]])
def test_a_nan_that_some_rows_see_in_a_value_alone(new):
    rng = synth.child_rng(624)
    lengths = [141, 90]
    cache, table, hold = build_cache(rng, lengths, 16, 2, 64, F16)
    at = lengths[1] - 2
    cache.v.view(torch.uint8)[int(table[1, at // 16]), at % 16, 1, 3] = 0x7f
    hold[1][1][at, 1, 3] = np.nan
    check(_rand(rng, sum(new), 4, 64), cache, table, hold, new, lengths)


@pytest.mark.parametrize("dtype,low,high", [(F16, -30, 12), (BF16, -110, 100)])
@pytest.mark.parametrize("new", [[1], [40]])
def test_units_over_the_types_whole_range(new, dtype, low, high):
    """Values whose units differ by many orders of magnitude, in one sequence."""
    rng = synth.child_rng(625)
    lengths = [300]
    cache, table, hold = build_cache(rng, lengths, 16, 1, 64, dtype, spread=0.0)
    for i in range(300):
        page, place, unit = int(table[0, i // 16]), i % 16, int(rng.integers(low, high + 1)) if i % 3 else low
        was = int(cache.v_exp[page, 0, place])
        cache.v_exp[page, 0, place] = 127 - 8 + unit
        hold[0][1][i] *= 2.0 ** (119 + unit - was)
    d = hold[0][1]
    rounded = torch.from_numpy(d).to(dtype).double().numpy()      # below fp16's normal range values are rounded where they are read
    hold[0][1] = rounded if dtype == F16 else d
    check(_rand(rng, sum(new), 2, 64, dtype=dtype), cache, table, hold, new, lengths)


def test_offsets_beyond_32_bits():
    """A cache of more than 4 GiB per array, its first and its last pages in use, written, read back and attended to."""
    rng = synth.child_rng(626)
    page, kv, dim, pages = 128, 8, 128, 33000
    cache = rb.Cache8(*(torch.empty((pages, page, kv, dim), dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2)),
                      *(torch.empty((pages, kv, page), dtype=torch.uint8, device="cuda") for _ in range(2)))
    assert cache.k.numel() > 1 << 32
    lengths, table = [300, 130], _ints([[pages - 1, 0, pages - 2], [pages // 2, 32768, 5]])
    t, first, now = 430, _starts([300, 130]), _ints([300, 130])
    x, y = _rand(rng, t, kv, dim), _rand(rng, t, kv, dim)
    rb.rb_cache8_append(cache, x, y, first, now, table)
    k, v = rb.rb_cache8_read(cache, first, now, table, t)
    torch.cuda.synchronize()
    hold = [[], []]
    for given, got in ((x, k), (y, v)):
        values, units = oracle.held_in_8_bits(_f64(given), "fp16")
        ref = values * np.exp2(units - 127.0)[..., None]
        assert np.array_equal(_f64(got), ref)
        hold[0].append(ref[:300]), hold[1].append(ref[300:])
    for new in ([1, 1], [70, 33]):
        check(_rand(rng, sum(new), 16, dim), cache, table, hold, new, lengths)


def test_in_a_graph_and_on_another_stream():
    """Entering, attention and reading back captured once, two graphs over one workspace, replayed with other lengths and other contents."""
    rng = synth.child_rng(627)
    lengths = [200, 777]
    cache, table, hold = build_cache(rng, lengths, 16, 2, 128, F16)
    q = _rand(rng, 2, 8, 128)
    first, now = _starts([1, 1]), _ints(lengths)
    new_k, new_v = _rand(rng, 2, 2, 128), _rand(rng, 2, 2, 128)
    ws = torch.empty(rb.lib.rb_attn_cache8_workspace_bytes(ctypes.byref(cache.struct()), 8, 2, 2), dtype=torch.uint8, device="cuda")
    rb.rb_attn_cache8(cache, q, first, now, table, workspace=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for graph in graphs:
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            rb.rb_cache8_append(cache, new_k, new_v, first, now, table)
            outs.append((rb.rb_attn_cache8(cache, q, first, now, table, workspace=ws), *rb.rb_cache8_read(cache, first, now, table, 2)))
    for i in range(4):
        now.copy_(_ints([100 + 7 * i, 700 - 60 * i]))
        new_k.copy_(_rand(rng, 2, 2, 128))
        torch.cuda.synchronize()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        want = (rb.rb_attn_cache8(cache, q, first, now, table), *rb.rb_cache8_read(cache, first, now, table, 2))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[i % 2], want))
        values, units = oracle.held_in_8_bits(_f64(new_k), "fp16")
        assert np.array_equal(_f64(want[1]), values * np.exp2(units - 127.0)[..., None])


def test_arrays_out_of_order_stay_inside():
    """Wrong arrays give wrong results and nothing else (the cache's own memory is one buffer with guards around it)."""
    rng = synth.child_rng(628)
    cache, table, _ = build_cache(rng, [40, 40, 40], 16, 2, 64, F16)
    q, x = _rand(rng, 9, 4, 64), _rand(rng, 9, 2, 64)
    for first, lengths in (([5, 2, 9, 1], [40, 40, 40]), ([0, 1, 2, 9], [1 << 30, -7, 2000000000]), ([0, 100, -3, 9], [40, 3, 4])):
        first, lengths = _ints(first), _ints(lengths)
        out = torch.full((11, 4, 64), 7.0, dtype=F16, device="cuda")
        rb.rb_cache8_append(cache, x, x, first, lengths, table)
        rb.rb_attn_cache8(cache, q, first, lengths, table, o=out[1:10])
        k, v = (torch.full((11, 2, 64), 7.0, dtype=F16, device="cuda") for _ in range(2))
        rb.rb_cache8_read(cache, first, lengths, table, 9, k[1:10], v[1:10])
        torch.cuda.synchronize()
        for y in (out, k, v):
            assert (y[0] == 7).all() and (y[10] == 7).all()
