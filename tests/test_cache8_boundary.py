"""CPU-only: the entry points of the cache in 8 bits and of sampling turn bad arguments into status codes before anything is enqueued, and the oracle
holds heads and draws tokens as it says."""
import ctypes
import math

import numpy as np
import pytest
import torch

import oracle
import synth
import paper_2602_05367_amd as rb


def _H(**kw):
    f = dict(heads=4, kv_heads=2, dim=64, dtype=rb.RB_F16, q_token=256, q_head=64, k_token=128, k_head=64, v_token=128, v_head=64)
    f.update(kw)
    return ctypes.byref(rb.binding.rb_heads(**f))


def _C(**kw):
    f = dict(k=0x1000, v=0x2000, k_exp=0x3000, v_exp=0x3800, pages=4, page_tokens=16, kv_heads=2, dim=64, dtype=rb.RB_F16, page_stride=2048, token_stride=128, head_stride=64)
    f.update(kw)
    return ctypes.byref(rb.binding.rb_cache8(**f))


BAD_CACHE = [(dict(k=0), rb.RB_ERR_NULL), (dict(v=0), rb.RB_ERR_NULL), (dict(k_exp=0), rb.RB_ERR_NULL), (dict(v_exp=0), rb.RB_ERR_NULL), (dict(pages=0), rb.RB_ERR_SHAPE),
             (dict(page_tokens=4), rb.RB_ERR_SHAPE), (dict(page_tokens=24), rb.RB_ERR_SHAPE), (dict(page_tokens=1 << 17), rb.RB_ERR_SHAPE), (dict(kv_heads=0), rb.RB_ERR_SHAPE),
             (dict(dim=20), rb.RB_ERR_SHAPE), (dict(dim=72), rb.RB_ERR_UNSUPPORTED), (dict(dim=144), rb.RB_ERR_UNSUPPORTED), (dict(dtype=rb.RB_F32), rb.RB_ERR_UNSUPPORTED),
             (dict(page_stride=-16), rb.RB_ERR_SHAPE), (dict(token_stride=48), rb.RB_ERR_SHAPE), (dict(token_stride=0), rb.RB_ERR_SHAPE), (dict(token_stride=1 << 26), rb.RB_ERR_SHAPE),
             (dict(head_stride=72), rb.RB_ERR_ALIGN), (dict(token_stride=136), rb.RB_ERR_ALIGN), (dict(k=0x1008), rb.RB_ERR_ALIGN), (dict(v_exp=0x3804), rb.RB_ERR_ALIGN)]


def _append(C=None, H=None, q=0x100, k=0x200, v=0x300, cos=0x400, sin=0x500, rows=9, rotary=64, first=0x600, lengths=0x700, table=0x800, width=3, n=2, tokens=5, q_out=0x900):
    return rb.lib.rb_cache8_append(C or _C(), H or _H(), q, k, v, cos, sin, rows, rotary, 0, first, lengths, table, width, n, tokens, q_out, None)


def _read(C=None, first=0x600, lengths=0x700, table=0x800, width=3, n=2, tokens=5, k=0x100, v=0x200):
    return rb.lib.rb_cache8_read(C or _C(), first, lengths, table, width, n, tokens, k, v, None)


def _attn(C=None, q=0x100, q_token=256, q_head=64, heads=4, first=0x600, lengths=0x700, table=0x800, width=3, n=2, tokens=5, scale=0.1, o=0x900, ws=0x1000, size=1 << 30):
    return rb.lib.rb_attn_cache8(C or _C(), q, q_token, q_head, heads, first, lengths, table, width, n, tokens, scale, o, ws, size, None)


@pytest.mark.parametrize("call", [_append, _read, _attn])
def test_refusals_of_caches_and_sequences(call):
    for kw, code in BAD_CACHE:
        # (tokens of a head count that the cache does not have come later)
        assert call(C=_C(**kw)) == code, kw
    for kw in (dict(n=0), dict(n=(1 << 20) + 1), dict(tokens=0), dict(tokens=(1 << 24) + 1), dict(width=0)):
        assert call(**kw) == rb.RB_ERR_SHAPE, kw
    for name in ("first", "lengths", "table"):
        assert call(**{name: None}) == rb.RB_ERR_NULL and call(**{name: 0x602}) == rb.RB_ERR_ALIGN, name


def test_append_refusals():
    assert rb.lib.rb_cache8_append(None, _H(), 0x100, 0x200, 0x300, None, None, 0, 0, 0, 0x600, 0x700, 0x800, 3, 2, 5, 0x900, None) == rb.RB_ERR_NULL
    for kw in (dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(cos=None), dict(sin=None)):
        assert _append(**kw) == rb.RB_ERR_NULL, kw
    for kw in (dict(H=_H(kv_heads=4)), dict(H=_H(dim=128)), dict(H=_H(dtype=rb.RB_BF16)), dict(rows=0), dict(rotary=4), dict(rotary=60), dict(rotary=72)):
        assert _append(**kw) == rb.RB_ERR_SHAPE, kw
    for name in ("q", "k", "v", "q_out", "cos", "sin"):
        assert _append(**{name: 0x108}) == rb.RB_ERR_ALIGN, name


def test_read_refusals():
    assert _read(k=None) == rb.RB_ERR_NULL and _read(v=None) == rb.RB_ERR_NULL and _read(k=0x108) == rb.RB_ERR_ALIGN and _read(v=0x202) == rb.RB_ERR_ALIGN


def test_attention_refusals():
    for kw in (dict(q=None), dict(o=None)):
        assert _attn(**kw) == rb.RB_ERR_NULL, kw
    for kw in (dict(heads=3), dict(heads=0), dict(q_token=-8)):
        assert _attn(**kw) == rb.RB_ERR_SHAPE, kw
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert _attn(scale=scale) == rb.RB_ERR_VALUE
    for kw in (dict(q=0x108), dict(o=0x902), dict(q_token=100), dict(ws=0x1004)):
        assert _attn(**kw) == rb.RB_ERR_ALIGN, kw
    need = rb.lib.rb_attn_cache8_workspace_bytes(_C(), 4, 2, 5)
    assert need > 0 and _attn(size=need - 1) == rb.RB_ERR_WORKSPACE and _attn(ws=None) == rb.RB_ERR_WORKSPACE
    # so many serve every smaller call
    sizes = [(n, tokens) for n in (1, 2, 3, 200) for tokens in (1, 5, 201, 700)]
    for n, tokens in sizes:
        most = rb.lib.rb_attn_cache8_workspace_bytes(_C(), 4, n, tokens)
        assert all(rb.lib.rb_attn_cache8_workspace_bytes(_C(), 4, a, b) <= most for a, b in sizes if a <= n and b <= tokens)
    assert rb.lib.rb_attn_cache8_workspace_bytes(_C(dim=72), 4, 2, 5) == 0


def _sample(logits=0x100, dtype=rb.RB_F16, stride=50, rows=3, vocab=50, u=0x200, temperature=0x300, top_k=0x400, top_p=0x500, min_p=0x600, tokens=0x700, ws=0x1000, size=1 << 30):
    return rb.lib.rb_sample(logits, dtype, stride, rows, vocab, u, temperature, top_k, top_p, min_p, tokens, ws, size, None)


def test_sample_refusals():
    for name in ("logits", "u", "tokens"):
        assert _sample(**{name: None}) == rb.RB_ERR_NULL, name
    assert _sample(dtype=3) == rb.RB_ERR_UNSUPPORTED and _sample(dtype=-1) == rb.RB_ERR_UNSUPPORTED
    for kw in (dict(rows=0), dict(rows=(1 << 20) + 1), dict(vocab=0, stride=0), dict(vocab=(1 << 22) + 1, stride=1 << 23), dict(stride=49), dict(stride=1 << 40), dict(stride=-1)):
        assert _sample(**kw) == rb.RB_ERR_SHAPE, kw
    assert _sample(logits=0x101) == rb.RB_ERR_ALIGN and _sample(logits=0x102, dtype=rb.RB_F32) == rb.RB_ERR_ALIGN
    for name in ("u", "temperature", "top_k", "top_p", "min_p", "tokens"):
        assert _sample(**{name: 0x202}) == rb.RB_ERR_ALIGN, name
    need = rb.lib.rb_sample_workspace_bytes(rb.RB_F16, 3, 400000)
    large = dict(vocab=400000, stride=400000)
    assert need > 0 and _sample(size=need - 1, **large) == rb.RB_ERR_WORKSPACE and _sample(ws=None, **large) == rb.RB_ERR_WORKSPACE and _sample(ws=0x1008, **large) == rb.RB_ERR_ALIGN
    # so many serve every smaller call
    sizes = [(dtype, rows, vocab) for dtype in (rb.RB_F16, rb.RB_F32) for rows in (1, 3, 40, 300, 1 << 20) for vocab in (1, 5000, 40000, 400000, 1 << 22)]
    for dtype, rows, vocab in sizes:
        most = rb.lib.rb_sample_workspace_bytes(dtype, rows, vocab)
        assert all(rb.lib.rb_sample_workspace_bytes(d, r, v) <= most for d, r, v in sizes if d == dtype and r <= rows and v <= vocab)
    assert rb.lib.rb_sample_workspace_bytes(rb.RB_F16, 0, 5) == rb.lib.rb_sample_workspace_bytes(5, 1, 400000) == 0


def test_binding_refuses_host_tensors_and_wrong_types():
    with pytest.raises(AssertionError):
        rb.Cache8(*(torch.zeros(2, 16, 2, 64, dtype=torch.uint8).view(torch.float8_e4m3fn) for _ in range(2)), *(torch.zeros(2, 2, 16, dtype=torch.uint8) for _ in range(2)))
    with pytest.raises(AssertionError):
        rb.rb_sample(torch.zeros(2, 9), torch.zeros(2))


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_oracle_holds_heads_as_torch_rounds_them(dtype):
    rng = synth.child_rng(600)
    x = torch.from_numpy(rng.standard_normal((500, 32)) * np.exp2(rng.integers(-20, 12, (500, 1)))).to(torch.float16 if dtype == "fp16" else torch.bfloat16)
    values, exponents = oracle.held_in_8_bits(x.double().numpy(), dtype)
    most = x.double().abs().amax(1).numpy() / np.exp2(exponents - 127.0)
    assert ((most > 224) & (most <= 448)).all()
    assert np.array_equal(values, (x.double() / torch.from_numpy(np.exp2(exponents - 127.0))[:, None]).float().to(torch.float8_e4m3fn).double().numpy())
    # the edges: the largest, zeros, infinities beside others, what one unit more would hold
    large = 65504.0 if dtype == "fp16" else float(torch.finfo(torch.bfloat16).max)
    x = np.array([[large, 1.0], [0.0, 0.0], [np.inf, 1.75], [np.nan, 1.7578125], [2.0 ** -133, 0.0]])
    values, exponents = oracle.held_in_8_bits(x, dtype)
    held = values * np.exp2(exponents - 127.0)[:, None]
    assert held[0, 0] == oracle.LARGEST_HELD[dtype] < large and not held[1].any() and exponents[1] == 1
    assert np.isnan(held[2, 0]) and values[2, 1] == 448 and values[3, 1] == 224 and exponents[4] == 1


def test_oracle_draws_as_it_says():
    x = np.log([0.1, 0.4, 0.3, 0.2])
    assert [oracle.next_token(x, u) for u in (0.0, 0.099, 0.101, 0.499, 0.501, 0.799, 0.801, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [oracle.next_token(x, u, top_k=2) for u in (0.0, 0.57, 0.58, 0.99)] == [1, 1, 2, 2]
    assert [oracle.next_token(x, u, top_p=0.75) for u in (0.0, 0.44, 0.45, 0.77, 0.78, 0.99)] == [1, 1, 2, 2, 3, 3]
    assert {oracle.next_token(x, u, top_p=0.39) for u in np.linspace(0, 0.99, 9)} == {1}
    assert {oracle.next_token(x, u, min_p=0.7) for u in np.linspace(0, 0.99, 9)} == {1, 2}
    assert oracle.next_token(x, 0.9, temperature=0.0) == 1 and oracle.next_token([-math.inf, math.nan], 0.5) == -1
    assert [oracle.next_token([1.0, math.inf, math.nan, math.inf], u) for u in (0.1, 0.6)] == [1, 3]
    assert [oracle.next_token([2.0, 2.0, 2.0], u, top_k=2) for u in (0.1, 0.6)] == [0, 1]
