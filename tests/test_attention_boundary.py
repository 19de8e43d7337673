"""CPU-only: attention and cache entry points turn bad arguments into status codes before anything is enqueued, and the
oracle's attention and its gradient are what they say."""
import ctypes

import numpy as np
import pytest

import oracle
import synth
import paper_2602_05367_amd as rb


def _H(**kw):
    f = dict(heads=4, kv_heads=2, dim=64, dtype=rb.RB_F16, q_token=256, q_head=64, k_token=128, k_head=64, v_token=128, v_head=64)
    f.update(kw)
    return ctypes.byref(rb.binding.rb_heads(**f))


def _C(**kw):
    f = dict(k=0x1000, v=0x2000, pages=4, page_tokens=16, kv_heads=2, dim=64, dtype=rb.RB_F16, page_stride=2048, token_stride=128, head_stride=64)
    f.update(kw)
    return ctypes.byref(rb.binding.rb_cache(**f))


BAD_HEADS = [(dict(heads=3), rb.RB_ERR_SHAPE), (dict(heads=0), rb.RB_ERR_SHAPE), (dict(kv_heads=0), rb.RB_ERR_SHAPE), (dict(dim=60), rb.RB_ERR_SHAPE),
             (dict(dim=0), rb.RB_ERR_SHAPE), (dict(dim=136), rb.RB_ERR_UNSUPPORTED), (dict(dtype=rb.RB_F32), rb.RB_ERR_UNSUPPORTED),
             (dict(dtype=9), rb.RB_ERR_UNSUPPORTED), (dict(q_token=-8), rb.RB_ERR_SHAPE), (dict(k_head=1 << 26), rb.RB_ERR_SHAPE), (dict(v_token=100), rb.RB_ERR_ALIGN)]
BAD_CACHE = [(dict(k=0), rb.RB_ERR_NULL), (dict(v=0), rb.RB_ERR_NULL), (dict(pages=0), rb.RB_ERR_SHAPE), (dict(page_tokens=4), rb.RB_ERR_SHAPE),
             (dict(page_tokens=24), rb.RB_ERR_SHAPE), (dict(page_tokens=1 << 17), rb.RB_ERR_SHAPE), (dict(kv_heads=0), rb.RB_ERR_SHAPE), (dict(dim=20), rb.RB_ERR_SHAPE),
             (dict(dim=256), rb.RB_ERR_UNSUPPORTED), (dict(dtype=rb.RB_F32), rb.RB_ERR_UNSUPPORTED), (dict(page_stride=-8), rb.RB_ERR_SHAPE),
             (dict(token_stride=1 << 26), rb.RB_ERR_SHAPE), (dict(head_stride=4), rb.RB_ERR_ALIGN), (dict(k=0x1008), rb.RB_ERR_ALIGN)]


def _prompt(H=None, q=0x100, k=0x200, v=0x300, first=0x400, first_k=None, n=1, tq=8, tk=8, scale=0.1, o=0x500, lse=None):
    return rb.lib.rb_attn_prompt(H or _H(), q, k, v, first, first_k, n, tq, tk, 1, scale, o, lse, None)


def test_prompt_refusals():
    assert rb.lib.rb_attn_prompt(None, 0x100, 0x200, 0x300, 0x400, None, 1, 8, 8, 1, 0.1, 0x500, None, None) == rb.RB_ERR_NULL
    for kw, code in BAD_HEADS:
        assert _prompt(H=_H(**kw)) == code, kw
    for name in ("q", "k", "v", "first", "o"):
        assert _prompt(**{name: None}) == rb.RB_ERR_NULL, name
    for kw in (dict(n=0), dict(n=(1 << 20) + 1), dict(tq=0), dict(tk=-1, first_k=0x600), dict(tk=9), dict(tq=(1 << 24) + 1, tk=(1 << 24) + 1)):
        assert _prompt(**kw) == rb.RB_ERR_SHAPE, kw
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert _prompt(scale=scale) == rb.RB_ERR_VALUE
    for kw in (dict(q=0x108), dict(k=0x202), dict(v=0x304), dict(o=0x508), dict(first=0x402), dict(lse=0x701), dict(first_k=0x602)):
        assert _prompt(**kw) == rb.RB_ERR_ALIGN, kw


def _grad(H=None, go=0x100, q=0x200, k=0x300, v=0x400, o=0x500, lse=0x600, first=0x700, first_k=None, n=1, tq=8, tk=8, scale=0.1, dq=0x800, dk=0x900, dv=0xa00,
          ws=0x1000, size=1 << 30):
    return rb.lib.rb_attn_prompt_grad(H or _H(), go, q, k, v, o, lse, first, first_k, n, tq, tk, 1, scale, dq, dk, dv, ws, size, None)


def test_gradient_refusals():
    for kw, code in BAD_HEADS:
        assert _grad(H=_H(**kw)) == code, kw
    for name in ("go", "q", "k", "v", "o", "lse", "first", "dq", "dk", "dv"):
        assert _grad(**{name: None}) == rb.RB_ERR_NULL, name
    for kw in (dict(n=0), dict(tq=0, tk=0), dict(tk=9), dict(tk=0, first_k=0xb00), dict(tq=(1 << 24) + 1, tk=(1 << 24) + 1)):
        assert _grad(**kw) == rb.RB_ERR_SHAPE, kw
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert _grad(scale=scale) == rb.RB_ERR_VALUE
    for name in ("go", "q", "k", "v", "o", "dq", "dk", "dv"):
        assert _grad(**{name: 0x108}) == rb.RB_ERR_ALIGN, name
    assert _grad(lse=0x602) == rb.RB_ERR_ALIGN and _grad(first=0x701) == rb.RB_ERR_ALIGN and _grad(ws=0x1004) == rb.RB_ERR_ALIGN
    need = rb.lib.rb_attn_grad_workspace_bytes(_H(), 8, 8)
    assert need >= 8 * 4 * 4 and _grad(size=need - 1) == rb.RB_ERR_WORKSPACE and _grad(ws=None) == rb.RB_ERR_WORKSPACE
    assert rb.lib.rb_attn_grad_workspace_bytes(None, 8, 8) == 0 and rb.lib.rb_attn_grad_workspace_bytes(_H(), 0, 8) == 0


def _paged(C=None, q=0x100, qt=256, qh=64, heads=4, first=0x400, lengths=0x500, table=0x600, width=3, n=2, tokens=2, scale=0.1, o=0x700, ws=0x8000, size=1 << 40):
    return rb.lib.rb_attn_paged(C or _C(), q, qt, qh, heads, first, lengths, table, width, n, tokens, scale, o, ws, size, None)


def test_paged_refusals():
    assert rb.lib.rb_attn_paged(None, 0x100, 256, 64, 4, 0x400, 0x500, 0x600, 3, 2, 2, 0.1, 0x700, 0x8000, 1 << 40, None) == rb.RB_ERR_NULL
    for kw, code in BAD_CACHE:
        assert _paged(C=_C(**kw)) == code, kw
    for name in ("q", "first", "lengths", "table", "o"):
        assert _paged(**{name: None}) == rb.RB_ERR_NULL, name
    for kw in (dict(heads=3), dict(heads=0), dict(qt=-8), dict(width=0), dict(n=0), dict(tokens=0), dict(tokens=(1 << 24) + 1)):
        assert _paged(**kw) == rb.RB_ERR_SHAPE, kw
    assert _paged(scale=0.0) == rb.RB_ERR_VALUE
    for kw in (dict(q=0x108), dict(qt=100), dict(o=0x704), dict(first=0x402), dict(lengths=0x501), dict(table=0x603), dict(ws=0x8008)):
        assert _paged(**kw) == rb.RB_ERR_ALIGN, kw
    need = rb.lib.rb_attn_paged_workspace_bytes(_C(), 4, 2, 2)
    if need:
        assert _paged(size=need - 1) == rb.RB_ERR_WORKSPACE and _paged(ws=None) == rb.RB_ERR_WORKSPACE
    assert rb.lib.rb_attn_paged_workspace_bytes(None, 4, 2, 2) == 0 and rb.lib.rb_attn_paged_workspace_bytes(_C(), 3, 2, 2) == 0


def _append(C=None, H=None, q=0x100, k=0x200, v=0x300, cos=0x400, sin=0x500, rows=9, rotary=64, first=0x600, lengths=0x700, table=0x800, width=2, n=1, tokens=3,
            q_out=0x900):
    return rb.lib.rb_cache_append(C or _C(), H or _H(), q, k, v, cos, sin, rows, rotary, 0, first, lengths, table, width, n, tokens, q_out, None)


def test_append_refusals():
    for kw, code in BAD_CACHE:
        assert _append(C=_C(**kw)) == code, kw
    for kw, code in BAD_HEADS:
        assert _append(H=_H(**kw)) == code, kw
    assert rb.lib.rb_cache_append(_C(), None, 0x100, 0x200, 0x300, None, None, 0, 0, 0, 0x600, 0x700, 0x800, 2, 1, 3, 0x900, None) == rb.RB_ERR_NULL
    for name in ("q", "k", "v", "cos", "sin", "first", "lengths", "table", "q_out"):
        assert _append(**{name: None}) == rb.RB_ERR_NULL, name
    for kw in (dict(H=_H(heads=4, kv_heads=4)), dict(H=_H(dim=32)), dict(H=_H(dtype=rb.RB_BF16)), dict(rows=0), dict(rotary=0), dict(rotary=12), dict(rotary=72),
               dict(width=0), dict(n=0), dict(tokens=0)):
        assert _append(**kw) == rb.RB_ERR_SHAPE, kw
    for kw in (dict(q=0x104), dict(k=0x208), dict(v=0x302), dict(cos=0x404), dict(sin=0x508), dict(q_out=0x908), dict(first=0x601), dict(table=0x802)):
        assert _append(**kw) == rb.RB_ERR_ALIGN, kw


# ------------------------------------------------------------ the oracle ---
def test_oracle_attention_by_hand():
    q, k, v = np.array([[1.0], [2.0]]), np.array([[0.0], [np.log(3.0)]]), np.array([[4.0], [8.0]])
    o, lse, _ = oracle.attention(q, k, v, [1, 2], 1.0)
    assert np.allclose(o, [[4.0], [(4 + 9 * 8) / 10]]) and np.allclose(lse, [0.0, np.log(10.0)])
    o, lse, _ = oracle.attention(q, k, v, [0, -3], 1.0)
    assert not o.any() and np.isneginf(lse).all()
    v[1] = np.nan
    assert oracle.attention(q, k, v, [1, 2], 1.0)[0][0] == 4.0


def test_oracle_gradient_against_differences():
    rng = synth.child_rng(330)
    n, m, d, scale, sees = 5, 7, 4, 0.6, [0, 1, 4, 7, 7]
    q, k, v, do = (rng.standard_normal(s) for s in ((n, d), (m, d), (m, d), (n, d)))
    (dq, dk, dv), wide = oracle.attention_grad(do, q, k, v, sees, scale)
    loss = lambda: float((oracle.attention(q, k, v, sees, scale)[0] * do).sum())
    for x, g in ((q, dq), (k, dk), (v, dv)):
        for i in np.ndindex(*x.shape):
            keep, e = x[i], 1e-6
            x[i] = keep + e
            up = loss()
            x[i] = keep - e
            down = loss()
            x[i] = keep
            assert abs((up - down) / (2 * e) - g[i]) < 1e-8
    assert all((np.abs(g) <= w + 1e-15).all() for g, w in zip((dq, dk, dv), wide))


@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_rotary_is_a_turn(interleaved):
    rng = synth.child_rng(331)
    x, angle = rng.standard_normal((3, 10)), rng.uniform(-3, 3, 4)
    y = oracle.rotary(x, np.cos(angle), np.sin(angle), interleaved)
    pairs = [(2 * i, 2 * i + 1) if interleaved else (i, i + 4) for i in range(4)]
    for t, (a, b) in zip(angle, pairs):
        z = (x[:, a] + 1j * x[:, b]) * np.exp(1j * t)
        assert np.allclose(y[:, a], z.real) and np.allclose(y[:, b], z.imag)
    assert np.array_equal(y[:, 8:], x[:, 8:])
