"""CPU-only: calls of attention whose blocks of rows are more than one launch has workgroups for are refused before any part of them is enqueued."""
import pytest

import paper_2602_05367_amd as rb
from test_attention_boundary import _C, _H, _grad, _paged, _prompt
from test_cache8_boundary import _C as _C8, _attn


def _heads(heads, kv):
    return _H(heads=heads, kv_heads=kv, q_token=heads * 64, k_token=kv * 64, v_token=kv * 64)


# single tokens (by the kernel for few rows), several (by the other)
@pytest.mark.parametrize("heads,kv,n,tokens", [(32, 32, 1 << 20, 1 << 20), (16, 16, 1 << 20, 1 << 20), (64, 16, 1 << 20, 1 << 24), (4096, 4096, 5000, 5000), (65536, 65536, 1, 1 << 20)])
def test_more_blocks_than_workgroups(heads, kv, n, tokens):
    cache = dict(kv_heads=kv, page_stride=16 * kv * 64, token_stride=kv * 64, head_stride=64)
    big = dict(size=1 << 60)
    assert _paged(C=_C(**cache), heads=heads, qt=heads * 64, n=n, tokens=tokens, **big) == rb.RB_ERR_SHAPE
    assert _attn(C=_C8(**cache), heads=heads, q_token=heads * 64, n=n, tokens=tokens, **big) == rb.RB_ERR_SHAPE
    assert _prompt(H=_heads(heads, kv), n=n, tq=tokens, tk=tokens) == rb.RB_ERR_SHAPE
    assert _grad(H=_heads(heads, kv), n=n, tq=tokens, tk=tokens, **big) == rb.RB_ERR_SHAPE


def test_gradients_of_half_as_many():
    """Workgroups of twice the threads."""
    assert _grad(H=_heads(8, 8), n=1 << 20, tq=1 << 20, tk=1 << 20, size=1 << 60) == rb.RB_ERR_SHAPE
