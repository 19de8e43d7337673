"""CPU-only: the workspaces of attention over the cache and of its gradient are bounds: what serves a call serves every smaller one."""
import ctypes

import pytest

import paper_2602_05367_amd as rb

SIZES = [1, 2, 7, 8, 31, 32, 33, 127, 128, 129, 512, 2000, 4096, 30000, 1 << 20, 1 << 24]
HEADS = [(32, 8, 128), (32, 32, 128), (64, 8, 64), (16, 1, 128), (40, 40, 96), (128, 1, 128), (8, 8, 8), (2048, 2048, 64)]


@pytest.mark.parametrize("heads,kv,dim", HEADS)
def test_paged(heads, kv, dim):
    C = rb.binding.rb_cache(0x1000, 0x2000, 4, 16, kv, dim, rb.RB_F16, 16 * kv * dim, kv * dim, dim)
    need = {(n, t): rb.lib.rb_attn_paged_workspace_bytes(ctypes.byref(C), heads, n, t) for n in SIZES if n <= 1 << 20 for t in SIZES}
    for (n, t), size in need.items():
        assert all(size >= need[a, b] for a, b in need if a <= n and b <= t), (n, t)
    assert need[1 << 20, 1] > 0


@pytest.mark.parametrize("heads,kv,dim", HEADS)
def test_gradient(heads, kv, dim):
    H = ctypes.byref(rb.binding.rb_heads(heads, kv, dim, rb.RB_F16, heads * dim, dim, kv * dim, dim, kv * dim, dim))
    need = {(q, k): rb.lib.rb_attn_grad_workspace_bytes(H, q, k) for q in SIZES for k in SIZES}
    for (q, k), size in need.items():
        assert size >= q * heads * 4 and all(size >= need[a, b] for a, b in need if a <= q and b <= k), (q, k)
