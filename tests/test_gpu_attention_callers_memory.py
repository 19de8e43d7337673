"""A caller's own workspace: its bytes count whatever its type, and one that is not device memory, or too small, is refused."""
import ctypes

import pytest
import torch

import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import F16, _rand, _starts

pytestmark = pytest.mark.gpu


def test_workspaces_of_other_types_and_places():
    rng = synth.child_rng(410)
    cache = rb.Cache(*(_rand(rng, 8, 16, 2, 64) for _ in range(2)))
    table, first, lengths = torch.arange(8, dtype=torch.int32).view(2, 4).cuda(), _starts([1, 1]), torch.tensor([50, 9], dtype=torch.int32).cuda()
    q = _rand(rng, 2, 4, 64)
    need = rb.lib.rb_attn_paged_workspace_bytes(ctypes.byref(cache.struct()), 4, 2, 2)
    want = rb.rb_attn_paged(cache, q, first, lengths, table)
    for dtype in (torch.uint8, torch.float16, torch.float32, torch.int64):
        ws = torch.empty(-(-need // dtype.itemsize), dtype=dtype, device="cuda")
        assert torch.equal(rb.rb_attn_paged(cache, q, first, lengths, table, workspace=ws), want), dtype
    for ws in (torch.empty(need, dtype=torch.uint8), torch.empty(need, dtype=torch.uint8).pin_memory(), torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(AssertionError):
            rb.rb_attn_paged(cache, q, first, lengths, table, workspace=ws)
    with pytest.raises(rb.RabitError):
        rb.rb_attn_paged(cache, q, first, lengths, table, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
