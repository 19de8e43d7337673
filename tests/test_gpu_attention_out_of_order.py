"""Arrays that are not in order give wrong results, but nothing outside the buffers is touched: sequences that start behind a call's first tokens, overlap, or
have lengths of any value, for fewer sequences than a wavefront has lanes and for more."""
import pytest
import torch

import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import F16, _rand, build_cache

pytestmark = pytest.mark.gpu
KEPT = 7.0


def _ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("more", [0, 90])      # sequences of no tokens behind the others
@pytest.mark.parametrize("first,lengths", [([5, 2, 9, 1], [40, 40, 40]), ([3, 3, 3, 9], [40, 40, 40]), ([0, 1, 2, 9], [1 << 30, -7, 2000000000]), ([0, 100, -3, 9], [40, 3, 4]),
                                           ([100, 100, 100, 100], [40, 40, 40]), ([-5, -4, -3, -2], [40, 40, 40])])
def test_cache_and_prompts(first, lengths, more):
    rng = synth.child_rng(380, more)
    cache, table, _ = build_cache(rng, lengths=[40, 40, 40] + [0] * more, page=16, kv=2, dim=64, dtype=F16)
    q, x = _rand(rng, 9, 4, 64), _rand(rng, 9, 2, 64)
    starts, lengths = _ints(first + first[-1:] * more), _ints(lengths + [0] * more)
    outs = [torch.full((11, 4, 64), KEPT, dtype=F16, device="cuda") for _ in range(3)]
    rb.rb_cache_append(cache, x, x, starts, lengths, table, q=q, q_out=outs[0][1:10])
    rb.rb_attn_paged(cache, q, starts, lengths, table, o=outs[1][1:10])
    rb.rb_attn_prompt(q, x, x, starts, o=outs[2][1:10])
    torch.cuda.synchronize()
    for o in outs:
        assert (o[0] == KEPT).all() and (o[10] == KEPT).all()
