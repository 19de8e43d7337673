"""The cache in 8 bits under arrays that are not in order: wrong results, and nothing else.  Each of the cache's four arrays lies in a buffer of its own with more than a page of known
bytes before and behind it; those, pages that no sequence has, and the rows around every result are as they were afterwards.  For fewer sequences than a wavefront has lanes and for more."""
import pytest
import torch

import synth
import paper_2602_05367_amd as rb
from test_gpu_attention import F16, _rand
from test_gpu_cache8 import E4M3, _ints, _table

pytestmark = pytest.mark.gpu
KEPT = 7.0


class Guarded:
    """Bytes of a pattern, in the middle of them an array of `shape`."""

    def __init__(self, shape, seed):
        n = 1
        for x in shape:
            n *= x
        self.edge = (n // shape[0] + 4096) // 16 * 16      # a page and more
        self.all = torch.randint(0, 126, (n + 2 * self.edge,), dtype=torch.uint8, generator=torch.Generator().manual_seed(seed)).cuda()
        self.array = self.all[self.edge:self.edge + n].view(shape)
        self.was = self.all.clone()

    def check(self, pages, label):
        """`pages`: those that may have changed."""
        now, was = self.all[:self.edge], self.was[:self.edge]
        assert torch.equal(now, was), (label, "before")
        end = self.edge + self.array.numel()
        assert torch.equal(self.all[end:], self.was[end:]), (label, "behind")
        kept = [p for p in range(self.array.shape[0]) if p not in pages]
        before = self.was[self.edge:end].view(self.array.shape)
        assert torch.equal(self.array[kept], before[kept]), (label, "another's page")


ORDERS = [([5, 2, 9, 1], [40, 40, 40]), ([3, 3, 3, 9], [40, 40, 40]), ([0, 1, 2, 9], [1 << 30, -7, 2000000000]), ([0, 100, -3, 9], [40, 3, 4]), ([100, 100, 100, 100], [40, 40, 40]),
          ([-5, -4, -3, -2], [40, 40, 40]), ([0, 3, 6, 9], [48, 49, 1 << 20]), ([9, 6, 3, 0], [(1 << 31) - 1, -(1 << 31), 0])]


@pytest.mark.parametrize("layout", ["tokens", "heads"])
@pytest.mark.parametrize("more", [0, 90])      # sequences of no tokens behind the others
@pytest.mark.parametrize("first,lengths", ORDERS)
def test_nothing_outside(first, lengths, more, layout):
    rng = synth.child_rng(680, more)
    page, kv, dim, heads, t = 16, 2, 64, 4, 9
    host_table, pages = _table(rng, [40, 40, 40] + [0] * more, page, spare=4)
    shape = (pages, kv, page, dim) if layout == "heads" else (pages, page, kv, dim)
    k, v, k_exp, v_exp = (Guarded(s, i) for i, s in enumerate((shape, shape, (pages, kv, page), (pages, kv, page))))
    arrays = [x.array.view(E4M3) for x in (k, v)]
    if layout == "heads":
        arrays = [x.transpose(1, 2) for x in arrays]
    cache = rb.Cache8(*arrays, k_exp.array, v_exp.array)
    used = {int(p) for p in host_table.ravel() if 0 <= p < pages}
    q, x = _rand(rng, t, heads, dim), _rand(rng, t, kv, dim)
    starts, now, table = _ints(first + first[-1:] * more), _ints(lengths + [0] * more), torch.from_numpy(host_table).cuda()
    cos, sin = (torch.full((300, dim // 2), c, device="cuda") for c in (0.6, 0.8))
    turned, o = (torch.full((t + 2, heads, dim), KEPT, dtype=F16, device="cuda") for _ in range(2))
    back = [torch.full((t + 2, kv, dim), KEPT, dtype=F16, device="cuda") for _ in range(2)]
    print(first, lengths, more, layout, flush=True)
    rb.rb_cache8_append(cache, x, x, starts, now, table, q=q, cos=cos, sin=sin, q_out=turned[1:t + 1])
    torch.cuda.synchronize()
    for name, a in (("k", k), ("v", v), ("k_exp", k_exp), ("v_exp", v_exp)):
        a.check(used, name)
        a.was.copy_(a.all)
    rb.rb_attn_cache8(cache, q, starts, now, table, o=o[1:t + 1])
    rb.rb_cache8_read(cache, starts, now, table, t, back[0][1:t + 1], back[1][1:t + 1])
    torch.cuda.synchronize()
    for name, a in (("k", k), ("v", v), ("k_exp", k_exp), ("v_exp", v_exp)):
        assert torch.equal(a.all, a.was), name      # reading changes nothing at all
    for y in (turned, o, *back):
        assert (y[0] == KEPT).all() and (y[t + 1] == KEPT).all()


@pytest.mark.parametrize("more", [0, 90])
def test_the_guards_see_what_is_stored(more):
    """Arrays in order: what the sequences' pages hold has changed, so the test above looks at the right bytes."""
    rng = synth.child_rng(681)
    page, kv, dim = 16, 2, 64
    host_table, pages = _table(rng, [40, 40, 40] + [0] * more, page, spare=4)
    k, v, k_exp, v_exp = (Guarded(s, i) for i, s in enumerate(((pages, page, kv, dim),) * 2 + ((pages, kv, page),) * 2))
    cache = rb.Cache8(k.array.view(E4M3), v.array.view(E4M3), k_exp.array, v_exp.array)
    x = _rand(rng, 9, kv, dim)
    rb.rb_cache8_append(cache, x, x, _ints([0, 3, 6, 9] + [9] * more), _ints([40, 40, 40] + [0] * more), torch.from_numpy(host_table).cuda())
    torch.cuda.synchronize()
    last = {int(host_table[i, 2]) for i in range(3)}
    for a in (k, v, k_exp, v_exp):
        a.check(last, "in order")
        with pytest.raises(AssertionError):
            a.check(set(), "in order")
