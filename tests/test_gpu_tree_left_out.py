"""Tokens that no sequence has, and sequences that are left out, in a result that the call makes itself: nothing of what the
memory held before is returned."""
import pytest

from tests.gpu_util import require_gpu
from tests.test_gpu_operators import Tree

pytestmark = pytest.mark.gpu


def _run(t, tokens, start, **kw):
    """t's sequences with q, k and v of `tokens` tokens, into memory that held sevens."""
    torch = t.torch
    wide = lambda x: torch.cat([x, x.new_ones((tokens - x.shape[0],) + x.shape[1:])])  # noqa: E731
    t.q, t.k, t.v = wide(t.q), wide(t.k), wide(t.v)
    if t.mask is not None:
        t.mask = wide(t.mask)
    start = torch.tensor(start, dtype=torch.int32).cuda()
    torch.cuda.synchronize()
    sevens = [torch.full(t.q.shape, 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    del sevens
    return t.run(start=start, **kw)


# rows of a kv head: 16, 32 and more, pairs whole and cut
@pytest.mark.parametrize("drafts", [1, 4, 8, 9, 40])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("longest", [100, 3000])
def test_left_out(longest, e4m3, drafts):
    torch = require_gpu()
    t = Tree(torch, 8, 2, 64, [longest, 0, 33], [drafts, 1, drafts], e4m3, seed=drafts)
    o, bound = t.want()
    n = t.start[-1]
    # padding behind the sequences
    out = _run(t, n + 37, t.start)
    assert bool(((out[:n].double() - o).abs() <= bound).all()) and bool((out[n:] == 0).all())
    # and before them (of the first sequence, whose tokens then belong to none)
    first = t.start[1]
    start = torch.tensor([first] + t.start[1:], dtype=torch.int32).cuda()
    out = t.run(start=start)
    assert bool((out[:first] == 0).all()) and bool((out[n:] == 0).all())
    assert bool(((out[first:n].double() - o[first:]).abs() <= bound[first:]).all())
    # a sequence with more drafts than the call allows, one whose tokens pass the end, one that runs backwards
    if drafts > 1:
        out = t.run(max_drafts=drafts - 1)
        kept = slice(t.start[1], t.start[2])
        assert bool(out[:t.start[1]].isnan().all()) and bool(out[t.start[2]:n].isnan().all()) and bool((out[n:] == 0).all())
        assert bool(((out[kept].double() - o[kept]).abs() <= bound[kept]).all())
    start = torch.tensor(t.start[:-1] + [1 << 30], dtype=torch.int32).cuda()
    out = t.run(start=start)
    assert bool(out[t.start[2]:].isnan().all()) and bool(((out[:t.start[2]].double() - o[:t.start[2]]).abs() <= bound[:t.start[2]]).all())
    start = torch.tensor([t.start[1], 0, t.start[2], n], dtype=torch.int32).cuda()
    out = t.run(start=start, max_drafts=drafts + 1)
    assert not bool((out == 7).all(-1).any())


def test_nothing_to_attend_for():
    """No sequences at all, and more than one launch takes of them, with tokens to spare."""
    torch = require_gpu()
    t = Tree(torch, 4, 2, 64, [], [])
    assert bool((_run(t, 300, [0]) == 0).all())
    t = Tree(torch, 2, 1, 64, [i % 40 for i in range(1500)], [i % 3 for i in range(1500)])
    o, bound = t.want()
    n = t.start[-1]
    out = _run(t, n + 11, t.start)
    assert bool(((out[:n].double() - o).abs() <= bound).all()) and bool((out[n:] == 0).all())


def test_given_output_is_left_as_it_is():
    torch = require_gpu()
    t = Tree(torch, 8, 2, 64, [30, 10], [2, 3])
    out = torch.full((t.start[-1] + 4, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    _run(t, t.start[-1] + 4, t.start, out=out)
    assert bool((out[t.start[-1]:] == 7).all()) and not bool((out[:t.start[-1]] == 7).all(-1).any())
