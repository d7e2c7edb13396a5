"""What cache_fork and cache_compact may write: pools that share memory are refused, and pages that somebody still holds are left as
they were, whatever the call came to."""
import pytest

from tests.cache4_util import Pool
from tests.test_gpu_pages import Search, _kp

pytestmark = pytest.mark.gpu


def test_pools_that_share_memory():
    """A pool that repeats its pages or layers (expand), the same pool twice, one within another, an output within a pool; what lies
    between a pool's pages may be another's."""
    torch, kp = _kp()
    s = Search(torch, [40, 10], seed=1, fmt="16")
    refs, table, lens = s.tensors()
    parents, (pool,) = s.i32([0, 0]), s.pools
    before, bits = pool.clone(), lambda x: x.view(torch.int16)  # noqa: E731
    for pools in ([pool[:, :1].expand(-1, s.n, -1, -1, -1, -1)], [pool[:1].expand(3, -1, -1, -1, -1, -1)], [pool, pool], [pool, pool[1:2]],
                  [pool[:, :, :1], pool[:, :, :2]]):
        for call in (lambda: kp.cache_fork(pools, refs, table, lens, parents), lambda: kp.cache_compact(pools, refs, table, lens)):
            with pytest.raises(kp.KvprmError, match="overlap"):
                call()
    flat = pool.view(torch.int32).flatten()
    out = (torch.empty_like(table), torch.empty_like(lens), flat[:s.n], torch.empty(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(kp.KvprmError, match="overlap"):
        kp.cache_fork([pool], refs, table, lens, parents, out=out)
    with pytest.raises(kp.KvprmError, match="overlap"):
        kp.cache_fork([pool], refs, table, lens, parents, workspace=flat[:1 << 14])
    assert torch.equal(bits(pool), bits(before))
    halves = kp.cache_fork([pool[:, :, :1], pool[:1, :, 1:], pool[1:, :, 1:]], refs, table, lens, parents)
    whole, again = before.clone(), kp.cache_fork([before], refs, table, lens, parents)
    assert all(torch.equal(a, b) for a, b in zip(halves, again))
    assert torch.equal(bits(pool), bits(before)) and not torch.equal(bits(pool), bits(whole))


@pytest.mark.parametrize("parents,room,width,short", [([1, 1], [0, 0], 2, False), ([1, 1, 2], [0, 40, 0], 4, False),
                                                      ([1, 1, 2], [0, 140, 0], 12, True), ([3, 3, 3, 3, 3], [30, 0, 99, 1, 2], 12, True),
                                                      ([0, 0, 1, 2, 2, 2, 3, -1], [200] * 8, 30, True)])
def test_a_step_that_runs_short(parents, room, width, short):
    """What is overwritten: of the old tables' pages those alone that no sequence with descendants lists.  A step is planned without
    pools, chosen anew where it would run short, and then keeps what its sequences hold."""
    torch, kp = _kp()
    s = Search(torch, [5, 5, 21, 40], spare=0, held=0, seed=4, width=4)
    refs, table, lens = s.tensors()
    before, copy = s.bytes(), [p.clone() for p in s.pools]
    planned = kp.cache_fork([], refs, table, lens, s.i32(parents), s.i32(room), width=width)
    assert s.same(before)
    made = kp.cache_fork(s.pools, refs, table, lens, s.i32(parents), s.i32(room), width=width)
    assert all(torch.equal(a, b) for a, b in zip(planned, made))
    assert [x.tolist() for x in made] == list(Pool(s.refs, s.table, s.lens).fork(parents, room, width)[:4])
    assert (int(made[3][1]) > 0) == short
    after = s.bytes()
    for b in range(4):
        pages = s.table[b][:-(-s.lens[b] // 16)]
        if b in parents:
            assert all(torch.equal(x[:, pages], y[:, pages]) for x, y in zip(before, after)), b
    # again, from the same tables, with parents that drop the same sequences: what they hold is what they held
    keep = sorted(set(p for p in parents if p >= 0))
    again = kp.cache_fork(s.pools, refs, table, lens, s.i32(keep))
    assert again[3][1] == 0
    for row, b in zip(again[0].tolist(), keep):
        n = -(-s.lens[b] // 16)
        assert all(torch.equal(x[:, row[:n]], y[:, s.table[b][:n]]) for x, y in zip(s.bytes(), before))
    # planned, then with others than those of the plan
    s.pools = copy
    assert s.same(before)
    kp.cache_fork([], refs, table, lens, s.i32(parents), s.i32(room), width=width)
    other = kp.cache_fork(s.pools, refs, table, lens, s.i32([0, 1, 2, 3]))
    assert other[3].tolist() == [0, 0]
    for row, b in zip(other[0].tolist(), range(4)):
        n = -(-s.lens[b] // 16)
        assert all(torch.equal(x[:, row[:n]], y[:, s.table[b][:n]]) for x, y in zip(s.bytes(), before))


def test_room_that_stays_unused():
    """Pages that were given as room and not reached keep their reference over the next step, until it is taken off."""
    torch, kp = _kp()
    s = Search(torch, [20], spare=6, held=0, seed=5, width=8)
    refs, table, lens = s.tensors()
    table, lens, refs, counts = kp.cache_fork(s.pools, refs, table, lens, s.i32([0]), s.i32([50]))
    assert counts.tolist() == [3, 0] and int((table[0] >= 0).sum()) == 5
    unused = table[0, 2:5].long()
    lost = kp.cache_fork(s.pools, refs, table, lens, s.i32([0]))
    assert lost[3].tolist() == [3, 0] and lost[2][unused].tolist() == [1, 1, 1]
    refs[unused] -= 1
    found = kp.cache_fork(s.pools, refs, table, lens, s.i32([0]), s.i32([90]))
    assert found[3].tolist() == [1, 0] and set(unused.tolist()) <= set(found[0][0].tolist())
