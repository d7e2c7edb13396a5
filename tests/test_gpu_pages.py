"""cache_fork and cache_compact against their definitions in plain Python (tests/cache4_util.py): every number, and every page of
every pool, bit by bit."""
import random

import pytest

from tests.cache4_util import Pool
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _kp():
    torch = require_gpu()
    import paper_2607_09153_gb300 as kp
    return torch, kp


class Search:
    """Sequences over a pool: some with a common beginning, some pages held by others, the rest free."""

    def __init__(self, torch, lens, shared=0, spare=20, held=3, seed=0, width=None, layers=3, nkv=2, hd=64, fmt="4"):
        self.torch, rng = torch, random.Random(seed)
        blocks = [-(-n // 16) for n in lens]
        common = [min(shared // 16, b) for b in blocks]
        pages = max([0] + common) + sum(b - c for b, c in zip(blocks, common)) + held + spare
        order = list(range(pages))
        rng.shuffle(order)
        beginning = [order.pop() for _ in range(max([0] + common))]
        width = max([1] + blocks) if width is None else width
        table = [beginning[:c] + [order.pop() for _ in range(b - c)] for b, c in zip(blocks, common)]
        refs = [0] * pages
        for row in table:
            for p in row:
                refs[p] += 1
        for _ in range(held):
            refs[order.pop()] += rng.randint(1, 3)
        self.table = [row + [rng.choice([-1, 0, 10 ** 9]) for _ in range(width - len(row))] for row in table]
        self.lens, self.refs, self.n = list(lens), refs, pages
        gen = torch.Generator(device="cuda").manual_seed(seed)
        shape = (layers, pages, 2, nkv, 16, hd)
        rnd = lambda s: torch.randint(0, 256, s, generator=gen, device="cuda", dtype=torch.uint8)  # noqa: E731
        if fmt == "4":
            self.pools = [rnd(shape[:-1] + (hd // 2,)), rnd(shape[:-1] + (hd // 32,))]
        elif fmt == "8":
            self.pools = [rnd(shape).view(torch.float8_e4m3fn), rnd(shape[:-1]).view(torch.float8_e8m0fnu)]
        else:
            self.pools = [rnd(shape[:-1] + (2 * hd,)).view(torch.bfloat16)]

    def i32(self, x, shape=None):
        t = self.torch.tensor(x, dtype=self.torch.int32)
        return (t if shape is None else t.view(shape)).cuda()

    def tensors(self):
        return self.i32(self.refs), self.i32(self.table, (len(self.lens), -1 if self.lens else 1)), self.i32(self.lens)

    def bytes(self):
        return [p.view(self.torch.uint8).clone() if p.element_size() == 1 else p.view(self.torch.int16).clone() for p in self.pools]

    def moved(self, before, copies):
        for pool in before:
            for a, b in copies:
                pool[:, b] = pool[:, a].clone()
        return before

    def same(self, want):
        return all(self.torch.equal(a, b) for a, b in zip(self.bytes(), want))


def _fork(s, parents, room=None, width=None, **kw):
    """cache_fork's answer, compared with the definition's."""
    torch, kp = s.torch, __import__("paper_2607_09153_gb300")
    width = width or len(s.table[0])
    want = Pool(s.refs, s.table, s.lens).fork(parents, room or [0] * len(parents), width)
    before = s.bytes()
    refs, table, lens = s.tensors()
    out = kp.cache_fork(s.pools, refs, table, lens, s.i32(parents), None if room is None else s.i32(room), width=width, **kw)
    torch.cuda.synchronize()
    for name, got, w in zip(("table", "lens", "refs", "counts"), out, want):
        assert got.tolist() == w, name
    assert s.same(s.moved(before, want[4]))
    assert refs.tolist() == s.refs and lens.tolist() == s.lens   # the inputs are left as they were
    return out, want


@pytest.mark.parametrize("fmt", ["4", "8", "16"])
@pytest.mark.parametrize("lens,shared,parents,room", [
    ([40], 0, [0], [0]), ([40], 0, [0, 0], [9, 8]), ([0], 0, [0, -1, 5], [1, 0, 33]), ([16, 32], 0, [1, 1, 0], [0, 16, 17]),
    ([100, 90, 64, 1], 64, [2, 0, 0, 3, 3, 3, 1], [4, 200, 0, 15, 16, 1, 2]), ([33] * 6, 32, [5] * 9, [3] * 9),
    ([77, 5], 0, [], []), ([200, 17, 0, 48], 16, [3, 2, 1, 0], None)])
def test_fork(lens, shared, parents, room, fmt):
    torch, _ = _kp()
    s = Search(torch, lens, shared, seed=len(parents), width=30, fmt=fmt, spare=60)
    _fork(s, parents, room)


def test_fork_of_nothing():
    """No sequences before; then no pages at all."""
    torch, kp = _kp()
    s = Search(torch, [], spare=7, held=0)
    e = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    table, lens, refs, counts = kp.cache_fork(s.pools, s.i32([0] * 7), e, e[:, 0].contiguous(), s.i32([-1, 3]), s.i32([20, 16]))
    assert table.tolist() == [[0, 1, -1, -1], [2, -1, -1, -1]] and lens.tolist() == [0, 0]
    assert refs.tolist() == [1, 1, 1, 0, 0, 0, 0] and counts.tolist() == [4, 0]
    none = [p[:, :0] for p in s.pools]
    out = kp.cache_fork(none, s.i32([]), e, e[:, 0].contiguous(), s.i32([-1]), s.i32([17]))
    assert out[0].tolist() == [[-1] * 4] and out[3].tolist() == [0, 2]


@pytest.mark.parametrize("seed", range(12))
def test_fork_random(seed):
    """Random searches: common beginnings, requests that begin, pages held by others, pools that run short, tables too narrow."""
    torch, _ = _kp()
    rng = random.Random(seed)
    n, m = rng.choice([1, 3, 40, 300]), rng.choice([1, 7, 64, 700])
    lens = [rng.randint(0, rng.choice([5, 60, 400])) for _ in range(n)]
    s = Search(torch, lens, rng.choice([0, 16, 200]), spare=rng.choice([0, 9, 3000]), seed=seed, layers=rng.choice([1, 2]), nkv=1,
               width=rng.choice([None, 30, 600]))
    best = [rng.randrange(n) for _ in range(max(1, n // 3))]
    parents = [rng.choice(best + [-1, n, -2 ** 31]) for _ in range(m)]
    _fork(s, parents, [rng.randint(0, 70) for _ in range(m)], width=rng.choice([None, 27, 40]))


def test_fork_shared_open_page():
    """A page that several sequences list: ended inside by some, full for another, and held by somebody else."""
    torch, _ = _kp()
    s = Search(torch, [40, 48, 20], seed=3)
    s.table[1][2] = s.table[0][2]                  # full for 1, ends inside for 0
    s.refs[s.table[0][2]] += 1
    _fork(s, [0, 1, 0])                            # 1 holds it: both of 0's are copied
    _fork(s, [0, 0])                               # 1 is dropped: the first of 0's keeps it
    s.refs[s.table[2][1]] += 1                     # somebody else holds 2's last page
    _fork(s, [2, 2], [12, 13])
    s.table[2] = list(s.table[0])                  # the same pages, of different lengths
    s.lens[2] = 35
    _fork(s, [2, 0, 2])


def test_fork_bad_inputs():
    """What the host cannot see: lengths that cannot be, pages outside the pool."""
    torch, _ = _kp()
    s = Search(torch, [40, 30, 64, 20], seed=5, width=6)
    s.lens[1], s.lens[2] = -3, 16 * 6 + 1
    _fork(s, [0, 1, 2, 1, 3], [0, 40, 5, 0, 2])
    s = Search(torch, [40, 30], seed=6, width=6)
    s.table[0][0], s.table[0][2], s.table[1][1] = -1, s.n, -2 ** 31
    _fork(s, [0, 1, 0, 1], [9, 2, 0, 60])


def test_fork_pools():
    """Layers that were allocated apart, layers and pages with strides, pages larger and smaller than a piece of a copy."""
    torch, kp = _kp()
    s = Search(torch, [40, 100], seed=7, fmt="8", nkv=8, hd=128)
    whole = s.pools
    s.pools = [p[i:i + 1] for p in whole for i in range(3)]
    _fork(s, [0, 0, 1, 1], [3, 4, 5, 6], width=9)
    big = torch.randint(0, 99, (5, s.n, 3, 1029, 4), device="cuda", dtype=torch.int32)
    s.pools = [big[1:4:2, :, :1], big[:, :, 1:2, :1028].transpose(0, 0), whole[0][:2]]
    with pytest.raises(ValueError):
        kp.cache_fork([big[..., :2]], *s.tensors(), s.i32([0]))
    rest = big[:, :, 2].clone()
    refs, table, lens = s.tensors()
    want = Pool(s.refs, s.table, s.lens).fork([1, 1], [0, 0], len(s.table[0]))
    before = [p.clone() if p.dtype == torch.int32 else p.view(torch.uint8).clone() for p in s.pools]
    kp.cache_fork(s.pools, refs, table, lens, s.i32([1, 1]))
    (a, b), = want[4]
    for p, q in zip(s.pools, before):
        q[:, b] = q[:, a].clone()
        assert torch.equal(p if p.dtype == torch.int32 else p.view(torch.uint8), q)
    assert torch.equal(big[:, :, 2], rest)
    assert kp.cache_fork([], refs, table, lens, s.i32([1, 1]))[0].tolist() == want[0]


def test_fork_of_a_large_pool():
    """More pages and table entries than the launch has threads, far beyond 2^32 bytes."""
    torch, _ = _kp()
    rng = random.Random(1)
    s = Search(torch, [rng.randint(0, 3000) for _ in range(200)], 1000, spare=60000, seed=1, layers=1, nkv=1)
    parents = [rng.randrange(100) for _ in range(260)]
    _fork(s, parents, [rng.randint(0, 900) for _ in parents], width=260)
    kp = __import__("paper_2607_09153_gb300")
    n = 150000
    pool = torch.zeros((1, n, 2, 8, 16, 64), dtype=torch.bfloat16, device="cuda")
    assert pool.numel() * 2 > 2 ** 32
    refs = torch.ones(n, dtype=torch.int32, device="cuda")
    refs[n - 1] = 0
    pool[0, n - 2] = 3.0
    table = torch.tensor([[n - 2]], dtype=torch.int32, device="cuda")
    out = kp.cache_fork([pool], refs, table, s.i32([5]), s.i32([0, 0]))
    assert out[0].tolist() == [[n - 2], [n - 1]] and bool((pool[0, n - 1] == 3.0).all())


def test_nothing_to_do_in_many_pools():
    """Every sequence dropped, and none to begin with, with layers that were allocated apart."""
    torch, kp = _kp()
    s = Search(torch, [40, 20], seed=8, layers=7)
    s.pools = [p[i:i + 1] for p in s.pools for i in range(7)]
    _fork(s, [])
    e = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    out = kp.cache_compact([p[:, :1] for p in s.pools], s.i32([2]), e, e[:, 0].contiguous())
    assert [x.tolist() for x in out] == [[], [2], [0], [1, 0]]


@pytest.mark.parametrize("m,width", [(3, 5), (1, 1), (0, 7)])
def test_results_are_tensors_like_others(m, width):
    """Results of odd sizes, written in place, and handed to the next calls."""
    torch, kp = _kp()
    s = Search(torch, [10, 0], seed=2, spare=5, width=3)
    refs, table, lens = s.tensors()
    room = s.i32([16] * m)
    table, lens, refs, counts = kp.cache_fork(s.pools, refs, table, lens, s.i32([0] * m), room, width=width)
    lens.add_(6)
    refs[s.n - 1] = 1
    counts.zero_()
    table[:, -1:] = -1
    assert table.is_contiguous() and tuple(table.shape) == (m, width) and lens.tolist() == [16] * m and counts.tolist() == [0, 0]
    now = Pool(refs.tolist(), table.tolist(), lens.tolist())
    out = kp.cache_compact(s.pools, refs, table, lens)
    assert [x.tolist() for x in out] == [list(x) for x in now.compact()[:4]]
    want = now.fork([-1] * m, [17] * m, width)
    assert [x.tolist() for x in kp.cache_fork(s.pools, refs, table, lens, s.i32([-1] * m), s.i32([17] * m))] == list(want[:4])


@pytest.mark.parametrize("seed", range(8))
@pytest.mark.parametrize("fmt", ["4", "16"])
def test_compact(seed, fmt):
    torch, kp = _kp()
    rng = random.Random(seed)
    n = rng.choice([0, 1, 5, 60])
    s = Search(torch, [rng.randint(0, rng.choice([20, 500])) for _ in range(n)], rng.choice([0, 48]), spare=rng.choice([0, 1, 500, 9000]),
               held=rng.choice([0, 4]), seed=seed, layers=2, nkv=1, fmt=fmt)
    if seed == 3:
        s.refs = [0] * s.n      # nothing in use, whatever the tables say
    if seed == 4 and n:
        s.table[0][0], s.lens[-1] = s.n + 5, -1
    want, before = Pool(s.refs, s.table, s.lens).compact(), s.bytes()
    refs, table, lens = s.tensors()
    out = kp.cache_compact(s.pools, refs, table, lens)
    torch.cuda.synchronize()
    for name, got, w in zip(("table", "refs", "moved", "counts"), out, want):
        assert got.tolist() == w, name
    assert s.same(s.moved(before, want[4])) and refs.tolist() == s.refs


def test_streams_graphs_and_outputs():
    """Caller's outputs, a side stream, a workspace, and a step of a search in a graph that is replayed on other descents."""
    torch, kp = _kp()
    s = Search(torch, [40, 100, 9], seed=9, spare=40, width=12)
    refs, table, lens = s.tensors()
    out = tuple(torch.full(x, 77, dtype=torch.int32, device="cuda") for x in ((4, 12), (4,), (s.n,), (2,)))
    parents, room = s.i32([0, 0, 1, 2]), s.i32([1, 2, 3, 40])
    want = Pool(s.refs, s.table, s.lens).fork([0, 0, 1, 2], [1, 2, 3, 40], 12)
    side = torch.cuda.Stream()
    got = kp.cache_fork(s.pools, refs, table, lens, parents, room, out=out, stream=side)
    torch.cuda.synchronize()
    assert all(a is b for a, b in zip(got, out)) and [o.tolist() for o in out] == list(want[:4])
    work = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    assert kp.cache_fork(s.pools, refs, table, lens, parents, room, width=12, workspace=work)[0].tolist() == want[0]
    with pytest.raises(kp.KvprmError, match="bytes"):
        kp.cache_fork(s.pools, refs, table, lens, parents, room, workspace=work[:256])
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    moved = kp.cache_compact(s.pools, out[2], out[0], out[1])   # (once before: eager scratch is not the graph's)
    with torch.cuda.graph(g):
        a = kp.cache_fork(s.pools, refs, table, lens, parents, room, width=12)
        b = kp.cache_compact(s.pools, a[2], a[0], a[1])
    for new, more in (([0, 0, 1, 2], [1, 2, 3, 40]), ([1, 1, 1, 1], [0, 0, 5, 60]), ([-1, 2, 2, 0], [100, 0, 0, 0])):
        parents.copy_(s.i32(new))
        room.copy_(s.i32(more))
        before = s.bytes()
        g.replay()
        torch.cuda.synchronize()
        want = Pool(s.refs, s.table, s.lens).fork(new, more, 12)
        assert [x.tolist() for x in a] == list(want[:4])
        then = Pool(want[2], want[0], want[1]).compact()
        assert [x.tolist() for x in b] == list(then[:4])
        assert s.same(s.moved(s.moved(before, want[4]), then[4]))
    assert len(moved) == 4


def test_refusals():
    torch, kp = _kp()
    s = Search(torch, [40, 10], seed=1)
    refs, table, lens = s.tensors()
    parents = s.i32([0, 1])
    for args, kw in (((s.pools, refs.long(), table, lens, parents), {}), ((s.pools, refs, table[0], lens, parents), {}),
                     ((s.pools, refs, table, lens[:1], parents), {}), ((s.pools, refs, table, lens, parents.long()), {}),
                     ((s.pools, refs, table, lens, parents, parents[:1]), {}), ((s.pools, refs[:-1], table, lens, parents), {}),
                     ((s.pools, refs, table, lens, parents), dict(out=(table, lens, refs))),
                     (([p[0] for p in s.pools], refs, table, lens, parents), {}),
                     (([p.cpu() for p in s.pools], refs, table, lens, parents), {}),
                     ((s.pools, refs.cpu(), table, lens, parents), {})):
        with pytest.raises((ValueError, TypeError)):
            kp.cache_fork(*args, **kw)
    counts = torch.empty(2, dtype=torch.int32, device="cuda")
    fresh = lambda: (torch.empty_like(table), torch.empty_like(lens), torch.empty_like(refs), counts)  # noqa: E731
    for i, x in ((0, table), (1, lens), (2, refs)):
        out = list(fresh())
        out[i] = x
        with pytest.raises(kp.KvprmError, match="overlap"):
            kp.cache_fork(s.pools, refs, table, lens, parents, out=tuple(out))
    out = list(fresh())
    out[1] = out[0].flatten()[:2]
    with pytest.raises(kp.KvprmError, match="overlap"):
        kp.cache_fork(s.pools, refs, table, lens, parents, out=tuple(out))
    with pytest.raises(kp.KvprmError, match="pools"):
        kp.cache_fork(s.pools * 60, refs, table, lens, parents)
    odd = torch.zeros((1, s.n, 24), dtype=torch.uint8, device="cuda")
    with pytest.raises(kp.KvprmError, match="16"):
        kp.cache_fork([odd], refs, table, lens, parents)
    with pytest.raises(kp.KvprmError, match="16"):
        kp.cache_compact([odd], refs, table, lens)
    with pytest.raises(kp.KvprmError, match="overlap"):
        kp.cache_compact(s.pools, refs, table, lens, out=(torch.empty_like(table), refs, torch.empty_like(refs), counts))
    kp.cache_compact(s.pools, refs, table, lens)
