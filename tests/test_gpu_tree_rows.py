"""The attention of drafted tokens, kernel by kernel: up to 16 and up to 32 query rows of a kv head (warp-level instructions,
tiles of 16 and of 32 rows) and more (tensor cores), each with the masks, tables, values and seams where it can go wrong."""
import math

import pytest

from tests.gpu_util import require_gpu
from tests.test_gpu_operators import Tree

pytestmark = pytest.mark.gpu

# most drafts of a sequence, with four query heads of each kv head, and the kernel's bounds on the rows
KINDS = [(1, 1, 16), (4, 1, 16), (5, 17, 32), (8, 17, 32), (9, 33, 1 << 20), (40, 33, 1 << 20)]
kinds = pytest.mark.parametrize("drafts,low,high", KINDS)
formats = pytest.mark.parametrize("e4m3", [False, True])
dims = pytest.mark.parametrize("hd", [64, 128])


def _tree(low, high, hd, lens, drafts, e4m3, **kw):
    torch = require_gpu()
    assert low <= 4 * max(drafts) <= high
    return torch, Tree(torch, 8, 2, hd, lens, drafts, e4m3, **kw)


@kinds
@formats
@dims
def test_peaked(hd, e4m3, drafts, low, high):
    """Scores hundreds of units apart, so that the running maximum moves again and again, and scales of both signs."""
    torch, t = _tree(low, high, hd, [999, 2048, 30], [drafts, (drafts + 1) // 2, 1], e4m3, seed=9, q_std=40.0)
    for scale in (None, 0.003, -0.05, 0.0):
        t.check(t.run(scale=scale), scale=scale)


@kinds
@formats
@pytest.mark.parametrize("mask", ["chain", "none", "random"])
def test_masks(mask, e4m3, drafts, low, high):
    """Rows that see nothing, bits of drafts that do not exist, and no mask at all."""
    torch, t = _tree(low, high, 128, [130, 0, 1000, 0, 16], [drafts, drafts, 1, 1, drafts], e4m3, mask=mask, seed=3)
    out = t.run()
    t.check(out)
    if mask == "none":
        assert bool((out[t.start[1]:t.start[2]] == 0).all() and (out[t.start[3]:t.start[4]] == 0).all())


@kinds
@formats
@dims
def test_cut_pairs(hd, e4m3, drafts, low, high):
    """Caches long enough to be shared by several CTAs, among short ones; the same bits every time."""
    torch, t = _tree(low, high, hd, [20011, 3, 700, 0, 6001], [drafts, 1, drafts, drafts, 1], e4m3, seed=4, q_std=1.0)
    out = t.run()
    t.check(out)
    assert all(torch.equal(out, t.run()) for _ in range(3))


@kinds
@formats
def test_not_finite_drafts(e4m3, drafts, low, high):
    """A draft that is not finite reaches the rows that see it and no others."""
    torch, t = _tree(low, high, 64, [50, 0, 1200], [drafts] * 3, e4m3, seed=6)
    want, bound = t.want()
    hurt = torch.zeros(t.q.shape[0], dtype=torch.bool, device="cuda")
    for s, j, x, i in ((0, drafts // 2, t.v, math.nan), (1, drafts - 1, t.v, math.inf), (2, drafts - 1, t.k, math.nan)):
        x[t.start[s] + j, :, 7] = i
        hurt[t.start[s]:t.start[s + 1]] |= t.seen[t.start[s]:t.start[s + 1], j]
    out = t.run()
    assert bool(((out.double() - want).abs() <= bound)[~hurt].all()) and bool(out[hurt].isnan().any(-1).all())
    assert int(hurt.sum()) >= 3


@kinds
@formats
def test_not_finite_cache(e4m3, drafts, low, high):
    """A NaN in a cached key reaches its kv head's rows of the sequence, and nothing else."""
    torch, t = _tree(low, high, 128, [50, 20, 1200], [drafts] * 3, e4m3, seed=7)
    want, bound = t.want()
    for s, token in ((0, 49), (2, 100)):
        page = int(t.table[s, token // 16])
        if e4m3:
            t.exps[page, 0, 1, token % 16] = 255
        else:
            t.pages[page, 0, 1, token % 16, 1] = math.nan
    out = t.run()
    ok = (out.double() - want).abs() <= bound
    assert bool(ok[:, :4].all()) and bool(ok[t.start[1]:t.start[2]].all())
    assert bool(out[:t.start[1], 4:].isnan().all()) and bool(out[t.start[2]:, 4:].isnan().all())


@kinds
@formats
def test_bad_tables(e4m3, drafts, low, high):
    """NaN for a sequence with a bad page or length, whole or cut; bad drafts are left out; others are untouched."""
    torch, t = _tree(low, high, 64, [50, 40, 33, 1500], [drafts] * 4, e4m3, seed=8)
    want, bound = t.want()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    fine = lambda o, s: bool(((o.double() - want).abs() <= bound)[t.start[s]:t.start[s + 1]].all())  # noqa: E731
    lost = lambda o, s: bool(o[t.start[s]:t.start[s + 1]].isnan().all())  # noqa: E731
    for page in (-1, t.pages.shape[0], 2 ** 31 - 1, -2 ** 31):
        table = t.table.clone()
        table[1, 1] = table[3, 70] = page
        o = t.run(table=table)
        assert fine(o, 0) and lost(o, 1) and fine(o, 2) and lost(o, 3)
    for n in (-1, -2 ** 31, 16 * t.width + 1, 2 ** 31 - 1):
        o = t.run(lens=i32([50, n, 33, 1500]))
        assert fine(o, 0) and lost(o, 1) and fine(o, 2) and fine(o, 3)
    five = torch.full_like(want, 5.0).bfloat16()
    start = t.start[:4] + [t.start[4] + 1]   # the last sequence's drafts pass the end
    o = t.run(start=i32(start), max_drafts=drafts + 1, out=five.clone())
    assert fine(o, 0) and fine(o, 1) and fine(o, 2) and bool((o[t.start[3]:] == 5.0).all())
    o = t.run(start=i32([-1] + t.start[1:]), out=five.clone())
    assert bool((o[:t.start[1]] == 5.0).all()) and fine(o, 1) and fine(o, 2) and fine(o, 3)


@kinds
@formats
def test_far_pages(e4m3, drafts, low, high):
    """Pages beyond 2^31 elements and 2^32 bytes of the pool: the same bits as near ones."""
    torch, t = _tree(low, high, 128, [70, 17, 1100], [drafts] * 3, e4m3, seed=2)
    n_pages = 600000 if e4m3 else 300000
    shape = (n_pages,) + t.pages.shape[1:]
    assert math.prod(shape) > 1 << 31 and math.prod(shape) * t.pages.element_size() > 1 << 32
    near = t.run()
    pool = torch.empty(shape, dtype=t.pages.dtype, device="cuda")
    exps = torch.zeros(shape[:4], dtype=torch.uint8, device="cuda") if e4m3 else None
    far = torch.full_like(t.table, -7)
    for b, n in enumerate(t.lens):
        for j in range((n + 15) // 16):
            to, page = n_pages - 1 - 7 * j - b, int(t.table[b, j])
            pool[to].copy_(t.pages[page])
            if e4m3:
                exps[to] = t.exps[page]
            far[b, j] = to
    t.pages, t.exps = pool, exps
    assert torch.equal(near, t.run(table=far))


@kinds
@formats
def test_capture(e4m3, drafts, low, high):
    """A captured call, replayed as the lengths change."""
    torch, t = _tree(low, high, 128, [6000, 50, 900], [drafts, drafts, 1], e4m3, seed=13)
    lens, start = (torch.tensor(x, dtype=torch.int32).cuda() for x in (t.lens, t.start))
    a = t.run()
    out = torch.zeros_like(a)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        t.run(lens=lens, start=start, out=out)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, out)
    for n in (4100, 77, 0):
        lens[0] = t.lens[0] = n
        g.replay()
        torch.cuda.synchronize()
        t.check(out)


# ---------------------------------------------------------------- every key counts, once
SEAMS = [[8000], [8001, 17], [513, 4097, 0, 128], [511, 512, 127, 129, 1], [2048] * 12]


def _exact_codes(torch, t, values, gen):
    """Puts values (0 or +-1) into the pages: in 8 bits as codes of 1/4 .. 4 under the exponents that make up for them."""
    if t.exps is None:
        t.pages.copy_(values.bfloat16())
        return
    by = torch.randint(-2, 3, t.exps.shape, generator=gen, device="cuda")
    t.pages.copy_((values * torch.exp2(by.double())[..., None]).to(torch.float8_e4m3fn))
    t.exps.copy_((127 - by).to(torch.uint8))


@kinds
@formats
@dims
@pytest.mark.parametrize("lens", SEAMS)
def test_counts(lens, hd, e4m3, drafts, low, high):
    """Equal scores, and a value of one in a single dimension: an output is the number of the keys seen that have it, over the
    number of all.  Weights of one and their sums are exact, and so is the output but for a division in fp32 and its rounding
    to bf16, whose steps are 2^-7 of it at most: a key of at most 128 in its dimension that is lost or doubled shows."""
    torch, t = _tree(low, high, hd, lens, [drafts] * len(lens), e4m3, seed=len(lens))
    gen = torch.Generator(device="cuda").manual_seed(1)
    t.q.zero_()
    values = torch.ones(t.pages.shape, dtype=torch.float64)
    values[:, 1, ..., 1:] = 0   # places that are not used would count for dimension 0
    table = t.table.tolist()
    dim = lambda p: (p + p // hd) % hd  # noqa: E731
    for s, n in enumerate(lens):
        for p in range(n):
            row = values[table[s][p // 16], 1, :, p % 16]
            row[:, 0] = 0
            row[:, dim(p)] = 1
    _exact_codes(torch, t, values.cuda(), gen)
    t.v.zero_()
    for i in range(t.v.shape[0]):
        t.v[i, :, i % hd] = 1.0
    out, seen, mine = t.run().cpu(), t.seen.cpu(), torch.arange(t.v.shape[0]) % hd
    for s, n in enumerate(lens):
        cached = torch.bincount(dim(torch.arange(n)), minlength=hd)
        for i in range(t.start[s], t.start[s + 1]):
            count = cached + torch.bincount(mine[seen[i, :drafts].nonzero()[:, 0] + t.start[s]], minlength=hd)
            assert int(count.max()) <= 128
            want = count.double() / count.sum()
            least, most = ((want * (1 + x)).bfloat16() for x in (-2.0 ** -21, 2.0 ** -21))
            assert bool(((out[i] == least) | (out[i] == most)).all()), (s, i, (out[i].double() - want).abs().max())


@kinds
@formats
@dims
@pytest.mark.parametrize("lens", SEAMS)
def test_one_key_each(lens, hd, e4m3, drafts, low, high):
    """Each query is one key's own signs, far above any other's score: its output is that key's value.  The keys are the
    first and last ones, those at pages', chunks' and parts' ends, and drafted ones."""
    torch, t = _tree(low, high, hd, lens, [drafts] * len(lens), e4m3, mask="chain", seed=len(lens) + 1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    sign = lambda shape: (2 * torch.randint(0, 2, shape, generator=gen, device="cuda") - 1).double()  # noqa: E731
    values = sign(t.pages.shape)
    _exact_codes(torch, t, values, gen)
    t.k.copy_(sign(t.k.shape))
    t.v.copy_(sign(t.v.shape))
    values, k, v, table = values.cpu(), t.k.cpu().double(), t.v.cpu().double(), t.table.tolist()
    q, want = torch.zeros(t.q.shape, dtype=torch.float64), torch.zeros(t.q.shape, dtype=torch.float64)
    turn = 0
    for s, n in enumerate(lens):
        places = sorted({p for b in range(0, n + 1, 128 * max(1, n // 2000)) for p in (b - 1, b, b + 15, b + 16) if 0 <= p < n}
                        | {p for p in (0, n - 1, n // 2, n - n % 16, n - n % 128) if 0 <= p < n})
        for i in range(t.start[s], t.start[s + 1]):
            for h in range(t.nq):
                g = h // 4
                turn += 1
                if not places or turn % 3 == 0:   # a draft up to itself
                    j = t.start[s] + turn % (i - t.start[s] + 1)
                    q[i, h], want[i, h] = k[j, g], v[j, g]
                else:
                    p = places[turn % len(places)]
                    page = table[s][p // 16]
                    q[i, h], want[i, h] = values[page, 0, g, p % 16], values[page, 1, g, p % 16]
    t.q.copy_(q)
    # scores: hd at the key; others' signs agree by chance (a sum of hd signs, whose exponential's mean is below
    # e^(hd / 2)): n e^(hd / 2 - hd) < 2e-10 of the whole
    assert torch.equal(t.run(scale=1.0).cpu(), want.bfloat16())
