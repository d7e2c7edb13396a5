"""The 4-bit cache against its definition in 64 bits (tests/cache4_util.py): codes and exponents bit by bit, expanded pages exactly,
attention within the bounds of tests/operators_util.py, at the sizes, masks and powers where it can go wrong."""
import math
import random

import pytest

from tests import cache4_util as ref4
from tests import operators_util as ref
from tests.cache4_util import Tree4
from tests.test_gpu_operators import DTYPES, HEADS, _gen, _kp, _randn

pytestmark = pytest.mark.gpu


def _pool4(torch, pages, nkv, hd, fill=0):
    return (torch.full((pages, 2, nkv, 16, hd // 2), fill, dtype=torch.uint8, device="cuda"),
            torch.full((pages, 2, nkv, 16, hd // 32), fill, dtype=torch.uint8, device="cuda"))


def _adverse_rows(torch, n, hd, gen):
    """Rows where an exponent or a rounding can go wrong: borders between codes, between exponents, the ends of the range."""
    x = torch.randn((n, hd), generator=gen, device="cuda")
    borders = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]
    near = [b * (1 + s * 2.0 ** -7) for b in borders for s in (-1, 0, 1)]
    rows = [torch.zeros(hd), torch.full((hd,), 6.0), torch.full((hd,), 6.0 * 2 ** -9), torch.full((hd,), 6.03125),
            torch.linspace(-1, 1, hd), torch.tensor([2.0 ** -i for i in range(hd)]), torch.full((hd,), 1e-38),
            torch.full((hd,), 3e38), torch.full((hd,), -2.0 ** -126), torch.arange(hd) * 1.0 + 0.5,
            torch.tensor([6.0] + [near[i % len(near)] * (-1) ** i for i in range(hd - 1)]).clamp(-6, 6),
            torch.tensor([3.0] + [near[i % len(near)] / 2 for i in range(hd - 1)]).clamp(-3, 3)]
    for i, r in enumerate(rows):
        if i < n:
            x[i] = r.cuda()
    return x


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nkv,hd", [(1, 64), (4, 128), (3, 64)])
def test_write_quantises_exactly(dtype, nkv, hd):
    """Codes and exponents bit by bit; slots outside the pool are left out, and nothing else is touched."""
    torch, kp = _kp()
    gen, n, pages = _gen(torch, hd + nkv), 41, 9
    dt = getattr(torch, dtype)
    k = _adverse_rows(torch, n * nkv, hd, gen).view(n, nkv, hd)
    if dtype == "float16":
        k = k.clamp(-65504, 65504)
    k, v = k.to(dt), (0.01 * torch.randn((n, nkv, hd), generator=gen, device="cuda")).to(dt)
    pool, exps = _pool4(torch, pages, nkv, hd, fill=0x35)
    slots = torch.randperm(pages * 16, generator=torch.Generator().manual_seed(1))[:n].cuda()
    slots[5], slots[9], slots[11] = -1, pages * 16, -(1 << 40)
    kp.cache_write(pool, slots, k, v, exponents=exps)
    want_c, want_e = _pool4(torch, pages, nkv, hd, fill=0x35)
    fine = (slots >= 0) & (slots < pages * 16)
    page, place = slots[fine] // 16, slots[fine] % 16
    for i, x in enumerate((k, v)):
        want_c[page, i, :, place], want_e[page, i, :, place] = ref4.quantise(x[fine].double())
    assert torch.equal(exps, want_e)
    # (a zero's sign is kept)
    assert torch.equal(pool, want_c)
    out = torch.full((pages + 2, 2, nkv, 16, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    src = torch.tensor([0, 3, pages - 1, pages, -1, 2], dtype=torch.int32, device="cuda")
    dst = torch.tensor([1, 0, pages + 1, 4, 5, pages + 2], dtype=torch.int32, device="cuda")
    packed = pool.view(torch.float4_e2m1fn_x2)
    assert kp.cache_expand(packed, exps.view(torch.float8_e8m0fnu), src, out, dst) is out
    values = ref4.values(want_c, want_e)
    for s, d in ((0, 1), (3, 0), (pages - 1, pages + 1)):
        assert torch.equal(out[d], values[s].bfloat16())
    rest = [i for i in range(pages + 2) if i not in (0, 1, pages + 1)]
    assert bool((out[rest] == 7.0).all())


@pytest.mark.parametrize("n,nkv", [(1, 2), (3, 40), (2500, 5)])
def test_write_many_heads(n, nkv):
    """One token, more rows than a CTA has threads for, more tokens than CTAs."""
    torch, kp = _kp()
    gen, hd, pages = _gen(torch, n), 128, (n + 15) // 16 + 1
    rows = torch.randn((n, 2 * nkv, hd), generator=gen, device="cuda").bfloat16()
    pool, exps = _pool4(torch, pages, nkv, hd)
    slots = torch.randperm(pages * 16, generator=torch.Generator().manual_seed(n))[:n].cuda()
    kp.cache_write(pool, slots, rows[:, :nkv], rows[:, nkv:], exponents=exps)
    at = [0, n // 3, n - 1]
    c, e = ref4.quantise(rows[at].double().unflatten(1, (2, nkv)))
    page, place = slots[at] // 16, slots[at] % 16
    assert torch.equal(pool[page, :, :, place], c) and torch.equal(exps[page, :, :, place], e)
    # all of them: within half a step of what was written, 1/6 of a block's largest value
    got = ref4.values(pool, exps)[slots // 16, :, :, slots % 16].unflatten(-1, (-1, 32))
    want = rows.double().unflatten(1, (2, nkv)).unflatten(-1, (-1, 32))
    assert bool(((got - want).abs() <= want.abs().amax(-1, keepdim=True) / 3 * 1.0001).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset", [0, 1])
def test_write_not_finite(dtype, offset):
    """Infinities become the largest code of the rest's scale; a block with a NaN reads as NaN, the others do not."""
    torch, kp = _kp()
    pool, exps = _pool4(torch, 2, 2, 64)
    k = torch.ones(3 * 2 * 64 + 1, device="cuda", dtype=getattr(torch, dtype))[offset:][:3 * 2 * 64].view(3, 2, 64)
    k[0, 0, 3], k[0, 1, 45], k[1, 0, 0], k[1, 1, 32:] = math.inf, -math.inf, math.nan, math.inf
    kp.cache_write(pool, torch.tensor([0, 1, 17], device="cuda"), k, torch.zeros_like(k), exponents=exps)
    out = torch.zeros((2, 2, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    kp.cache_expand(pool, exps, torch.arange(2, dtype=torch.int32, device="cuda"), out)
    big = 6 * 2.0 ** -2   # 1 <= 6 2^-2
    assert out[0, 0, 0, 0, 3] == big and out[0, 0, 1, 0, 45] == -big and out[0, 0, 0, 0, 4] == 1
    assert bool(out[0, 0, 0, 1, :32].isnan().all()) and bool((out[0, 0, 0, 1, 32:] == 1).all())
    assert bool((out[0, 0, 1, 1, :32] == 1).all()) and bool((out[0, 0, 1, 1, 32:] == 6 * 2.0 ** -127).all())
    assert bool((out[1, 0, :, 1] == 1).all()) and bool((out[:, 1] == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved,rd,hd", [(False, 128, 128), (True, 128, 128), (False, 64, 64), (False, 32, 128),
                                               (True, 32, 64), (False, 34, 64)])
@pytest.mark.parametrize("n,offset", [(5, 0), (700, 1)])
def test_write_rotates(dtype, interleaved, rd, hd, n, offset):
    """Keys rotated on the way, values not, from columns of wider rows at any alignment."""
    torch, kp = _kp()
    gen, nkv = _gen(torch, n + rd), 3
    dt = getattr(torch, dtype)
    rows = _randn(torch, (n, 2 * nkv * hd + 8), gen, dt)
    k = rows[:, offset:offset + nkv * hd].view(n, nkv, hd)
    v = rows[:, offset + nkv * hd:offset + 2 * nkv * hd].view(n, nkv, hd)
    rope = kp.Rope(rd, interleaved=interleaved)
    pos = torch.randint(0, 131072, (n,), generator=gen, device="cuda", dtype=torch.int32)
    pages = (n + 15) // 16
    slots = torch.randperm(pages * 16, generator=torch.Generator().manual_seed(2))[:n].cuda()
    pool, exps = _pool4(torch, pages, nkv, hd)
    kp.cache_write(pool, slots, k, v, exponents=exps, rope=rope, positions=pos)
    want = torch.stack([ref.rotate(k, pos, ref.frequencies(rd), interleaved), v.double()], 1).unflatten(-1, (-1, 32))
    # the rotation is off by 6e-7 of two magnitudes of its pair at most, whose other element may be in another block
    near = 1.2e-6 * want.abs().amax((-1, -2), keepdim=True) * math.sqrt(2)
    page, place = slots // 16, slots % 16
    e = exps[page, :, :, place].double() - 127
    got = ref4.values(pool[page, :, :, place], exps[page, :, :, place]).unflatten(-1, (-1, 32))
    most = want.abs().amax(-1)
    least, top = (torch.ceil(torch.log2((most + f * near[..., 0]).clamp(min=1e-300) / 6) + f * 1e-9) for f in (-1, 1))
    assert bool(((e >= least) & (e <= top)).all())
    scale = torch.exp2(e)[..., None]
    y = want.abs() / scale   # half a step: 1/4 below 2, 1/2 below 4, 1 above
    step = torch.where(y < 2, 0.25, torch.where(y < 4, 0.5, 1.0)) * scale
    assert bool(((got - want).abs() <= step + near).all())


def test_refusals():
    torch, kp = _kp()
    pool, exps = _pool4(torch, 2, 2, 64)
    x = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    kp.cache_write(pool, slots[:0], x[:0], x[:0], exponents=exps)
    for args, kw in (((pool, slots, x, x), {}), ((pool, slots, x, x), dict(exponents=exps[..., :1])),
                     ((pool, slots, x, x), dict(exponents=exps[..., 0].contiguous())),
                     ((pool, slots, x[..., :32], x[..., :32]), dict(exponents=exps)),
                     ((pool.view(torch.int8), slots, x, x), dict(exponents=exps)),
                     ((pool.transpose(0, 2), slots, x, x), dict(exponents=exps)),
                     ((pool.cpu(), slots, x, x), dict(exponents=exps.cpu()))):
        with pytest.raises((ValueError, TypeError)):
            kp.cache_write(*args, **kw)
    src = torch.zeros(1, dtype=torch.int32, device="cuda")
    for shape in ((2, 2, 2, 16, 32), (2, 2, 1, 16, 64)):
        with pytest.raises(ValueError):
            kp.cache_expand(pool, exps, src, torch.zeros(shape, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(kp.KvprmError):   # head_dim 32
        small, e = _pool4(torch, 2, 2, 32)
        kp.cache_write(small, slots, x[..., :32], x[..., :32], exponents=e)


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("nq,nkv,hd", HEADS)
@pytest.mark.parametrize("width", [None, 100])
def test_tree_small(nq, nkv, hd, width):
    """Lengths about a page's and a block's ends, one token to a few, on the kernels for short calls and on those for long ones."""
    torch, _ = _kp()
    t = Tree4(torch, nq, nkv, hd, [0, 1, 15, 16, 17, 64, 65, 200], [1, 3, 2, 1, 17, 1, 5, 4], seed=nq + hd, max_blocks=width)
    t.check(t.run())
    if width:
        return
    t = Tree4(torch, nq, nkv, hd, [0, 1, 15, 16, 17, 64, 65, 200], [1] * 8, seed=nq + hd + 1)
    t.check(t.run())


@pytest.mark.parametrize("nq,nkv,hd", [(4, 1, 64), (14, 2, 128), (3, 3, 128)])
@pytest.mark.parametrize("mask", ["tree", "chain", "none", "random"])
@pytest.mark.parametrize("drafts", [[64, 33, 70, 1, 32, 31], [2, 2, 1, 2, 1, 2], [5, 4, 5, 3, 0, 1]])
def test_tree_wide(nq, nkv, hd, mask, drafts):
    """Drafts across mask words and row tiles, with rows that see nothing at all (empty caches, empty masks)."""
    torch, _ = _kp()
    t = Tree4(torch, nq, nkv, hd, [130, 0, 1000, 127, 128, 129], drafts, mask, seed=nkv)
    out = t.run()
    t.check(out)
    if mask == "none":
        assert bool((out[t.start[1]:t.start[2]] == 0).all())


@pytest.mark.parametrize("lens,drafts", [([20011], [1]), ([20011], [2]), ([20011], [4]), ([20011], [9]),
                                         ([5000, 3, 7777], [40, 2, 33]), ([12345], [64]), ([0] * 3 + [9000] + [0] * 3, [1] * 7),
                                         ([14000, 9999] * 3, [9, 200, 6, 12, 40, 5])])
def test_tree_long(lens, drafts):
    """Long caches, whose parts many CTAs score and one joins."""
    torch, _ = _kp()
    t = Tree4(torch, 8, 2, 128, lens, drafts, seed=len(lens), q_std=1.0)
    out = t.run()
    t.check(out)
    assert torch.equal(out, t.run())


def test_tree_many_sequences():
    torch, _ = _kp()
    rng = random.Random(4)
    t = Tree4(torch, 2, 1, 64, [rng.randint(0, 40) for _ in range(1500)], [rng.randint(0, 2) for _ in range(1500)])
    t.check(t.run())


@pytest.mark.parametrize("drafts", [[1, 1], [5, 40], [2, 4], [8, 8]])
def test_tree_peaked(drafts):
    """Scores hundreds of units apart, rising and falling along the cache: the running maximum moves again and again."""
    torch, _ = _kp()
    t = Tree4(torch, 8, 2, 128, [999, 2048], drafts, seed=9, q_std=40.0)
    t.check(t.run())
    t.check(t.run(scale=0.003), scale=0.003)
    t.check(t.run(scale=-0.05), scale=-0.05)
    t.check(t.run(scale=0.0), scale=0.0)


@pytest.mark.parametrize("drafts", [1, 3, 12, 20])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("apart", ["keys", "values", "both"])
def test_tree_powers_apart(apart, hd, drafts):
    """Blocks up to 2^60 apart within a page and from page to page, zero blocks among them; queries that make up for it."""
    torch, _ = _kp()
    t = Tree4(torch, 2, 1, hd, [333, 40, 700], [drafts, 1, 2], seed=13, q_std=0.25)
    gen = _gen(torch, 14)
    shape = t.exps[:, 0].shape
    # by page: a window, a window far off, blocks all over
    kind = torch.arange(shape[0], device="cuda").view(-1, 1, 1, 1) % 3
    for i, name in ((0, "keys"), (1, "values")):
        if apart not in (name, "both"):
            continue
        near, far, over = (torch.randint(*r, shape, generator=gen, device="cuda") for r in ((118, 122), (85, 92), (60, 125)))
        e = torch.where(kind == 0, near, torch.where(kind == 1, far, over))
        e[torch.rand(shape, generator=gen, device="cuda") < 0.1] = 0
        t.exps[:, i] = e.to(torch.uint8)
    t.remake()
    t.check(t.run())


@pytest.mark.parametrize("exponent", [100, 60, 8, -8, -40, -100, -126])
@pytest.mark.parametrize("drafts,width", [(1, None), (20, None), (20, 100)])
def test_tree_scales(exponent, drafts, width):
    """A whole cache at one far power: values anywhere in the range, keys where queries make up for it.  (With a wide table many rows
    go to the tensor cores.)"""
    torch, _ = _kp()
    t = Tree4(torch, 2, 1, 128, [64, 17], [drafts, 1], seed=3, q_std=2.0 ** -max(-30, min(exponent, 100)), max_blocks=width)
    t.exps[:, 0] = 127 + max(-30, exponent)
    t.exps[:, 1] = 127 + exponent
    t.remake()
    if exponent > 0:   # (drafts of such queries and keys weigh as much as the cache)
        t.k.mul_(2.0 ** min(exponent, 100))
    t.v.mul_(2.0 ** exponent if exponent > -126 else 2.0 ** -120)
    t.check(t.run())


@pytest.mark.parametrize("drafts,width", [(1, None), (4, None), (20, None), (20, 100)])
@pytest.mark.parametrize("up", [True, False])
def test_tree_far_queries(up, drafts, width):
    """Queries at the ends of bf16's range, whole ones beyond 2^127 or below 2^-126, with keys that make up for it."""
    torch, _ = _kp()
    t = Tree4(torch, 4, 2, 128, [300, 17, 0], [drafts, 1, 2], seed=31, max_blocks=width)
    power = 125 if up else -130
    t.q = (t.q.double() * 2.0 ** power).clamp(-3e38, 3e38).bfloat16()
    t.exps[:, 0] = t.exps[:, 0].int().add(-120 if up else 120).to(torch.uint8)
    t.k.mul_(2.0 ** (-120 if up else 120))
    t.remake()
    scale = 2.0 ** (-5 if up else 10) * 128 ** -0.5
    t.check(t.run(scale=scale), scale)


@pytest.mark.parametrize("drafts,width", [(1, None), (4, None), (20, None), (20, 100)])
@pytest.mark.parametrize("mask", ["tree", "none"])
def test_tree_drafts_beyond_the_cache(mask, drafts, width):
    """Drafted values 2^160 of the cached ones, seen and not seen."""
    torch, _ = _kp()
    t = Tree4(torch, 4, 2, 128, [300, 17, 40], [drafts, 1, 2], mask=mask, seed=32, max_blocks=width)
    t.exps[:, 1] -= 60
    t.remake()
    t.v.mul_(2.0 ** 100)
    t.check(t.run())


@pytest.mark.parametrize("drafts,width", [(1, None), (2, None), (4, None), (20, None), (20, 100)])
def test_tree_zero_blocks(drafts, width):
    """Rows of zeros (exponent 0), whole pages of them, and the first page."""
    torch, _ = _kp()
    t = Tree4(torch, 4, 2, 128, [200, 30, 16], [drafts] * 3, seed=21, max_blocks=width)
    for b, j in ((0, 0), (0, 4), (1, 1), (2, 0)):
        p = int(t.table[b, j])
        t.pages[p], t.exps[p] = 0, 0
    p = int(t.table[0, 2])
    t.pages[p, :, :, ::3], t.exps[p, :, :, ::3] = 0, 0
    t.remake()
    t.check(t.run())


@pytest.mark.parametrize("drafts,width", [(1, None), (3, None), (6, None), (20, None), (20, 100)])
def test_tree_not_finite(drafts, width):
    """Drafts that are not finite reach the rows that see them and no others; a NaN in the cache reaches its sequence: a key's all
    of it, a value's the 32 dimensions of its block."""
    torch, _ = _kp()
    t = Tree4(torch, 4, 2, 64, [50, 0, 33], [drafts, 40, 2], seed=6, max_blocks=width)
    want, bound = t.want()
    hurt = torch.zeros(t.q.shape[0], dtype=torch.bool, device="cuda")
    for s, j, x, i in ((0, drafts // 2, t.v, math.nan), (0, drafts - 1, t.v, math.inf), (1, 35, t.k, math.nan), (1, 20, t.v, -math.inf)):
        x[t.start[s] + j, :, 7] = i
        hurt[t.start[s]:t.start[s + 1]] |= t.seen[t.start[s]:t.start[s + 1], j]
    out = t.run()
    ok = (out.double() - want).abs() <= bound
    assert bool(ok[~hurt].all()) and bool(out[hurt].isnan().any(-1).all())
    page, s2 = int(t.table[2, 1]), t.start[2]
    t.exps[page, 1, 0, 0, 1] = 255
    out = t.run()
    fine = (out.double() - want).abs() <= bound
    assert bool(out[s2:, :2, 32:].isnan().all()) and bool(fine[s2:, :2, :32].all()) and bool(fine[s2:, 2:].all())
    t.exps[page, 0, 1, 0, 0] = 255
    out = t.run()
    assert bool(out[s2:, 2:].isnan().all()) and bool(((out.double() - want).abs() <= bound)[s2:, :2, :32].all())


@pytest.mark.parametrize("width", [None, 100])
def test_tree_bad_tables(width):
    """What the host cannot see: NaN for a sequence with a bad page or length, others untouched; bad drafts left out."""
    torch, _ = _kp()
    for drafts in ([3, 4, 5, 40], [1, 1, 2, 1]):
        t = Tree4(torch, 4, 2, 64, [50, 40, 33, 300], drafts, seed=8, max_blocks=width)
        want, bound = t.want()
        i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()  # noqa: E731
        fine = lambda o, s: bool(((o.double() - want).abs() <= bound)[t.start[s]:t.start[s + 1]].all())  # noqa: E731
        lost = lambda o, s: bool(o[t.start[s]:t.start[s + 1]].isnan().all())  # noqa: E731
        for page in (-1, t.pages.shape[0], 2 ** 31 - 1, -2 ** 31):
            table = t.table.clone()
            table[1, 1] = table[3, 7] = page
            o = t.run(table=table)
            assert fine(o, 0) and lost(o, 1) and fine(o, 2) and lost(o, 3)
        for n in (-1, -2 ** 31, 16 * t.width + 1, 2 ** 31 - 1):
            o = t.run(lens=i32([50, 40, n, 300]))
            assert fine(o, 0) and fine(o, 1) and lost(o, 2) and fine(o, 3)
        out = torch.full_like(want, 5.0).bfloat16()
        start = list(t.start)
        start[4] += 1   # the last sequence's drafts pass the end
        o = t.run(start=i32(start), out=out)
        assert fine(o, 0) and fine(o, 1) and fine(o, 2) and bool((o[start[3]:] == 5.0).all())
        assert bool(t.run(start=i32(start))[start[3]:].isnan().all())


@pytest.mark.parametrize("drafts", [1, 20, 40])
def test_tree_empty_pool(drafts):
    """A pool without pages: sequences that have not started are answered, others NaN."""
    torch, _ = _kp()
    t = Tree4(torch, 4, 2, 64, [0, 0], [drafts, 2], seed=2, extra_pages=0, max_blocks=3)
    assert t.pages.shape[0] == 0
    t.check(t.run())
    out = t.run(lens=torch.tensor([0, 5], dtype=torch.int32).cuda())
    assert bool(out[drafts:].isnan().all()) and not bool(out[:drafts].isnan().any())


def test_tree_far_pages():
    """Pages beyond 2^32 bytes of the pool, attended to, written and read back."""
    torch, kp = _kp()
    n_pages, nkv, hd = 280000, 8, 128
    t = Tree4(torch, 16, nkv, hd, [70, 17], [3, 20], seed=2)
    pool, exps = _pool4(torch, n_pages, nkv, hd)
    assert pool.numel() > 2 ** 32
    for drafts in ([3, 20], [1, 1]):
        t = Tree4(torch, 16, nkv, hd, [70, 17], drafts, seed=2)
        far = torch.full_like(t.table, -7)
        for b, n in enumerate(t.lens):
            for j in range((n + 15) // 16):
                to = n_pages - 1 - 7 * j - b
                pool[to], exps[to] = t.pages[int(t.table[b, j])], t.exps[int(t.table[b, j])]
                far[b, j] = to
        near, own = t.run(), t.pages
        t.pages, e = pool, t.exps
        assert torch.equal(near, t.run(table=far, exponents=exps))
    kp.cache_write(pool, torch.tensor([(n_pages - 1) * 16 + 3], device="cuda"), t.k[:1], t.v[:1], exponents=exps)
    out = torch.zeros((1, 2, nkv, 16, hd), dtype=torch.bfloat16, device="cuda")
    kp.cache_expand(pool, exps, torch.tensor([n_pages - 1], dtype=torch.int32, device="cuda"), out)
    assert torch.equal(out[0, 1, :, 3], ref4.values(*ref4.quantise(t.v[0].double())).bfloat16())


@pytest.mark.parametrize("drafts", [[5, 30], [1, 2], [3, 4]])
def test_tree_strides(drafts):
    """Other orders of the heads' and tokens' strides, and an output of its own strides: the same bits."""
    torch, _ = _kp()
    t = Tree4(torch, 6, 2, 64, [40, 100], drafts, seed=12)
    a, n = t.run(), sum(drafts)
    out = torch.full((6, n, 72), 3.0, dtype=torch.bfloat16, device="cuda")
    t.k, t.v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (t.k, t.v))
    b = t.run(q=t.q.contiguous(), out=out[..., :64].transpose(0, 1))
    assert torch.equal(a, b) and bool((out[..., 64:] == 3.0).all())
    t.check(t.run(max_len=1))
    t.pages, t.exps = t.pages.view(torch.float4_e2m1fn_x2), t.exps.view(torch.float8_e8m0fnu)
    assert torch.equal(a, t.run())


@pytest.mark.parametrize("drafts", [[12, 3], [1, 1], [40, 1]])
def test_tree_streams(drafts):
    """Calls on several streams at once, each with scratch of its own, and one captured into a graph."""
    torch, _ = _kp()
    t = Tree4(torch, 8, 2, 128, [6000, 5000], drafts, seed=13)
    a = t.run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [[t.run(stream=s, out=torch.empty_like(a)) for _ in range(4)] for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(a, o) for many in outs for o in many)
    lens, start = torch.tensor(t.lens, dtype=torch.int32).cuda(), torch.tensor(t.start, dtype=torch.int32).cuda()
    out = torch.zeros_like(a)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        t.run(lens=lens, start=start, out=out)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, out)
    lens[0] = 77
    t.lens[0] = 77
    g.replay()
    torch.cuda.synchronize()
    t.check(out)


def test_tree_refusals():
    torch, kp = _kp()
    t = Tree4(torch, 4, 2, 64, [40, 10], [3, 2], seed=1)
    for kw in (dict(exponents=None), dict(exponents=t.exps[..., :1]), dict(q=t.q[..., :32])):
        with pytest.raises((ValueError, TypeError)):
            t.run(**kw)
    with pytest.raises(kp.KvprmError):
        t.run(workspace=torch.zeros(8, dtype=torch.uint8, device="cuda"))
    x = t.q.detach().clone().requires_grad_()
    with pytest.raises(RuntimeError, match="tree_attention"):
        t.run(q=x).float().sum().backward()
