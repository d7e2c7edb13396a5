"""The operators around the cache against their definitions in 64 bits (tests/operators_util.py): bounds derived from the
roundings that the header names, at the sizes, strides and masks where an index or a rounding can go wrong."""
import math
import random

import pytest

from tests import operators_util as ref
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu
DTYPES = ("bfloat16", "float16", "float32")
UNIT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -24}   # half a unit in the last place
SMALLEST = {"bfloat16": 2.0 ** -134, "float16": 2.0 ** -25, "float32": 2.0 ** -150}


def _kp():
    torch = require_gpu()
    import paper_2607_09153_gb300 as kp
    return torch, kp


def _gen(torch, seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(torch, shape, gen, dtype, std=1.0):
    return (std * torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)).to(dtype)


# ---------------------------------------------------------------- rotary
def _rope_bound(x, y, dtype, magnitude=1.0):
    """The angle is exact to 2^-32 turns, its 32-bit fraction to 2^-25 half turns, sine and cosine to 2 units each; two
    products and a sum: 6e-7 of the pair's magnitudes covers them; then the output's rounding."""
    size = x.double().abs().amax(-1, keepdim=True).clamp(min=1e-30) * magnitude
    return 6e-7 * 2 * size + UNIT[dtype] * y.abs() + SMALLEST[dtype]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,hd,rd", [(1, (1,), 64, 64), (16, (28, 4), 128, 128), (7, (3, 1, 2), 128, 64),
                                                (1300, (5,), 80, 48), (33, (2, 2), 66, 34), (3, (1,), 256, 256),
                                                (5, (4,), 64, 2), (9001, (2,), 64, 16)])
def test_rope(dtype, interleaved, tokens, heads, hd, rd):
    torch, kp = _kp()
    dt, gen = getattr(torch, dtype), _gen(torch, tokens + hd)
    rope = kp.Rope(rd, base=5e5, interleaved=interleaved, scaling="smooth", factor=8.0, original_len=8192,
                   magnitude=1.25)
    freq = ref.frequencies(rd, 5e5, "smooth", 8.0, 8192)
    pos = torch.randint(0, 1 << 20, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    xs = [_randn(torch, (tokens, h, hd), gen, dt) for h in heads]
    for inverse, call in ((False, rope.rotate), (True, rope.rotate_backward)):
        for x, y in zip(xs, call(pos, *xs)):
            want = ref.rotate(x, pos, freq, interleaved, 1.25, inverse)
            assert y.dtype == dt and y.is_contiguous()
            assert ((y.double() - want).abs() <= _rope_bound(x, want, dtype, 1.25)).all()
            assert torch.equal(y[..., rd:], x[..., rd:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_extreme_positions(interleaved):
    """Angles stay exact at every int32 position: against whole-number arithmetic on the handle's own table."""
    torch, kp = _kp()
    rope = kp.Rope(128, interleaved=interleaved)
    pos = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 131071, 1 << 24, (1 << 24) + 1]
    x = _randn(torch, (len(pos), 3, 128), _gen(torch, 5), torch.float32)
    (y,) = rope.rotate(torch.tensor(pos, dtype=torch.int32, device="cuda"), x)
    turns = rope.turns()
    ang = torch.tensor([[2 * math.pi * ((p * t) % 2 ** 64) / 2 ** 64 for t in turns] for p in pos],
                       dtype=torch.float64, device="cuda")
    ones = torch.ones(len(pos), device="cuda")
    for i in range(len(pos)):
        want = ref.rotate(x[i:i + 1], ones[:1], ang[i], interleaved)
        assert ((y[i:i + 1].double() - want).abs() <= _rope_bound(x[i:i + 1], want, "float32")).all(), pos[i]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("offset", [0, 1, 8])
def test_rope_strides(dtype, interleaved, offset):
    """Columns of a projection's rows, at any alignment, into other columns and in place; nothing else is touched."""
    torch, kp = _kp()
    dt, gen, n = getattr(torch, dtype), _gen(torch, 3), 37
    rope, freq = kp.Rope(48, interleaved=interleaved), ref.frequencies(48)
    rows = _randn(torch, (n, 8 * 64 + 16), gen, dt)
    before = rows.clone()
    x = rows[:, offset:offset + 5 * 64].view(n, 5, 64)
    k = rows[:, offset + 320:offset + 448].view(n, 2, 64).transpose(0, 1).contiguous().transpose(0, 1)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 1000
    to = torch.full((n, 7, 64 + 16), 9.0, dtype=dt, device="cuda")
    out, ko = to[:, 1:6, 8:72], torch.empty_like(k)
    rope.rotate(pos, x, k, out=(out, ko))
    want = ref.rotate(x, pos, freq, interleaved)
    assert ((out.double() - want).abs() <= _rope_bound(x, want, dtype)).all()
    want_k = ref.rotate(k, pos, freq, interleaved)
    assert ((ko.double() - want_k).abs() <= _rope_bound(k, want_k, dtype)).all()
    out.fill_(9.0)
    assert bool((to == 9.0).all())
    rope.rotate(pos, x, out=(x,))
    assert ((x.double() - want).abs() <= _rope_bound(before[:, offset:offset + 320].view(n, 5, 64), want, dtype)).all()
    x.copy_(before[:, offset:offset + 320].view(n, 5, 64))
    assert torch.equal(rows, before)


def test_rope_gradient():
    """rotate_backward is rotate's transpose: by the formula's inner product, and by differences of rotate itself (a
    linear map: they are exact up to rounding)."""
    torch, kp = _kp()
    gen, n = _gen(torch, 11), 23
    for interleaved in (False, True):
        rope = kp.Rope(32, interleaved=interleaved, magnitude=0.7)
        pos = torch.randint(0, 99999, (n,), generator=gen, device="cuda", dtype=torch.int32)
        x, dy = (_randn(torch, (n, 3, 64), gen, torch.float32) for _ in range(2))
        (y,), (dx,) = rope.rotate(pos, x), rope.rotate_backward(pos, dy)
        lhs, rhs = (dy.double() * y.double()).sum(), (dx.double() * x.double()).sum()
        assert abs(lhs - rhs) <= 1e-6 * (dy.double().abs() * y.double().abs()).sum()
        loss = lambda z: (rope.rotate(pos, z)[0].double() * dy.double()).sum()  # noqa: E731
        for _ in range(4):
            h = _randn(torch, x.shape, gen, torch.float32)
            diff = (loss(x + h) - loss(x - h)) / 2
            exact = ((x + h).double() - (x - h).double()) / 2   # the step that 32 bits took
            assert abs(diff - (dx.double() * exact).sum()) <= 4e-6 * (dx.double().abs() * (x.abs() + h.abs()).double()).sum()


def test_rope_empty_and_refusals():
    torch, kp = _kp()
    rope = kp.Rope(64)
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    x = torch.zeros(4, 2, 64, device="cuda")
    assert rope.rotate(pos[:0], x[:0])[0].shape == (0, 2, 64)
    assert rope.rotate(pos, x[:, :0])[0].shape == (4, 0, 64)
    for args in ((pos.long(), x), (pos[:3], x), (pos, x.cpu()), (pos.cpu(), x), (pos, x[0]), (pos, x.transpose(1, 2)),
                 (pos, x, x[:3]), (pos,), (pos, x, x, x, x, x)):
        with pytest.raises((ValueError, TypeError)):
            rope.rotate(*args)
    with pytest.raises(TypeError):
        rope.rotate(pos, x.double())
    with pytest.raises(TypeError):
        rope.rotate(pos, x, x.half())
    with pytest.raises(ValueError):
        rope.rotate(pos, x, out=(x[:, :1],))
    with pytest.raises(kp.KvprmError):
        rope.rotate(pos, x[..., :32])


# ---------------------------------------------------------------- cache write, expand
def _pool(torch, pages, nkv, hd, e4m3, fill=0):
    if not e4m3:
        return torch.full((pages, 2, nkv, 16, hd), float(fill), dtype=torch.bfloat16, device="cuda"), None
    codes = torch.full((pages, 2, nkv, 16, hd), fill, dtype=torch.uint8, device="cuda")
    return codes.view(torch.float8_e4m3fn), torch.full((pages, 2, nkv, 16), fill, dtype=torch.uint8, device="cuda")


def _adverse_rows(torch, n, hd, gen):
    """Rows where an exponent or a rounding can go wrong."""
    x = torch.randn((n, hd), generator=gen, device="cuda")
    rows = [torch.zeros(hd), torch.full((hd,), 448.0), torch.full((hd,), 448.0 * 2 ** -9), torch.full((hd,), 450.0),
            torch.linspace(-1, 1, hd), torch.tensor([2.0 ** -i for i in range(hd)]), torch.full((hd,), 1e-38),
            torch.full((hd,), 3e38), torch.full((hd,), -2.0 ** -126), torch.arange(hd) * 1.0 + 0.5,
            torch.tensor([448.0] + [2.0 ** -10 * (i % 7) for i in range(hd - 1)]),
            torch.tensor([-256.0] + [(16 + (i % 16)) * 0.5 + 0.25 for i in range(hd - 1)])]
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
    k = _adverse_rows(torch, n * nkv, hd, gen).view(n, nkv, hd).to(dt)
    v = (0.01 * torch.randn((n, nkv, hd), generator=gen, device="cuda")).to(dt)
    if dtype == "float16":
        k = k.clamp(-65504, 65504)
    pool, exps = _pool(torch, pages, nkv, hd, True, fill=3)
    slots = torch.randperm(pages * 16, generator=torch.Generator().manual_seed(1))[:n].cuda()
    slots[5], slots[9], slots[11] = -1, pages * 16, -(1 << 40)
    kp.cache_write(pool, slots, k, v, exponents=exps)
    codes, want_c, want_e = pool.view(torch.uint8).cpu(), torch.full(pool.shape, 3, dtype=torch.uint8), \
        torch.full(exps.shape, 3, dtype=torch.uint8)
    for t in range(n):
        slot = int(slots[t])
        if not 0 <= slot < pages * 16:
            continue
        for i, x in enumerate((k, v)):
            for h in range(nkv):
                c, e = ref.quantise(x[t, h].double())
                want_c[slot // 16, i, h, slot % 16], want_e[slot // 16, i, h, slot % 16] = c, e
    assert torch.equal(exps.cpu(), want_e)
    assert torch.equal(codes, want_c)
    # and read back: what the codes stand for, exactly (bf16 holds it while it is a normal number)
    out = torch.full((pages + 2, 2, nkv, 16, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    src = torch.tensor([0, 3, pages - 1, pages, -1, 2], dtype=torch.int32, device="cuda")
    dst = torch.tensor([1, 0, pages + 1, 4, 5, pages + 2], dtype=torch.int32, device="cuda")
    assert kp.cache_expand(pool, exps, src, out, dst) is out
    values = ref.e4m3_values()[want_c.long()] * 2.0 ** (want_e.double() - 127)[..., None]
    for s, d in ((0, 1), (3, 0), (pages - 1, pages + 1)):
        assert torch.equal(out[d].cpu(), values[s].bfloat16())
    rest = [i for i in range(pages + 2) if i not in (0, 1, pages + 1)]
    assert bool((out[rest] == 7.0).all())
    whole = torch.zeros((pages, 2, nkv, 16, hd), dtype=torch.bfloat16, device="cuda")
    kp.cache_expand(pool, exps, torch.arange(pages, dtype=torch.int32, device="cuda"), whole)
    assert torch.equal(whole.cpu(), values.bfloat16())


def test_write_not_finite():
    """Infinities become the largest code of the rest's scale; a row with a NaN reads as NaN, here and in attention."""
    torch, kp = _kp()
    pool, exps = _pool(torch, 2, 2, 64, True)
    k = torch.ones((3, 2, 64), device="cuda")
    k[0, 0, 3], k[0, 1, 5], k[1, 0, 0], k[1, 1] = math.inf, -math.inf, math.nan, math.inf
    kp.cache_write(pool, torch.tensor([0, 1, 17], device="cuda"), k, torch.zeros_like(k), exponents=exps)
    out = torch.zeros((2, 2, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    kp.cache_expand(pool, exps, torch.arange(2, dtype=torch.int32, device="cuda"), out)
    big = 448 * 2.0 ** -8
    assert out[0, 0, 0, 0, 3] == big and out[0, 0, 1, 0, 5] == -big and out[0, 0, 0, 0, 4] == 1
    assert bool(out[0, 0, 0, 1].isnan().all()) and bool((out[0, 0, 1, 1] == 448 * 2.0 ** -127).all())
    assert bool((out[1, 0, :, 1] == 1).all()) and bool((out[:, 1] == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("e4m3", [True, False])
@pytest.mark.parametrize("interleaved,rd,hd", [(False, 128, 128), (True, 128, 128), (False, 64, 64), (False, 32, 128),
                                               (True, 32, 64), (False, 34, 64), (True, 22, 128)])
@pytest.mark.parametrize("n,offset", [(5, 0), (700, 1)])
def test_write_rotates(dtype, e4m3, interleaved, rd, hd, n, offset):
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
    pool, exps = _pool(torch, pages, nkv, hd, e4m3)
    kp.cache_write(pool, slots, k, v, exponents=exps, rope=rope, positions=pos)
    want = torch.stack([ref.rotate(k, pos, ref.frequencies(rd), interleaved), v.double()], 1)   # [n][2][nkv][hd]
    near = 1.2e-6 * want.abs().amax(-1, keepdim=True) * math.sqrt(2)   # of the rotation, as in _rope_bound
    page, place = slots // 16, slots % 16
    got = pool[page, :, :, place].double() if not e4m3 else \
        pool.view(torch.uint8)[page, :, :, place].view(torch.float8_e4m3fn).double()
    if not e4m3:
        assert ((got - want).abs() <= near + UNIT["bfloat16"] * want.abs() + 1e-38).all()
        return
    e = exps[page, :, :, place].double() - 127
    most = want.abs().amax(-1)
    least, top = (torch.ceil(torch.log2((most * f).clamp(min=1e-300) / 448)) for f in (1 - 1e-6, 1 + 1e-6))
    assert bool(((e >= least) & (e <= top)).all())
    scale = torch.exp2(e)[..., None]
    # half a step of e4m3 at the value: 2^-4 of its power of two, at least 2^-10 of the row's scale
    step = torch.exp2(torch.floor(torch.log2((want.abs() / scale).clamp(min=2.0 ** -6)))) * 2.0 ** -4 * scale
    assert ((got * scale - want).abs() <= step * (1 + 1e-5) + near).all()


def test_write_empty_and_refusals():
    torch, kp = _kp()
    pool, exps = _pool(torch, 2, 2, 64, True)
    x = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    kp.cache_write(pool, slots[:0], x[:0], x[:0], exponents=exps)
    empty, _ = _pool(torch, 0, 2, 64, False)
    kp.cache_write(empty, slots, x, x)
    rope, pos = kp.Rope(64), slots.int()
    for args, kw in (((pool, slots, x, x), {}), ((pool, slots.int(), x, x), dict(exponents=exps)),
                     ((pool, slots[:2], x, x), dict(exponents=exps)),
                     ((pool, slots, x[:, :1], x[:, :1]), dict(exponents=exps)),
                     ((pool, slots, x, x.half()), dict(exponents=exps)),
                     ((pool, slots, x, x), dict(exponents=exps.int())),
                     ((pool, slots, x, x), dict(exponents=exps[:1])),
                     ((pool, slots, x, x), dict(exponents=exps, rope=rope)),
                     ((pool, slots, x, x), dict(exponents=exps, positions=pos)),
                     ((pool.view(torch.uint8), slots, x, x), dict(exponents=exps)),
                     ((pool.transpose(0, 2), slots, x, x), dict(exponents=exps)),
                     ((pool.cpu(), slots, x, x), dict(exponents=exps.cpu()))):
        with pytest.raises((ValueError, TypeError)):
            kp.cache_write(*args, **kw)
    with pytest.raises(ValueError):
        kp.cache_write(empty, slots, x, x, exponents=exps)
    with pytest.raises(kp.KvprmError):
        kp.cache_write(pool, slots, x, x, exponents=exps, rope=kp.Rope(128), positions=pos)
    with pytest.raises(ValueError):
        kp.cache_expand(pool, exps, pos, torch.zeros((2, 2, 2, 16, 64), device="cuda"))


# ---------------------------------------------------------------- tree attention
class Tree:
    """Sequences with caches in scattered pages of a pool whose unused places hold NaN (exponents: anything)."""

    def __init__(self, torch, nq, nkv, hd, lens, drafts, e4m3=False, mask="tree", seed=0, q_std=2.0, extra_pages=5,
                 max_blocks=None):
        self.torch, self.nq, self.nkv, self.hd, self.lens, self.drafts = torch, nq, nkv, hd, list(lens), list(drafts)
        gen, rng = _gen(torch, seed), random.Random(seed)
        blocks = [(n + 15) // 16 for n in lens]
        n_pages = sum(blocks) + extra_pages
        self.width = max([1] + blocks) if max_blocks is None else max_blocks
        order = list(range(n_pages))
        rng.shuffle(order)
        table = [[-7] * self.width for _ in lens]
        shape = (n_pages, 2, nkv, 16, hd)
        values = _randn(torch, shape, gen, torch.float32)
        values[:, 1] += 0.3   # values with a mean: a dropped or doubled key shows
        used = torch.zeros(n_pages, 16, dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(blocks[b]):
                p = order.pop()
                table[b][j] = p
                used[p, :max(0, min(16, n - 16 * j))] = True
        used = used.cuda()[:, None, None, :]
        if e4m3:
            self.exps = torch.randint(117, 124, shape[:4], generator=gen, device="cuda", dtype=torch.uint8)
            codes = (values * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
            self.values = codes.double() * torch.exp2(self.exps.double() - 127)[..., None]
            codes.view(torch.uint8)[~used.expand(shape[:4])] = 0x7F
            self.exps[~used.expand(shape[:4])] = 255
            self.pages = codes
        else:
            self.exps = None
            self.pages = values.bfloat16()
            self.values = self.pages.double()
            self.pages[~used.expand(shape[:4])] = math.nan
        self.table = torch.tensor(table, dtype=torch.int32).view(len(table), self.width).cuda()
        self.start = [0]
        for t in drafts:
            self.start.append(self.start[-1] + t)
        n = self.start[-1]
        rows = _randn(torch, (n, nq + 2 * nkv, hd), gen, torch.bfloat16)
        self.q, self.k, self.v = rows[:, :nq], rows[:, nq:nq + nkv], rows[:, nq + nkv:]
        self.q.mul_(q_std)
        most = max([1] + list(drafts))
        if mask == "chain":
            self.mask = None
            self.seen = torch.zeros((n, most), dtype=torch.bool)
            for s, t in enumerate(drafts):
                self.seen[self.start[s]:self.start[s + 1], :t] = torch.ones((t, t), dtype=torch.bool).tril()
        else:
            if mask == "tree":
                import paper_2607_09153_gb300 as kp
                parents = [rng.randint(-1, i - 1) for t in drafts for i in range(t)]
                self.mask = kp.tree_mask(parents, self.start)
            elif mask == "none":   # nothing among the drafts
                self.mask = torch.zeros((n, (most + 31) // 32), dtype=torch.int32)
            else:                  # any bits at all, also of drafts that do not exist
                self.mask = torch.tensor([[rng.randint(-2 ** 31, 2 ** 31 - 1) for _ in range((most + 31) // 32)]
                                          for _ in range(n)], dtype=torch.int32).view(n, -1)
            self.seen = ref.unpack_mask(self.mask, most)
            for s, t in enumerate(drafts):
                self.seen[self.start[s]:self.start[s + 1], t:] = False
            self.mask = self.mask.cuda()
        self.seen = self.seen.cuda()

    def run(self, **kw):
        import paper_2607_09153_gb300 as kp
        torch = self.torch
        args = dict(max_drafts=max([1] + self.drafts), exponents=self.exps, mask=self.mask)
        args.update(kw)
        lens, start = (args.pop(k) if k in args else torch.tensor(v, dtype=torch.int32).cuda()
                       for k, v in (("lens", self.lens), ("start", self.start)))
        table = args.pop("table", self.table)
        return kp.tree_attention(args.pop("q", self.q), self.k, self.v, self.pages, table, lens, start, **args)

    def rows(self):
        out = []
        for b, n in enumerate(self.lens):
            ids = self.table[b, :(n + 15) // 16].long()
            kv = self.values[ids].permute(1, 0, 3, 2, 4).reshape(2, -1, self.nkv, self.hd)[:, :n]
            out.append((kv[0], kv[1]))
        return out

    def want(self, scale=None):
        scale = self.hd ** -0.5 if scale is None else scale
        o, a, peak = ref.attention(self.q, self.k, self.v, self.rows(), self.lens, self.start, self.seen, scale)
        most = max(n + t for n, t in zip(self.lens, self.drafts)) if self.lens else 0
        return o, ref.attention_bound(o, a, peak, most, self.hd)

    def check(self, out, scale=None):
        o, bound = self.want(scale)
        off = (out.double() - o).abs()
        assert bool((off <= bound).all()), f"off by {float((off / bound).max()):.2f} bounds"


HEADS = [(4, 2, 64), (1, 1, 128), (12, 2, 128), (7, 1, 64), (16, 1, 128), (6, 6, 64), (28, 4, 128)]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("nq,nkv,hd", HEADS)
def test_tree_small(nq, nkv, hd, e4m3):
    """Lengths about a page's and a block's ends, one token to a few."""
    torch, _ = _kp()
    t = Tree(torch, nq, nkv, hd, [0, 1, 15, 16, 17, 64, 65, 200], [1, 3, 2, 1, 17, 1, 5, 4], e4m3, seed=nq + hd)
    t.check(t.run())


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("nq,nkv,hd", [(4, 1, 64), (14, 2, 128), (3, 3, 128)])
@pytest.mark.parametrize("mask", ["tree", "chain", "none", "random"])
def test_tree_wide(nq, nkv, hd, mask, e4m3):
    """Drafts across mask words and row tiles, with rows that see nothing at all (empty caches, empty masks)."""
    torch, _ = _kp()
    t = Tree(torch, nq, nkv, hd, [130, 0, 1000, 127, 128, 129], [64, 33, 70, 1, 32, 31], e4m3, mask, seed=nkv)
    out = t.run()
    t.check(out)
    if mask == "none":
        assert bool((out[t.start[1]:t.start[2]] == 0).all())


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("lens,drafts", [([20011], [1]), ([20011], [9]), ([5000, 3, 7777], [40, 2, 33]),
                                         ([12345], [64]), ([0] * 3 + [9000] + [0] * 3, [1] * 7),
                                         ([14000, 9999] * 3, [9, 200, 6, 12, 40, 5])])
def test_tree_long(lens, drafts, e4m3):
    """Long caches, whose parts many CTAs score and one joins."""
    torch, _ = _kp()
    t = Tree(torch, 8, 2, 128, lens, drafts, e4m3, seed=len(lens), q_std=1.0)
    out = t.run()
    t.check(out)
    assert torch.equal(out, t.run())   # parts are joined in order, whichever CTA is last


def test_tree_many_sequences():
    """More sequences than one launch takes, some without drafted tokens."""
    torch, _ = _kp()
    rng = random.Random(4)
    t = Tree(torch, 2, 1, 64, [rng.randint(0, 40) for _ in range(1500)], [rng.randint(0, 2) for _ in range(1500)])
    t.check(t.run())


@pytest.mark.parametrize("e4m3", [False, True])
def test_tree_peaked(e4m3):
    """Scores hundreds of units apart, rising and falling along the cache: the running maximum moves again and again."""
    torch, _ = _kp()
    t = Tree(torch, 8, 2, 128, [999, 2048], [5, 40], e4m3, seed=9, q_std=40.0)
    t.check(t.run())
    t.check(t.run(scale=0.003), scale=0.003)
    t.check(t.run(scale=-0.05), scale=-0.05)


@pytest.mark.parametrize("drafts", [1, 20])
@pytest.mark.parametrize("exponent", [6, 8, 30, -40])
def test_tree_small_codes_count(drafts, exponent):
    """Rows of e4m3's subnormal codes alone (0 .. 7/8 2^-6), at scales on both sides of what one bf16 factor holds."""
    torch, kp = _kp()
    t = Tree(torch, 2, 1, 128, [64], [drafts], True, seed=3, q_std=2.0 ** -max(0, exponent))
    codes = t.pages.view(torch.uint8)
    codes[:] = torch.randint(0, 8, codes.shape, device="cuda", dtype=torch.uint8)
    t.exps[:] = 127 + exponent
    t.values = t.pages.double() * 2.0 ** exponent
    t.check(t.run())


@pytest.mark.parametrize("drafts", [1, 12, 20])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("weight", ["none", "alike"])
def test_tree_value_powers_apart(weight, hd, drafts):
    """Value rows up to 2^70 apart.  "none": the large ones have no weight at all; "alike": weights that fall as the powers
    rise, so that every power's rows count."""
    torch, kp = _kp()
    t = Tree(torch, 2, 1, hd, [333, 40], [drafts, 1], True, seed=13, q_std=0.25)
    t.q[..., 0] = 16.0
    away = torch.randint(-30, 41, t.exps[:, 1].shape, generator=_gen(torch, 14), device="cuda")
    nat = away.double() * math.log(2.0) * hd ** 0.5 / 16   # of dimension 0 of a key: e^-(away ln 2)
    if weight == "none":
        nat = torch.where(away > 0, 400.0, 0.0)
    t.exps[:, 0], t.exps[:, 1] = 127, (120 + away).to(torch.uint8)
    t.pages[:, 0, ..., 0] = (-nat).clamp(-448, 448).to(torch.float8_e4m3fn)
    t.pages[:, 0, ..., 1:] = (_randn(torch, t.pages[:, 0, ..., 1:].shape, _gen(torch, 15), torch.float32) * 0.5).to(
        torch.float8_e4m3fn)
    t.pages[:, 1] = (_randn(torch, t.pages[:, 1].shape, _gen(torch, 16), torch.float32) * 100).clamp(-448, 448).to(
        torch.float8_e4m3fn)
    t.values = t.pages.double() * torch.exp2(t.exps.double() - 127)[..., None]
    t.check(t.run())


@pytest.mark.parametrize("e4m3", [False, True])
def test_tree_not_finite(e4m3):
    """Drafts that are not finite reach the rows that see them and no others; a NaN in the cache reaches its sequence."""
    torch, _ = _kp()
    t = Tree(torch, 4, 2, 64, [50, 0, 33], [20, 40, 2], e4m3, seed=6)
    want, bound = t.want()
    hurt = torch.zeros(t.q.shape[0], dtype=torch.bool, device="cuda")
    for s, j, x, i in ((0, 3, t.v, math.nan), (0, 18, t.v, math.inf), (1, 35, t.k, math.nan), (1, 20, t.v, -math.inf)):
        x[t.start[s] + j, :, 7] = i
        hurt[t.start[s]:t.start[s + 1]] |= t.seen[t.start[s]:t.start[s + 1], j]
    out = t.run()
    ok = (out.double() - want).abs() <= bound
    assert bool(ok[~hurt].all()) and bool(out[hurt].isnan().any(-1).all())
    assert 0 < int(hurt.sum()) < t.q.shape[0]
    page = int(t.table[2, 0])
    if e4m3:
        t.exps[page, 0, 0, 5] = 255
    else:
        t.pages[page, 0, 0, 5, 1] = math.nan
    out = t.run()
    assert bool(out[t.start[2]:, :2].isnan().all()) and bool(ok[t.start[2]:, 2:].all())


@pytest.mark.parametrize("e4m3", [False, True])
def test_tree_bad_tables(e4m3):
    """What the host cannot see: NaN for a sequence with a bad page or length, others untouched; bad drafts left out."""
    torch, _ = _kp()
    t = Tree(torch, 4, 2, 64, [50, 40, 33, 300], [3, 4, 5, 40], e4m3, seed=8)
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
    o = t.run(start=i32([0, 3, 7, 12, 53]), out=out)   # the last sequence's drafts pass the end
    assert fine(o, 0) and fine(o, 1) and fine(o, 2) and bool((o[12:] == 5.0).all())
    o = t.run(start=i32([-3, 3, 7, 2, 52]), out=torch.full_like(out, 5.0))
    assert bool((o[:3] == 5.0).all()) and fine(o, 1)
    o = t.run(max_drafts=39, out=torch.full_like(out, 5.0))
    assert fine(o, 2) and bool((o[12:] == 5.0).all())


def test_tree_far_pages():
    """Pages beyond 2^31 elements and 2^32 bytes of the pool."""
    torch, kp = _kp()
    n_pages, nkv, hd = 70000, 8, 128
    t = Tree(torch, 16, nkv, hd, [70, 17], [3, 20], seed=2)
    pool = torch.empty((n_pages, 2, nkv, 16, hd), dtype=torch.bfloat16, device="cuda")
    far = torch.full_like(t.table, -7)
    for b, n in enumerate(t.lens):
        for j in range((n + 15) // 16):
            to = n_pages - 1 - 7 * j - b
            pool[to] = t.pages[int(t.table[b, j])]
            far[b, j] = to
    near = t.run()
    t.pages = pool
    assert torch.equal(near, t.run(table=far))
    # a token written that far out, and the quantised page there read back
    slots = torch.tensor([(n_pages - 1) * 16 + 3], device="cuda")
    kp.cache_write(pool, slots, t.k[:1], t.v[:1])
    assert torch.equal(pool[-1, 0, :, 3], t.k[0]) and torch.equal(pool[-1, 1, :, 3], t.v[0])
    del pool
    t.pages = None
    n_pages = 140000
    codes, exps = _pool(torch, n_pages, nkv, hd, True)
    kp.cache_write(codes, torch.tensor([(n_pages - 1) * 16 + 3], device="cuda"), t.k[:1], t.v[:1], exponents=exps)
    out = torch.zeros((1, 2, nkv, 16, hd), dtype=torch.bfloat16, device="cuda")
    kp.cache_expand(codes, exps, torch.tensor([n_pages - 1], dtype=torch.int32, device="cuda"), out)
    c, e = ref.quantise(t.v[0, 5].double())
    assert torch.equal(out[0, 1, 5, 3].cpu(), (ref.e4m3_values()[c.long()] * 2.0 ** (e - 127)).bfloat16())


@pytest.mark.parametrize("e4m3", [False, True])
def test_tree_strides(e4m3):
    """Other orders of the heads' and tokens' strides, and an output of its own strides: the same bits."""
    torch, _ = _kp()
    t = Tree(torch, 6, 2, 64, [40, 100], [5, 30], e4m3, seed=12)
    a = t.run()
    out = torch.full((6, 35, 72), 3.0, dtype=torch.bfloat16, device="cuda")
    t.k, t.v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (t.k, t.v))
    b = t.run(q=t.q.contiguous(), out=out[..., :64].transpose(0, 1))
    assert torch.equal(a, b) and bool((out[..., 64:] == 3.0).all())
    t.check(t.run(max_len=1))   # another launch size may sum in another order


def test_tree_streams():
    """Calls on several streams at once, each with scratch of its own, and one captured into a graph."""
    torch, _ = _kp()
    t = Tree(torch, 8, 2, 128, [6000, 5000], [12, 3], seed=13)
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
    lens[0] = 77   # the lengths are the device's: the same graph on other lengths
    t.lens[0] = 77
    g.replay()
    torch.cuda.synchronize()
    t.check(out)


def test_tree_refusals():
    torch, kp = _kp()
    t = Tree(torch, 4, 2, 64, [40, 10], [3, 2], seed=1)
    assert t.run(q=t.q, mask=t.mask).shape == t.q.shape
    for kw in (dict(mask=t.mask[:3]), dict(mask=t.mask.long()), dict(q=t.q[:3]), dict(q=t.q.float()), dict(q=t.q[..., :32]),
               dict(exponents=t.mask), dict(table=t.table.long()), dict(table=t.table[0]),
               dict(out=torch.empty((5, 4, 64), device="cuda")), dict(out=torch.empty((5, 4, 32), dtype=t.q.dtype, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            t.run(**kw)
    for kw in (dict(max_drafts=0), dict(max_drafts=2000), dict(scale=math.nan), dict(q=t.q[:, :3]),
               dict(workspace=torch.zeros(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(kp.KvprmError) as e:
            t.run(**kw)
        assert "kvprm_tree" in str(e.value)
    odd = torch.zeros((5, 4, 72), dtype=torch.bfloat16, device="cuda")[..., 4:68]
    with pytest.raises(kp.KvprmError):
        t.run(q=odd)
    none = Tree(torch, 4, 2, 64, [], [])
    assert none.run().shape == (0, 4, 64)
