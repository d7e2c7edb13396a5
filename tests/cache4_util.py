"""4-bit pages and the pages' bookkeeping by their definitions (plain torch in 64 bits, plain Python), for the tests."""
import math

import torch

from tests.test_gpu_operators import Tree, _gen, _randn

VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def block_exponent(most):
    """The least e >= -127 with most <= 6 2^e (most a Python float)."""
    e = -127
    while most > 6 * 2.0 ** e:
        e += 1
    return e


def codes_of(y):
    """e2m1 codes (0 .. 15) of 64-bit values, to nearest, ties to the even code, at most 6."""
    grid = torch.tensor(VALUES, dtype=torch.float64, device=y.device)
    m = y.abs().clamp(max=6.0)
    hi = torch.searchsorted(grid, m.contiguous()).clamp(max=7)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - m, m - grid[lo]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code + 8 * torch.signbit(y).long()).to(torch.uint8)


def pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def values(pages, exps):
    """What 4-bit rows stand for, in 64 bits; NaN where the exponent is 255."""
    grid = torch.tensor(VALUES + [-v for v in VALUES], dtype=torch.float64, device=pages.device)
    y = torch.stack([grid[(pages & 15).long()], grid[(pages >> 4).long()]], -1).flatten(-2)
    power = torch.where(exps == 255, math.nan, torch.exp2(exps.double() - 127))
    return (y.unflatten(-1, (-1, 32)) * power[..., None]).flatten(-2)


def quantise(rows):
    """(pages, exponents) of finite rows [...][head_dim] in 64 bits."""
    y = rows.unflatten(-1, (-1, 32))
    e = torch.tensor([block_exponent(float(m)) for m in y.abs().amax(-1).flatten()], device=rows.device).view(y.shape[:-1])
    return pack(codes_of(y * torch.exp2(-e.double())[..., None]).flatten(-2)), (e + 127).to(torch.uint8)


class Tree4(Tree):
    """Tree over 4-bit pages; blocks that nobody may read have the exponent of NaN."""

    def __init__(self, torch, nq, nkv, hd, lens, drafts, mask="tree", seed=0, q_std=2.0, spread=4, **kw):
        super().__init__(torch, nq, nkv, hd, lens, drafts, False, mask, seed, q_std, **kw)
        gen = _gen(torch, seed + 1000)
        shape = self.pages.shape
        unused = self.pages[..., 0].isnan()
        rows = _randn(torch, shape, gen, torch.float32, 2.2).double()
        rows[:, 1] += 0.5
        self.pages = pack(codes_of(rows))
        self.exps = torch.randint(127 - spread, 127, shape[:-1] + (hd // 32,), generator=gen, device="cuda", dtype=torch.uint8)
        self.values = values(self.pages, self.exps)
        self.exps[unused] = 255

    def want(self, scale=None):
        """Tree's, whose bound takes every weight to be off by 2^-8 of itself at most.  Up to 32 query rows' weights over 4-bit
        pages are fp16 (a tighter 2^-11), times 2^12 over that of the running maximum, a score that was met: the largest is
        stored as 2^12 or more.  Below 2^-14 a stored weight is off by up to half a step, 2^-25, so by 2^-37 of the largest,
        and an output by as much of all the cached values that the weights multiply."""
        o, bound = super().want(scale)
        group = self.nq // self.nkv
        for s, (_, vals) in enumerate(self.rows()):
            at = slice(self.start[s], self.start[s + 1])
            bound[at] += 2.0 ** -37 * vals.abs().sum(0).repeat_interleave(group, 0)
        return o, bound

    def remake(self):
        """After a change of pages or exponents."""
        self.values = values(self.pages, self.exps)
        self.values[self.values.isnan()] = 0.0   # (of places that are not looked at)


class Pool:
    """A search's pages as the definition moves them, by plain Python; pages: a token that marks what each page holds."""

    def __init__(self, refs, table, lens):
        self.refs, self.table, self.lens = list(refs), [list(r) for r in table], list(lens)
        self.n = len(self.refs)

    def _held(self, s):
        n = self.lens[s]
        return -(-n // 16) if 0 <= n <= 16 * len(self.table[s]) else 0

    def fork(self, parents, room, width):
        """(table, lens, refs, counts, copies)."""
        n, refs, inside = len(self.lens), self.refs, lambda p: 0 <= p < self.n  # noqa: E731
        parents = [p if 0 <= p < n else None for p in parents]
        after = list(refs)
        for s in range(n):
            for p in self.table[s][:self._held(s)]:
                if inside(p):
                    after[p] -= 1
        ends = []
        for p in parents:
            held = 0 if p is None else min(self._held(p), width)
            full = 0 if p is None or not held else self.lens[p] // 16
            for page in [] if p is None else self.table[p][:min(full, width)]:
                if inside(page):
                    after[page] += 1
            end = self.table[p][full] if p is not None and full < held else None
            ends.append(end if end is not None and inside(end) else None)
        kept = {}
        for i, end in enumerate(ends):
            if end is not None and after[end] <= 0:
                kept.setdefault(end, i)
        for page in kept:
            after[page] = 1
        free = [p for p in range(self.n) if after[p] <= 0]
        short, table, lens, copies = 0, [], [], []

        def take():
            nonlocal short
            if not free:
                short += 1
                return -1
            after[free[0]] = 1
            return free.pop(0)

        for i, (p, end, more) in enumerate(zip(parents, ends, room)):
            length = 0 if p is None else self.lens[p]
            held = 0 if p is None else min(self._held(p), width)
            row = [] if p is None else self.table[p][:held]
            if end is not None and kept.get(end) != i:
                row[length // 16] = take()
                if row[length // 16] >= 0:
                    copies.append((end, row[length // 16]))
            bad = p is not None and self._held(p) == 0 and length != 0
            want = 0 if bad else -(-(length + max(0, more)) // 16)
            row += [take() for _ in range(min(want, width) - len(row))]
            short += max(0, want - max(len(row), min(want, width)))
            table.append(row + [-1] * (width - len(row)))
            lens.append(length)
        return table, lens, after, [len(free), short], copies

    def compact(self):
        """(table, refs, moved, counts, copies)."""
        live = [p for p in range(self.n) if self.refs[p] > 0]
        holes = [p for p in range(len(live)) if self.refs[p] <= 0]
        high = [p for p in live if p >= len(live)]
        moved = [p if self.refs[p] > 0 else -1 for p in range(self.n)]
        refs = [r if r > 0 and p < len(live) else 0 for p, r in enumerate(self.refs)]
        for a, b in zip(high, holes):
            moved[a], refs[b] = b, self.refs[a]
        table = [[(moved[p] if 0 <= p < self.n else p) if b < self._held(s) else -1 for b, p in enumerate(row)]
                 for s, row in enumerate(self.table)]
        return table, refs, moved, [len(live), len(high)], list(zip(high, holes))
