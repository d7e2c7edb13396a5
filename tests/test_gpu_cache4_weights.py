"""Weights over 4-bit pages are fp16 up to 32 query rows of a kv head: a bound that weights in bf16 do not keep."""
import pytest

from tests import operators_util as ref
from tests.cache4_util import Tree4
from tests.test_gpu_operators import _kp

pytestmark = pytest.mark.gpu


def _bound(o, a, values):
    """How far an output may be: each weight is rounded to fp16 (2^-11 of it, where bf16 takes 2^-8; below 2^-26 of the largest 2^-37 of
    that, for all the values); the scores' sums of these queries and keys are whole numbers of 2^-3 below 2^9, exact in any order, so a
    score below 2^5, in units of log2, has two roundings of 2^-24 of it, a difference of scores a third, and exp2 adds 2^-21: 2^-17 of a
    weight; up to 200 fp32 additions of sums (a page's 16 keys and more at a time): 2^-16; the output's rounding to bf16."""
    return (2.0 ** -11 + 2.0 ** -17 + 2.0 ** -16) * a + 2.0 ** -37 * values + 2.0 ** -8 * o.abs() + 1e-30


@pytest.mark.parametrize("lens", [[30] * 8, [3000] * 8, [30 + i % 50 for i in range(300)]])
@pytest.mark.parametrize("drafts", [1, 2, 4])
@pytest.mark.parametrize("hd", [64, 128])
def test_opposite_values(lens, drafts, hd):
    """Three keys of a sequence, wherever they are, outweigh the others by 2^30: one of no value, and two of about half its weight, whose
    values are opposite.  What is left of them is small, and a weight's rounding shows."""
    torch, _ = _kp()
    nkv, group = 2, 8
    t = Tree4(torch, nkv * group, nkv, hd, lens, [drafts] * len(lens), mask="none", seed=hd + drafts)
    gen = torch.Generator(device="cuda").manual_seed(1)
    t.q.copy_(1 + torch.randint(-2, 3, t.q.shape, generator=gen, device="cuda") / 16)
    t.pages[:, 0], t.exps[:, 0] = 0, 0
    t.exps[:, 1] = 127
    high, low, count = (5, 4, 6) if hd == 64 else (4, 3, 16)   # (codes: 3 and 2 in six places, 2 and 1.5 in sixteen)
    for s, n in enumerate(lens):
        places = 5 * s % 11, 11 + s % 6, n - 1 - 3 * s % 13
        assert len(set(places)) == 3
        at = [(int(t.table[s, x // 16]), x % 16) for x in places]
        for i, (p, x) in enumerate(at):
            t.exps[p, 0, :, x] = 127
            t.pages[p, 0, :, x] = 17 * high
            if i:   # in the low halves of bytes of its own
                t.pages[p, 0, :, x, i - 1:i - 1 + 2 * count:2] = 16 * high + low
        t.pages[at[0][0], 1, :, at[0][1]] = 0
        t.pages[at[2][0], 1, :, at[2][1]] = t.pages[at[1][0], 1, :, at[1][1]] ^ 0x88
    t.remake()
    rows, scale = t.rows(), hd ** -0.5
    want, a, _ = ref.attention(t.q, t.k, t.v, rows, t.lens, t.start, t.seen, scale)
    bound = _bound(want, a, torch.cat([v.abs().sum(0).repeat_interleave(group, 0).expand(drafts, -1, -1) for _, v in rows]))
    assert bool(((t.run().double() - want).abs() <= bound).all())
    # what weights in bf16 would make of it
    worse = torch.empty_like(want)
    for s, (k, v) in enumerate(rows):
        at = slice(t.start[s], t.start[s + 1])
        k, v = (x.repeat_interleave(group, 1) for x in (k, v))
        w = torch.einsum("thd,khd->thk", t.q[at].double(), k) * scale
        w = (w - w.amax(-1, keepdim=True)).exp()
        worse[at] = torch.einsum("thk,khd->thd", (4096 * w).bfloat16().double(), v) / (4096 * w).sum(-1, keepdim=True)
    share = float(((worse - want).abs() > bound).any(-1).double().mean())
    assert share > 0.2, share
