"""Attention over 4-bit pages at the ends of what its rows can hold, up to 32 query rows of a kv head: against the definition in 64
bits, as tests/test_gpu_cache4.py, on calls whose pairs are whole (a CTA each, or several) and cut (parts that are joined)."""
import pytest

from tests.cache4_util import Tree4
from tests.test_gpu_operators import _kp

pytestmark = pytest.mark.gpu
# (lens, drafts, kv heads): whole pairs, a CTA each; several of a CTA; parts of long ones, beside short ones that one warp has
CALLS = {"whole": ([64, 17, 300], [1, 3, 2], 2), "many": ([40 + i for i in range(150)], [1] * 150, 4),
         "cut": ([5000, 17, 3000], [1, 2, 3], 2), "cut_rows": ([5000, 17], [8, 5], 2)}


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("q_std", [2.0, 0.0])
def test_large_cached_values(call, q_std):
    """Values up to 2^120, whose sum over the keys no fp32 number holds, though bf16 holds their mean; equal weights among them."""
    torch, _ = _kp()
    lens, drafts, nkv = CALLS[call]
    t = Tree4(torch, 2 * nkv, nkv, 128, lens, drafts, seed=41, q_std=q_std)
    t.exps[:, 1] += 117                      # 123 .. 126 (and, where nobody looks, 255)
    t.remake()
    out = t.run()
    assert bool(out.isfinite().all())
    t.check(out)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("far", [0, 60, -60])
def test_large_drafted_values(call, far):
    """Drafted values up to 2^120 beside cached ones of about one, 2^60 and 2^-60."""
    torch, _ = _kp()
    lens, drafts, nkv = CALLS[call]
    t = Tree4(torch, 2 * nkv, nkv, 64, lens, drafts, seed=42)
    t.exps[:, 1] = (t.exps[:, 1].int() + far).clamp(max=255).to(torch.uint8)
    t.remake()
    t.v.mul_(2.0 ** 118)
    out = t.run()
    assert bool(out.isfinite().all())
    t.check(out)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("apart", [17, 20, 31, 45])
@pytest.mark.parametrize("some", [False, True])
def test_queries_far_apart(call, apart, some):
    """Query rows (all, or a sequence's first drafted token's alone) with one element 2^apart of the others, where all keys are zero: the
    scores are made of the small ones, with keys that make up for it."""
    torch, _ = _kp()
    lens, drafts, nkv = CALLS[call]
    t = Tree4(torch, 2 * nkv, nkv, 128, lens, drafts, seed=43)
    rows = t.start[:-1] if some else slice(None)
    t.q[rows] *= 2.0 ** -apart
    t.q[rows, :, 5] = 1.5
    t.pages[:, 0, :, :, 2] &= 0x0F           # dimension 5
    t.k[:, :, 5] = 0
    if some:                                 # (the other rows' scores: keys are as large for them)
        others = [i for i in range(t.q.shape[0]) if i not in rows]
        t.q[others] *= 2.0 ** -apart
    t.exps[:, 0] = (t.exps[:, 0].int() + apart).clamp(max=254).to(torch.uint8)
    t.k.mul_(2.0 ** apart)
    t.remake()
    t.check(t.run())


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("mixed", [False, True])
def test_keys_of_the_least_power(call, mixed):
    """Key blocks with the least exponent byte, 0, whose codes are not zero, with queries of 2^124; others' beside them."""
    torch, _ = _kp()
    lens, drafts, nkv = CALLS[call]
    t = Tree4(torch, 2 * nkv, nkv, 64, lens, drafts, seed=44)
    least = torch.rand(t.exps[:, 0].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) < (0.4 if mixed else 2)
    t.exps[:, 0] = torch.where(least, 0, t.exps[:, 0] - 121)   # 0, and 2 .. 5
    t.q.mul_(2.0 ** 124)
    t.k.mul_(2.0 ** -125)
    t.remake()
    t.check(t.run())


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("mixed", [False, True])
def test_values_of_the_least_power(call, mixed):
    """Value blocks with the least exponent byte: outputs among the least that bf16 holds, in steps of 2^-133."""
    torch, _ = _kp()
    lens, drafts, nkv = CALLS[call]
    t = Tree4(torch, 2 * nkv, nkv, 64, lens, drafts, mask="none", seed=45)
    least = torch.rand(t.exps[:, 1].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) < (0.4 if mixed else 2)
    t.exps[:, 1] = torch.where(least, 0, t.exps[:, 1] - 121)
    t.remake()
    want, bound = t.want()
    assert bool(((t.run().double() - want).abs() <= bound - 1e-30 + 2.0 ** -133).all())
