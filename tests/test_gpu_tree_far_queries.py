"""Attention over 8-bit pages with query rows at the ends of bf16's range, and with elements far apart."""
import pytest

from tests.test_gpu_operators import Tree, _kp

pytestmark = pytest.mark.gpu
CALLS = {"short": ([64, 17, 300], [1, 3, 2]), "long": ([5000, 17, 3000], [1, 2, 3]), "rows": ([5000, 17, 40], [8, 5, 16])}


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("apart", [17, 20, 31])
def test_queries_far_apart(call, apart):
    """One element of a query row is 2^apart of the others, where all keys are zero: the scores are made of the small ones, with keys
    that make up for it."""
    torch, _ = _kp()
    lens, drafts = CALLS[call]
    t = Tree(torch, 4, 2, 128, lens, drafts, True, seed=43)
    t.q.mul_(2.0 ** -apart)
    t.q[..., 5] = 1.5
    t.pages.view(torch.uint8)[:, 0, ..., 5] = 0
    t.values[:, 0, ..., 5] = 0
    t.k[..., 5] = 0
    fine = t.exps[:, 0] < 255
    t.exps[:, 0] = torch.where(fine, t.exps[:, 0].int() + apart, 255).to(torch.uint8)
    t.values[:, 0] *= 2.0 ** apart
    t.k.mul_(2.0 ** apart)
    t.check(t.run())


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("up", [True, False])
def test_queries_at_the_ends(call, up):
    """Whole query rows beyond 2^127 or below 2^-126, with keys that make up for it."""
    torch, _ = _kp()
    lens, drafts = CALLS[call]
    t = Tree(torch, 4, 2, 128, lens, drafts, True, seed=31)
    power, keys = (125, -110) if up else (-130, 120)
    t.q.copy_((t.q.double() * 2.0 ** power).clamp(-3e38, 3e38))
    fine = t.exps[:, 0] < 255
    t.exps[:, 0] = torch.where(fine, t.exps[:, 0].int() + keys, 255).to(torch.uint8)
    t.values[:, 0] *= 2.0 ** keys
    t.k.mul_(2.0 ** keys)
    scale = 2.0 ** (-15 if up else 10) * 128 ** -0.5
    t.check(t.run(scale=scale), scale)
