"""Strides that belong to nobody: of a dimension of one element, and of tensors without any."""
import pytest

from tests.gpu_util import require_gpu
from tests.test_gpu_operators import Tree, _pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
def test_one_token_of_odd_rows(e4m3):
    """A drafted token cut out of rows that are no multiple of 16 bytes apart; one kv head between others'."""
    torch = require_gpu()
    t = Tree(torch, 4, 1, 64, [77], [1], e4m3, seed=3)
    a = t.run()
    rows = torch.zeros((3, 6 * 64 + 4), dtype=torch.bfloat16, device="cuda")
    for name, at, n in (("q", 0, 4), ("k", 4, 1), ("v", 5, 1)):
        x = torch.as_strided(rows, (1, n, 64), (rows.stride(0), 64 if n > 1 else 3, 1), 64 * at)
        x.copy_(getattr(t, name))
        setattr(t, name, x)
    out = torch.as_strided(torch.zeros(9 * 64, dtype=torch.bfloat16, device="cuda"), (1, 4, 64), (5, 64, 1), 64)
    assert torch.equal(t.run(out=out), a) and torch.equal(t.run(), a)
    t.check(a)


def test_empty_tensors():
    """No tokens, whatever the strides say."""
    torch = require_gpu()
    import paper_2607_09153_gb300 as kp
    none = torch.as_strided(torch.zeros(1, device="cuda"), (0, 2, 64), (0, 0, 0))
    rope, pos = kp.Rope(64), torch.zeros(0, dtype=torch.int32, device="cuda")
    assert rope.rotate(pos, none)[0].shape == (0, 2, 64)
    pool, exps = _pool(torch, 2, 2, 64, True, fill=5)
    kp.cache_write(pool, pos.long(), none, none, exponents=exps, rope=rope, positions=pos)
    assert bool((pool.view(torch.uint8) == 5).all())
    none, start = none.bfloat16(), torch.zeros(1, dtype=torch.int32, device="cuda")
    none = torch.as_strided(none, (0, 2, 64), (0, 0, 0))
    out = kp.tree_attention(none, none, none, pool, pos.view(0, 1), pos, start, max_drafts=1, exponents=exps)
    assert out.shape == (0, 2, 64)
    empty = torch.as_strided(torch.zeros(1, device="cuda"), (3, 0, 64), (0, 0, 0))
    assert rope.rotate(torch.zeros(3, dtype=torch.int32, device="cuda"), empty)[0].shape == (3, 0, 64)


def test_a_head_is_still_side_by_side():
    torch = require_gpu()
    import paper_2607_09153_gb300 as kp
    x = torch.zeros((3, 2, 128), device="cuda")[..., ::2]
    with pytest.raises(ValueError, match="side by side"):
        kp.Rope(64).rotate(torch.zeros(3, dtype=torch.int32, device="cuda"), x)
