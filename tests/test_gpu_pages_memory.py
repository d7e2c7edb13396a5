"""What cache_fork and cache_compact may write: pools that share memory are refused, and pages that somebody still holds are left as
they were, whatever the call came to."""
import pytest

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
