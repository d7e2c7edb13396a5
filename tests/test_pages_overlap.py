"""cache_fork and cache_compact refuse pools whose pages overlap, one another, an array of the call or its workspace, before anything is
enqueued, and take every other layout: against the pages' bytes, counted one by one.  (No GPU: a call that is not refused fails at
its launch.)"""
import ctypes
import random

import pytest

import paper_2607_09153_gb300 as kp
from paper_2607_09153_gb300 import operators as ops
from tests.test_pages import _arrays, _compact, _fork


@pytest.fixture(autouse=True)
def no_gpu():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")


def _refused(rc):
    return rc == kp.KVPRM_EINVAL and "overlap" in ops.lib().kvprm_operator_error().decode()


def _pages(pool, n):
    return [(pool.base + layer * pool.layer_stride + p * pool.page_stride, pool.page_bytes) for layer in range(pool.layers) for p in range(n)
            if pool.page_bytes]


def _meet(spans):
    spans = sorted(spans)
    return any(a + n > b for (a, n), (b, _) in zip(spans, spans[1:]))


BASE = 1 << 44


@pytest.mark.parametrize("call", [_fork, _compact])
@pytest.mark.parametrize("seed", range(300))
def test_pools(call, seed):
    """One to three pools with strides of any sign, in any nesting, beside and between each other, of one page and one layer too.
    Pools between each other's pages are taken where these are as far apart; the others may be refused."""
    rng = random.Random(seed)
    x, n = _arrays(), rng.choice([1, 2, 5, 16])
    stride = 16 * rng.choice([1, 2, 3, 7, 40, 64]) * rng.choice([1, 1, -1])
    pools = []
    for _ in range(rng.randint(1, 3)):
        pools.append(ops.KvprmPool(base=BASE + 16 * rng.randint(0, 300), layer_stride=16 * rng.randint(-200, 200) * rng.choice([0, 1, 1, 1]),
                                   page_stride=stride if rng.random() < 0.9 else 16 * rng.randint(0, 9), page_bytes=16 * rng.choice([0, 1, 1, 2, 3]),
                                   layers=rng.choice([0, 1, 1, 2, 3, 6])))
    rc = call(x, pools, n_pages=n)
    meet = _meet([s for p in pools for s in _pages(p, n)])
    if meet:
        assert _refused(rc)
    elif len({p.page_stride for p in pools if p.layers and p.page_bytes}) <= 1 or n == 1:
        assert not _refused(rc) and rc == kp.KVPRM_ECUDA


@pytest.mark.parametrize("call", [_fork, _compact])
def test_layouts_that_are_fine(call):
    """Layers apart, layers within pages, keys and values of one tensor, and more pools than a launch takes at once."""
    x, page = _arrays(), 4096
    pool = lambda **kw: ops.KvprmPool(**{**dict(base=BASE, layer_stride=16 * page, page_stride=page, page_bytes=page, layers=28), **kw})  # noqa: E731
    for pools in ([pool()], [pool(layer_stride=page, page_stride=28 * page)],
                  [pool(page_bytes=page // 2), pool(base=BASE + page // 2, page_bytes=page // 2)],
                  [pool(base=BASE + 16 * page * i, layers=1, layer_stride=0) for i in range(96)],
                  [pool(layer_stride=20 * page), pool(base=BASE + 16 * page, layer_stride=20 * page, page_stride=page // 4, page_bytes=page // 4)],
                  [pool(layers=14, layer_stride=32 * page), pool(base=BASE + 16 * page, layers=14, layer_stride=32 * page)],
                  [pool(page_bytes=48), pool(base=BASE + 48, layers=14, layer_stride=32 * page, page_bytes=16), pool(base=BASE + 64, layers=1, page_bytes=64)],
                  [pool(layers=1 << 20, page_bytes=0)], [pool(layers=0, page_stride=0)]):
        rc = call(x, pools)
        assert rc == kp.KVPRM_ECUDA, ops.lib().kvprm_operator_error().decode()


@pytest.mark.parametrize("call", [_fork, _compact])
def test_overlaps(call):
    x, page = _arrays(), 4096
    pool = lambda **kw: ops.KvprmPool(**{**dict(base=BASE, layer_stride=16 * page, page_stride=page, page_bytes=page, layers=28), **kw})  # noqa: E731
    for pools in ([pool(page_stride=0)], [pool(layer_stride=0)], [pool(page_bytes=page + 16)], [pool(page_stride=-page, layer_stride=15 * page)],
                  [pool(), pool()], [pool(), pool(base=BASE + 28 * 16 * page - 16, layers=1)],
                  [pool(base=BASE + 16 * page * i, layers=1, layer_stride=0) for i in range(95)] + [pool(base=BASE + page * 64 + 16, layers=1, page_bytes=16)],
                  [pool(layers=1 << 30, layer_stride=48, page_stride=64, page_bytes=16)]):
        assert _refused(call(x, pools))
    for name in ("refs", "lens", "refs_out", "table_out", "counts"):
        base = ctypes.addressof(x[name]) // 16 * 16
        assert _refused(call(x, [pool(base=base, layers=1, page_bytes=16, page_stride=4096)])), name
        assert _refused(call(x, [pool(), pool(base=base - 28 * 15 * 16 * 64, layer_stride=1024 * 15, page_stride=1024, page_bytes=512, layers=29)])), name
    # the workspace is 2^20 bytes from 256 on, of which the call needs a few KB
    assert _refused(call(x, [pool(base=1024, layers=1, page_bytes=16)]))
    assert not _refused(call(x, [pool(base=1 << 16, layers=1, page_bytes=16)]))
    assert _refused(call(x, refs=512)) and _refused(call(x, counts=1024))
