"""The NaN codes of 8-bit pages (0x7F and 0xFF) under an ordinary exponent, as pages that were quantised elsewhere may hold
them: every reader takes them as NaN, whatever the number of query rows, and they reach what the definition says alone."""
import math

import pytest

from tests.gpu_util import require_gpu
from tests.test_gpu_operators import Tree, _pool

pytestmark = pytest.mark.gpu


def _plant(t, seq, token, kv, head, dim, code):
    page = int(t.table[seq, token // 16])
    t.pages.view(t.torch.uint8)[page, kv, head, token % 16, dim] = code
    t.values[page, kv, head, token % 16, dim] = math.nan


def _check(t, out):
    o, bound = t.want()
    lost = o.isnan()
    assert t.torch.equal(out.isnan(), lost)
    off = (out.double() - o).abs()[~lost]
    assert bool((off <= bound[~lost]).all()) and 0 < int(lost.sum()) < lost.numel()


# query rows of a kv head: 16 and 32 at most on warp-level instructions, more on the tensor cores (one tile, two, three)
@pytest.mark.parametrize("drafts", [1, 4, 8, 9, 32, 33, 65])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("code", [0x7F, 0xFF])
def test_attention(code, hd, drafts):
    """In values: one dimension of every row that reads the head.  In keys: all of them."""
    torch = require_gpu()
    lens = [40, 333, 0, 1300]
    t = Tree(torch, 8, 2, hd, lens, [drafts] * 4, True, seed=drafts)
    for i, (seq, token) in enumerate(((0, 0), (0, 39), (1, 200), (3, 1299), (3, 640))):
        _plant(t, seq, token, 1, i % 2, (7 + 29 * i) % hd, code)
    out = t.run()
    _check(t, out)
    _plant(t, 1, 332, 0, 1, hd - 1, code)
    _plant(t, 3, 127, 0, 0, 2, code)
    out = t.run()
    _check(t, out)
    assert bool(out[t.start[1]:t.start[2], 4:].isnan().all()) and bool(out[t.start[3]:, :4].isnan().all())


def test_wide_powers():
    """Beside rows whose power of two needs two factors, and in a cache long enough to be shared by several CTAs."""
    torch = require_gpu()
    for drafts in (3, 8, 20):
        t = Tree(torch, 4, 1, 128, [5000], [drafts], True, seed=5)
        t.exps[:, 1, :, ::3] = 140
        t.values = t.pages.double() * torch.exp2(t.exps.double() - 127)[..., None]
        for i, token in enumerate((0, 17, 2500, 4999)):
            _plant(t, 0, token, 1, 0, 5 + 31 * i, 0x7F)
        _check(t, t.run())


def test_expand():
    torch = require_gpu()
    import paper_2607_09153_gb300 as kp
    pool, exps = _pool(torch, 2, 1, 64, True, fill=56)
    codes = pool.view(torch.uint8)
    codes[1, 0, 0, 3, 9], codes[1, 1, 0, 15, 63] = 0x7F, 0xFF
    out = torch.zeros((2, 2, 1, 16, 64), dtype=torch.bfloat16, device="cuda")
    kp.cache_expand(pool, exps, torch.arange(2, dtype=torch.int32, device="cuda"), out)
    want = torch.zeros_like(out, dtype=torch.bool)
    want[1, 0, 0, 3, 9] = want[1, 1, 0, 15, 63] = True
    assert torch.equal(out.isnan(), want)
