"""Prompts written in 4 bits, long enough that a thread takes several tokens: every code and exponent bit by bit, against the definition
in 64 bits over whole tensors."""
import math

import pytest

from tests import cache4_util as ref4
from tests.test_gpu_cache4 import _adverse_rows, _pool4
from tests.test_gpu_operators import DTYPES, _gen, _kp

pytestmark = pytest.mark.gpu


def _quantised(torch, x):
    """(codes, exponent bytes) of rows [...][head_dim]: infinities are the largest code of the rest's scale, a block with a NaN has the
    exponent 255."""
    y = x.double().unflatten(-1, (-1, 32))
    nan, finite = y.isnan().any(-1), y.isfinite()
    most = torch.where(finite, y, 0.0).abs().amax(-1)
    m, e = torch.frexp(most)                                  # most = m 2^e with m in [1/2, 1), and 6 = 3/4 2^3
    e = torch.where(most == 0, -127, torch.where(m > 0.75, e - 2, e - 3).clamp(min=-127))
    codes = ref4.codes_of(torch.where(y.isnan(), 0.0, y) * torch.exp2(-e.double())[..., None])
    return ref4.pack(codes.flatten(-2)), torch.where(nan, 255, e + 127).to(torch.uint8), nan


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("hd,nkv,odd", [(64, 5, 1), (64, 4, 0), (128, 3, 1), (128, 40, 1), (64, 1, 3)])
def test_long_prompts(dtype, offset, hd, nkv, odd):
    torch, kp = _kp()
    dt, gen = getattr(torch, dtype), _gen(torch, hd + nkv)
    pieces = 2 * nkv * hd // (16 if dtype == "bfloat16" and offset == 0 else 8)
    n = -(-8 * 256 * torch.cuda.get_device_properties(0).multi_processor_count // pieces)   # two tokens a thread from here on
    n += 1 - n % 2 + (1 - odd if odd < 2 else odd - 1)                                      # odd or even
    assert n % 2 == (odd > 0)
    rows = torch.randn((n, 2 * nkv * hd + 8), generator=gen, device="cuda")
    rows *= torch.exp2(torch.randint(-12, 12, (n, 1), generator=gen, device="cuda").float())
    adverse = _adverse_rows(torch, 64, hd, gen)
    x = rows[:, offset:offset + 2 * nkv * hd].view(n, 2 * nkv, hd)
    half = (n + 1) // 2                                       # token t and t + half are a thread's
    for t in (0, half - 1, half, n - 1, 100, half + 101):
        x[t] = adverse[t % 7:t % 7 + 2 * nkv] if 2 * nkv <= 57 else adverse.repeat(2, 1)[:2 * nkv]
    if dtype == "float16":
        rows.clamp_(-65504, 65504)
    for t, i, value in ((7, 3, math.nan), (half + 9, 40, math.nan), (11, 0, math.inf), (half + 12, hd - 1, -math.inf)):
        x[t, t % (2 * nkv), i] = value
    x[13, 0, 32:], x[half + 13, 1, :32] = math.inf, -math.inf
    rows = rows.to(dt)
    x = rows[:, offset:offset + 2 * nkv * hd].view(n, 2 * nkv, hd)
    pages = (n + 15) // 16 + 2
    slots = torch.randperm(pages * 16, generator=torch.Generator().manual_seed(n))[:n].cuda()
    slots[::13], slots[5], slots[half + 5], slots[half + 6] = -1, pages * 16, -(1 << 40), 1 << 40
    pool, exps = _pool4(torch, pages, nkv, hd, fill=0x35)
    kp.cache_write(pool, slots, x[:, :nkv], x[:, nkv:], exponents=exps)
    want_c, want_e = _pool4(torch, pages, nkv, hd, fill=0x35)
    fine = (slots >= 0) & (slots < pages * 16)
    page, place = slots[fine] // 16, slots[fine] % 16
    c, e, nan = (y.unflatten(1, (2, nkv)) for y in _quantised(torch, x[fine]))
    want_c[page, :, :, place], want_e[page, :, :, place] = c, e
    assert torch.equal(exps, want_e)
    lost = (want_e == 255)[..., None]                         # (whose codes may be any)
    assert bool(nan.any()) and torch.equal(pool.unflatten(-1, (-1, 16)).masked_fill(lost, 0), want_c.unflatten(-1, (-1, 16)).masked_fill(lost, 0))
