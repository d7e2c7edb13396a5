"""The rotary angles against frequencies in 60 digits: the table, and (on the GPU) the largest positions.

A frequency f over 2 pi is computed in 64-bit floating point: half a unit of its exponent moves it by |ln f| 2^-53 of itself,
the power, 2 pi and the division by some four units more.  f |ln f| and f are at most 0.37 and 1, so the turns are off by
at most (0.37 + 4) / 2 pi 2^-53 < 2^-53 (measured: 2^-55).
"""
from decimal import Decimal, getcontext
from fractions import Fraction

import pytest

import paper_2607_09153_gb300 as kp
from tests.gpu_util import require_gpu

getcontext().prec = 60
TABLE = Fraction(1, 2 ** 53)   # turns


def _atan_inv(n):
    term, total, k = Decimal(1) / n, Decimal(0), 1
    while abs(term) > Decimal(10) ** -65:
        total += term / k if k % 4 == 1 else -term / k
        term /= n * n
        k += 2
    return total


TWO_PI = 8 * (4 * _atan_inv(5) - _atan_inv(239))


def _turns(rd, base, scaling="none", factor=1.0):
    """Turns per position of each pair."""
    base, factor = Decimal(base), Decimal(factor)
    if scaling == "base":
        base *= factor ** (Decimal(rd) / (rd - 2))
    out = [base ** (Decimal(-2 * i) / rd) / TWO_PI for i in range(rd // 2)]
    return [Fraction(x / factor if scaling == "linear" else x) for x in out]


CASES = [(128, 1e4, "none", 1.0), (64, 5e5, "none", 1.0), (256, 1e6, "none", 1.0), (98, 1e4, "linear", 7.5),
         (128, 1e4, "base", 4.0), (2, 1e4, "none", 1.0)]


@pytest.mark.parametrize("rd,base,scaling,factor", CASES)
def test_table(rd, base, scaling, factor):
    got = kp.Rope(rd, base=base, scaling=scaling, factor=factor).turns()
    for g, w in zip(got, _turns(rd, base, scaling, factor)):
        assert abs(Fraction(g, 2 ** 64) - w) <= TABLE


@pytest.mark.gpu
@pytest.mark.parametrize("rd,base,scaling,factor", CASES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_largest_positions(rd, base, scaling, factor, interleaved):
    """An angle is off by the table's error times the position, 2^-32 turns of the upper half that is kept and 2^-26 of its
    rounding to 24 bits; sine and cosine, two products and a sum as in test_gpu_operators.py."""
    import math
    torch = require_gpu()
    rope = kp.Rope(rd, base=base, interleaved=interleaved, scaling=scaling, factor=factor)
    pos = [2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, 1 << 17, (1 << 24) + 1, 99991, 1, 0]
    x = torch.randn((len(pos), 2, rd), generator=torch.Generator(device="cuda").manual_seed(rd), device="cuda")
    y = rope.rotate(torch.tensor(pos, dtype=torch.int32, device="cuda"), x)[0].double().cpu()
    x, turns = x.double().cpu(), _turns(rd, base, scaling, factor)
    first, second = (slice(0, rd, 2), slice(1, rd, 2)) if interleaved else (slice(0, rd // 2), slice(rd // 2, rd))
    for i, p in enumerate(pos):
        angle = torch.tensor([2 * math.pi * float((p * t) % 1) for t in turns], dtype=torch.float64)
        a, b = x[i][:, first], x[i][:, second]
        size = (a * a + b * b).sqrt()
        off = 2 * math.pi * (abs(p) * 2.0 ** -53 + 2.0 ** -32 + 2.0 ** -26) + 6e-7
        assert bool(((y[i][:, first] - (a * angle.cos() - b * angle.sin())).abs() <= off * size + 1e-9).all()), p
        assert bool(((y[i][:, second] - (b * angle.cos() + a * angle.sin())).abs() <= off * size + 1e-9).all()), p
