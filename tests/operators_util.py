"""The operators' definitions in 64 bits (plain torch, one sequence and head at a time), for the tests."""
import math

import torch

PAGE = 16


def frequencies(rd, base=1e4, scaling="none", factor=1.0, original_len=0, low=1.0, high=32.0):
    """Angle per position of each pair."""
    if scaling == "base":
        base = base * factor ** (rd / (rd - 2))
    out = []
    for i in range(rd // 2):
        f = base ** (-2 * i / rd)
        n = original_len * f / (2 * math.pi)
        if scaling == "linear":
            f = f / factor
        elif scaling == "smooth":
            w = min(1.0, max(0.0, (n - low) / (high - low)))
            f = w * f + (1 - w) * f / factor
        elif scaling == "ramp":
            pair = [rd * math.log(original_len / (2 * math.pi * t)) / (2 * math.log(base)) for t in (high, low)]
            a, b = max(0, math.floor(pair[0])), min(rd - 1, math.ceil(pair[1]))
            w = 1 - min(1.0, max(0.0, (i - a) / max(b - a, 1e-3)))
            f = w * f + (1 - w) * f / factor
        out.append(f)
    return torch.tensor(out, dtype=torch.float64)


def rotate(x, positions, freq, interleaved=False, magnitude=1.0, inverse=False):
    """x [tokens][heads][head_dim] in 64 bits."""
    x = x.double()
    rd = 2 * len(freq)
    angle = positions.double()[:, None, None] * freq.to(x.device)
    cos, sin = magnitude * angle.cos(), magnitude * angle.sin() * (-1 if inverse else 1)
    first = torch.arange(rd // 2, device=x.device) * 2 if interleaved else torch.arange(rd // 2, device=x.device)
    second = first + (1 if interleaved else rd // 2)
    out = x.clone()
    out[..., first] = x[..., first] * cos - x[..., second] * sin
    out[..., second] = x[..., second] * cos + x[..., first] * sin
    return out


# every e4m3 value by its code
def e4m3_values():
    out = []
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        v = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        if e == 15 and m == 7:
            v = math.nan
        out.append(-v if code & 128 else v)
    return torch.tensor(out, dtype=torch.float64)


def row_exponent(most):
    """The least e >= -127 with most <= 448 2^e (most a Python float)."""
    if most == 0:
        return -127
    e = math.frexp(most)[1] - 9
    if most > 448 * 2.0 ** e:
        e += 1
    return max(e, -127)


def quantise(row):
    """(codes, exponent byte) of one row of finite 64-bit values, to nearest, ties to the even code."""
    e = row_exponent(float(row.abs().max()))
    y = row * 2.0 ** -e
    grid = e4m3_values()[:127]   # 0 .. 448
    at = torch.searchsorted(grid, y.abs().cpu().contiguous())
    hi = at.clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - y.abs().cpu(), y.abs().cpu() - grid[lo]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code + 128 * torch.signbit(y).cpu().long()).to(torch.uint8), e + 127


def attention(q, k, v, rows, lens, start, mask, scale):
    """rows[s] = (keys, values) [cached][n_kv][head_dim] of sequence s in 64 bits; mask: bool [tokens][longest].
    Returns (o, a, peak): outputs, sum_j w_j |v_j| and the largest sum_d |q_d k_jd| * scale, for error bounds."""
    n_kv, group = k.shape[1], q.shape[1] // k.shape[1]
    o = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    a, peak = torch.zeros_like(o), torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    for s, n in enumerate(lens):
        s0, s1 = start[s], start[s + 1]
        for h in range(q.shape[1]):
            g = h // group
            keys = torch.cat([rows[s][0][:, g], k[s0:s1, g].double()])
            vals = torch.cat([rows[s][1][:, g], v[s0:s1, g].double()])
            keep = torch.cat([torch.ones((s1 - s0, n), dtype=torch.bool, device=q.device), mask[s0:s1, :s1 - s0]], 1)
            for t in range(s1 - s0):
                at = keep[t].nonzero()[:, 0]
                if len(at) == 0:
                    continue
                x = q[s0 + t, h].double()
                w = torch.softmax(keys[at] @ x * scale, 0)
                o[s0 + t, h] = w @ vals[at]
                a[s0 + t, h] = w @ vals[at].abs()
                peak[s0 + t, h] = (keys[at].abs() @ x.abs()).max() * abs(scale)
    return o, a, peak


def attention_bound(o, a, peak, most_keys, head_dim):
    """How far a bf16 output may be: each weight is rounded to bf16 (2^-8 of it at most: 8 significant bits); a score is a sum of head_dim
    products in fp32 (whatever the order: head_dim units of 2^-23 of the sum of magnitudes), which moves weights by as
    much in both numerator and denominator, and exp2 adds 2^-21; the sums over the keys are fp32 additions, at least
    16 of them at a time; the output is rounded to bf16."""
    weights = 2.0 ** -8 + 2 * head_dim * 2.0 ** -23 * peak[..., None] + 2.0 ** -20 + (most_keys / 8 + 64) * 2.0 ** -23
    return weights * a + 2.0 ** -8 * o.abs() + 1e-30


def unpack_mask(mask, longest):
    j = torch.arange(longest, device=mask.device)
    return ((mask[:, j // 32] >> (j % 32)) & 1).bool()
