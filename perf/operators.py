"""The operators around the scored cache whose time counts: rotary positions, the quantised cache (its write and its
expansion into scoring pages) and the attention of a tree of drafted tokens over it.

A case is a dict of plain values.  `op` and what goes with it:
  "rope", "rope_back"  tokens, nq, nkv, hd    q [tokens][nq][hd] and k [tokens][nkv][hd], or their gradients
                       rd                     elements of a head that are rotated (the rest passes)
                       interleaved            pairs (2i, 2i + 1) instead of (i, i + rd / 2)
                       scaling, factor        how the frequencies are stretched for long contexts
                       dtype, fused           fused: q and k are columns of one projection's rows
                       top                    positions below this one
  "write"              tokens, nkv, hd, dtype, fused, format, rotate (keys rotated on the way), top
  "expand"             n pages of a pool of `pool`, nkv, hd: e4m3 pages into bf16 scoring pages
  "attend"             n sequences of up to `drafts` drafted tokens each, nq, nkv, hd, format
                       cache                  "equal": len cached tokens each; "ragged": len / 16 .. len, one of them 0
  shape_seed           draws the ragged lengths (the sizes belong to the case, the values to the seed)
"""
import math
import random

import torch

own = False

PAGE = 16
BASE = 1e4
ORIGINAL = 32768          # the context that stretched frequencies were trained on
LOW, HIGH = 1.0, 32.0     # turns within it: frequencies below LOW are stretched, above HIGH kept

SHAPES = {   # heads of the repository's scorers
    "tiny": dict(nq=4, nkv=2, hd=64),
    "small64": dict(nq=16, nkv=4, hd=64),
    "1p5b": dict(nq=12, nkv=2, hd=128),
    "7b": dict(nq=28, nkv=4, hd=128),
    "8b": dict(nq=32, nkv=8, hd=128),
}
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _rope(name, op, shape, tokens, rd, dtype="bf16", interleaved=False, scaling="none", factor=1.0, fused=True,
          top=32768):
    return dict(name=name, op=op, tokens=tokens, rd=rd, dtype=dtype, interleaved=interleaved, scaling=scaling,
                factor=factor, fused=fused, top=top, **SHAPES[shape])


def _write(name, shape, tokens, format="e4m3", dtype="bf16", rotate=True, fused=True, top=32768):
    return dict(name=name, op="write", tokens=tokens, format=format, dtype=dtype, rotate=rotate, fused=fused, top=top,
                **SHAPES[shape])


def _expand(name, shape, n, pool):
    return dict(name=name, op="expand", n=n, pool=pool, **SHAPES[shape])


def _attend(name, shape, n, drafts, cache, len_, format, shape_seed=1):
    return dict(name=name, op="attend", n=n, drafts=drafts, cache=cache, len=len_, format=format,
                shape_seed=shape_seed, **SHAPES[shape])


def listed():
    return [
        # one decoding step of 16 sampled answers: latency only
        _rope("rope_step_7b", "rope", "7b", 16, 128),
        # trajectories re-encoded from text, contexts stretched fourfold: q and k in the projection's rows
        _rope("rope_long_8b", "rope", "8b", 32768, 128, scaling="smooth", factor=4.0, top=131072),
        # training the scorer: gradients in 32 bits, half of each narrow head rotated, neighbours paired
        _rope("rope_back_fp32", "rope_back", "small64", 9001, 32, dtype="fp32", interleaved=True, fused=False),
        # one decoding step of a 64-wide beam: rotated, quantised and put into the pages in one go
        _write("write_step_7b", "7b", 64),
        # whole trajectories put into the cache
        _write("write_prompt_8b", "8b", 30001),
        # a few pages of one candidate made readable to the scorer
        _expand("expand_few_small", "small64", 24, 40),
        # a batch's pages made readable to the scorer
        _expand("expand_batch_8b", "8b", 4099, 4200),
        # the smallest step: four short sequences, one token each
        _attend("attend_tiny", "tiny", 4, 1, "equal", 128, "bf16"),
        # plain decoding of many uneven sequences over the quantised cache
        _attend("attend_decode_7b", "7b", 64, 1, "ragged", 9001, "e4m3"),
        # a small tree of drafts behind few, long contexts
        _attend("attend_long_8b", "8b", 8, 8, "equal", 32768, "bf16"),
        # best-of-16 with a middling tree each, uneven contexts
        _attend("attend_tree_1p5b", "1p5b", 16, 21, "ragged", 4096, "bf16"),
        # wide trees (every row of the tensor cores' tiles in use) over the quantised cache
        _attend("attend_wide_7b", "7b", 16, 64, "ragged", 16384, "e4m3"),
    ]


def draw(rng):
    def logint(lo, hi):
        return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    while True:
        op = rng.choice(["rope", "rope_back", "write", "expand", "attend", "attend", "attend"])
        shape = rng.choice(["tiny", "small64", "1p5b", "7b", "8b"])
        hd, nkv, nq = SHAPES[shape]["hd"], SHAPES[shape]["nkv"], SHAPES[shape]["nq"]
        if op in ("rope", "rope_back"):
            scaling = rng.choice(["none", "linear", "base", "ramp", "smooth"])
            c = _rope("", op, shape, logint(1, 32768), rng.choice([hd, hd, hd // 2, hd // 4]),
                      rng.choice(["bf16", "fp16", "fp32"]), rng.random() < 0.5, scaling,
                      1.0 if scaling == "none" else rng.choice([2.0, 4.0, 7.5]), rng.random() < 0.5,
                      rng.choice([4096, 32768, 131072]))
        elif op == "write":
            c = _write("", shape, logint(1, 32768), rng.choice(["e4m3", "e4m3", "bf16"]),
                       rng.choice(["bf16", "fp16", "fp32"]), rng.random() < 0.5, rng.random() < 0.5)
        elif op == "expand":
            n = logint(1, 4096)
            c = _expand("", shape, n, n + logint(1, 64))
        else:
            c = _attend("", shape, logint(1, 64), logint(1, 64), rng.choice(["equal", "ragged"]), logint(1, 65536),
                        rng.choice(["bf16", "e4m3"]), rng.randrange(1 << 30))
            cached, longest = sum(_lens(c)), max(_lens(c))
            # no dearer than the largest listed case, and what the plain form holds in 32 bits fits a few GB
            if cached * c["drafts"] * nq > 16 * 64 * 28 * 9000 or cached > 1 << 18:
                continue
            if c["n"] * longest * nkv * hd > 1 << 29 or c["n"] * c["drafts"] * nq * longest > 1 << 30:
                continue
        del c["name"]
        return c


# ---------------------------------------------------------------- sizes
def _lens(c):
    rng = random.Random(c["shape_seed"])
    if c["cache"] == "equal":
        return [c["len"]] * c["n"]
    lens = [rng.randint(max(1, c["len"] // 16), c["len"]) for _ in range(c["n"])]
    if c["n"] > 2:
        lens[c["n"] // 2] = 0   # a sequence that has not started
    return lens


def _drafts(c):
    """Drafted tokens of each sequence: as many as asked for, or in a ragged batch at least half of them."""
    rng = random.Random(c["shape_seed"] + 1)
    if c["cache"] == "equal":
        return [c["drafts"]] * c["n"]
    return [c["drafts"]] + [rng.randint((c["drafts"] + 1) // 2, c["drafts"]) for _ in range(c["n"] - 1)]


def work(case):
    c = case
    hd, nq, nkv = c["hd"], c["nq"], c["nkv"]
    if c["op"] in ("rope", "rope_back"):
        size = DTYPES[c["dtype"]].itemsize
        moved = c["tokens"] * (nq + nkv) * hd
        return {"bytes": 2 * size * moved + 4 * c["tokens"], "flops": 3 * c["tokens"] * (nq + nkv) * c["rd"]}
    if c["op"] == "write":
        size = DTYPES[c["dtype"]].itemsize
        rows = 2 * c["tokens"] * nkv
        out = rows * hd + rows if c["format"] == "e4m3" else 2 * rows * hd
        return {"bytes": size * rows * hd + out + (12 if c["rotate"] else 8) * c["tokens"], "flops": 4 * rows * hd}
    if c["op"] == "expand":
        rows = 2 * c["n"] * nkv * PAGE
        return {"bytes": 3 * rows * hd + rows + 16 * c["n"], "flops": rows * hd}
    lens, drafts = _lens(c), _drafts(c)
    n = sum(drafts)
    row = 2 * nkv * ((hd + 1) if c["format"] == "e4m3" else 2 * hd)
    pages = sum((x + PAGE - 1) // PAGE for x in lens)
    total = row * sum(lens) + 2 * n * hd * (2 * nq + 2 * nkv) + 4 * n * ((c["drafts"] + 31) // 32)
    pairs = sum(t * (x + (t + 1) / 2) for t, x in zip(drafts, lens))
    return {"bytes": total + 4 * (pages + 2 * c["n"] + 1), "flops": 4 * hd * nq * pairs}


# ---------------------------------------------------------------- inputs
def _frequencies(c):
    """Angle per position of each pair, in 64 bits."""
    rd, factor = c["rd"], c.get("factor", 1.0)
    scaling, base = c.get("scaling", "none"), BASE
    if scaling == "base":
        base *= factor ** (rd / (rd - 2))
    freq = []
    # the pairs that turn HIGH and LOW times within the original context
    at = lambda turns: rd * math.log(ORIGINAL / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(0, math.floor(at(HIGH))), min(rd - 1, math.ceil(at(LOW)))
    for i in range(rd // 2):
        f = base ** (-2.0 * i / rd)
        if scaling == "linear":
            f /= factor
        elif scaling == "ramp":
            stretched = min(1.0, max(0.0, (i - lo) / max(hi - lo, 1e-3)))
            f = f * (1 - stretched) + f / factor * stretched
        elif scaling == "smooth":
            kept = min(1.0, max(0.0, (ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW)))
            f = f * kept + f / factor * (1 - kept)
        freq.append(f)
    return freq


def _turns(freq):
    """The frequencies in 2^-64 turns: a position's angle is then exact in wrapping whole numbers."""
    whole = [round(f / (2 * math.pi) * 2 ** 64) % 2 ** 64 for f in freq]
    return torch.tensor([w - 2 ** 64 if w >= 2 ** 63 else w for w in whole], dtype=torch.int64, device="cuda")


def _normal(shape, std, gen, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _heads(n, heads, hd, std, fused, gen, dtype):
    """One tensor [n][h][hd] for each of `heads`, dense or columns of shared rows."""
    if not fused:
        return [_normal((n, h, hd), s, gen, dtype) for h, s in zip(heads, std)]
    rows = _normal((n, sum(heads), hd), 1.0, gen, dtype)
    out, at = [], 0
    for h, s in zip(heads, std):
        out.append(rows[:, at:at + h])
        out[-1].mul_(s)
        at += h
    return out


def _pool(pages, nkv, hd, format, gen):
    """A used pool: pages [pages][2][nkv][16][hd], and for e4m3 a power of two for each row [pages][2][nkv][16]."""
    shape = (pages, 2, nkv, PAGE, hd)
    if format == "bf16":
        return _normal(shape, 1.0, gen, torch.bfloat16), None
    # codes as quantised N(0, 1) rows have them: the largest of a row between 224 and 448
    codes = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
    step = max(1, (1 << 26) // (2 * nkv * PAGE * hd))
    for a in range(0, pages, step):
        codes[a:a + step] = _normal((min(step, pages - a),) + shape[1:], 100.0, gen, torch.float32).clamp_(
            -448.0, 448.0).to(torch.float8_e4m3fn)
    exponents = torch.randint(127 - 8, 127 - 5, shape[:-1], dtype=torch.uint8, device="cuda", generator=gen)
    return codes, exponents.view(torch.float8_e8m0fnu)


def _tree_masks(drafts, words, cpu):
    """Ancestors (itself among them) of each drafted token, as bits: token t's parent is one of the tokens before it
    in its sequence, or the end of the cache."""
    total, most = sum(drafts), max(drafts)
    parent = torch.rand((len(drafts), most), generator=cpu)
    bits = torch.zeros((len(drafts), most, words * 32), dtype=torch.bool)
    rows = torch.arange(len(drafts))
    for t in range(most):
        p = (parent[:, t] * (t + 1)).long() - 1
        if t:
            bits[:, t] = bits[rows, p.clamp(min=0)] & (p >= 0)[:, None]
        bits[:, t, t] = True
    weight = torch.tensor([1 << j for j in range(32)], dtype=torch.int64)
    packed = (bits.view(len(drafts), most, words, 32).long() * weight).sum(-1)
    packed = torch.where(packed >= 1 << 31, packed - (1 << 32), packed).int()
    return torch.cat([packed[b, :t] for b, t in enumerate(drafts)]).reshape(total, words).cuda()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cpu = torch.Generator().manual_seed(seed)
    hd, nq, nkv = c["hd"], c["nq"], c["nkv"]
    x = dict(c)
    if c["op"] in ("rope", "rope_back") or c.get("rotate"):
        n = c["tokens"]
        x.setdefault("rd", hd)
        x.setdefault("interleaved", False)
        freq = _frequencies(x)
        x["turns"] = _turns(freq)
        # a prompt's positions run on from a start of their own, a step's are anywhere
        first = torch.randint(0, max(1, c["top"] - n), (n if n < 256 else 1,), generator=cpu, dtype=torch.int32)
        x["positions"] = (first if n < 256 else first + torch.arange(n, dtype=torch.int32)).cuda()
        if own:
            import paper_2607_09153_gb300 as kp
            x["rope"] = kp.Rope(x["rd"], base=BASE, interleaved=x["interleaved"], scaling=x.get("scaling", "none"),
                                factor=x.get("factor", 1.0), original_len=ORIGINAL, low=LOW, high=HIGH)
    if c["op"] in ("rope", "rope_back"):
        x["q"], x["k"] = _heads(c["tokens"], (nq, nkv), hd, (1.0, 1.0), c["fused"], gen, DTYPES[c["dtype"]])
    elif c["op"] == "write":
        n = c["tokens"]
        x["k"], x["v"] = _heads(n, (nkv, nkv), hd, (2.0, 0.5), c["fused"], gen, DTYPES[c["dtype"]])
        step = n < 256
        pages = (n if step else (n + PAGE - 1) // PAGE) + 3
        x["pages"], x["exponents"] = _pool(pages, nkv, hd, c["format"], gen)
        order = torch.randperm(pages, generator=cpu)
        if step:   # a slot somewhere in a page of its own for each sequence
            slots = order[:n] * PAGE + torch.randint(0, PAGE, (n,), generator=cpu)
        else:      # prompts: page after page, in no particular order of pages
            slots = order[torch.arange(n) // PAGE] * PAGE + torch.arange(n) % PAGE
        slots[torch.rand(n, generator=cpu) < 0.02] = -1   # padding of the batch: not written
        x["slots"] = slots.cuda()
    elif c["op"] == "expand":
        x["pages"], x["exponents"] = _pool(c["pool"], nkv, hd, "e4m3", gen)
        x["src"] = torch.randperm(c["pool"], generator=cpu)[:c["n"]].int().cuda()
        x["dst"] = torch.randperm(c["n"] + 1, generator=cpu)[:c["n"]].int().cuda()
        x["out"] = torch.zeros((c["n"] + 1, 2, nkv, PAGE, hd), dtype=torch.bfloat16, device="cuda")
    else:
        lens, drafts = _lens(c), _drafts(c)
        blocks = [(n + PAGE - 1) // PAGE for n in lens]
        total = sum(blocks) + 3
        x["pages"], x["exponents"] = _pool(total, nkv, hd, c["format"], gen)
        order = torch.randperm(total, generator=cpu).int()
        table, at = torch.zeros((c["n"], max(1, max(blocks))), dtype=torch.int32), 0
        for b, k in enumerate(blocks):
            table[b, :k] = order[at:at + k]
            at += k
        start = torch.tensor([0] + drafts).cumsum(0).int()
        # scores q.k / sqrt(hd) with a spread of about two, as a trained model's
        x["q"], x["k"], x["v"] = _heads(int(start[-1]), (nq, nkv, nkv), hd, (2.0, 1.0, 1.0), True, gen, torch.bfloat16)
        x.update(table=table.cuda(), lens=torch.tensor(lens, dtype=torch.int32).cuda(), start=start.cuda(),
                 mask=_tree_masks(drafts, (c["drafts"] + 31) // 32, cpu), longest=max(lens))
    return x


# ---------------------------------------------------------------- one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(x):
    import paper_2607_09153_gb300 as kp
    if x["op"] == "rope":
        return list(x["rope"].rotate(x["positions"], x["q"], x["k"]))
    if x["op"] == "rope_back":
        return list(x["rope"].rotate_backward(x["positions"], x["q"], x["k"]))
    if x["op"] == "write":
        kp.cache_write(x["pages"], x["slots"], x["k"], x["v"], exponents=x["exponents"], rope=x.get("rope"),
                       positions=x.get("positions"))
        return {"pages": x["pages"], "exponents": x["exponents"]}
    if x["op"] == "expand":
        return kp.cache_expand(x["pages"], x["exponents"], x["src"], x["out"], x["dst"])
    return kp.tree_attention(x["q"], x["k"], x["v"], x["pages"], x["table"], x["lens"], x["start"],
                             max_drafts=x["drafts"], max_len=x["longest"], exponents=x["exponents"], mask=x["mask"])


def _rotated(x, y, back=False):
    """y [tokens][heads][hd] in 32 bits, rotated by its tokens' angles (back: by their negatives)."""
    turn = (x["positions"].long()[:, None] * x["turns"]) >> 32
    angle = (turn.float() * (math.pi / 2 ** 31))[:, None, :]
    cos, sin = angle.cos(), angle.sin() * (-1.0 if back else 1.0)
    rd, y = x["rd"], y.float()
    a, b = (y[..., 0:rd:2], y[..., 1:rd:2]) if x["interleaved"] else (y[..., :rd // 2], y[..., rd // 2:rd])
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([a, b], -1).flatten(-2) if x["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([r, y[..., rd:]], -1)


def _quantised(y):
    """e4m3 codes and the exponent of each row: the smallest power of two that brings its largest value to 448 or
    less, at least 2^-127."""
    most = y.abs().amax(-1)
    m, e = torch.frexp(most)   # most = m 2^e, 1/2 <= m < 1; 448 = 7/8 2^9
    e = torch.where(most == 0, -127, torch.where(m > 0.875, e - 8, e - 9).clamp(min=-127))
    half = torch.div(-e, 2, rounding_mode="floor")   # 2^-e in two factors that 32 bits hold
    codes = y * torch.ldexp(torch.ones_like(most), half)[..., None] * torch.ldexp(torch.ones_like(most), -e - half)[..., None]
    return codes.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(codes, exponents):
    """What e4m3 rows stand for, in 32 bits."""
    return codes.float() * exponents.float()[..., None]


def _run_plain(x):
    if x["op"] in ("rope", "rope_back"):
        return [_rotated(x, y, x["op"] == "rope_back").to(y.dtype) for y in (x["q"], x["k"])]
    if x["op"] == "write":
        k = _rotated(x, x["k"]) if x["rotate"] else x["k"].float()
        kv = torch.stack([k, x["v"].float()], 1)   # [tokens][2][nkv][hd]
        slots, n_slots = x["slots"], x["pages"].shape[0] * PAGE
        # a token without a slot goes to one past the end of the pool
        slots = torch.where(slots < 0, n_slots, slots)

        def put(pool, rows):   # pool [pages][2][nkv][16]..., by its bytes or half words
            flat = pool.view(torch.uint8 if pool.element_size() == 1 else torch.int16)
            flat = torch.cat([flat.transpose(1, 3).transpose(2, 3).flatten(0, 1), torch.zeros_like(flat[:1, :, :, 0])])
            flat[slots] = rows.view(flat.dtype)
            back = flat[:-1].unflatten(0, (-1, PAGE)).transpose(2, 3).transpose(1, 3)
            pool.view(flat.dtype).copy_(back)

        if x["format"] == "bf16":
            put(x["pages"], kv.bfloat16())
        else:
            codes, exponents = _quantised(kv)
            put(x["pages"], codes)
            put(x["exponents"], exponents)
        return {"pages": x["pages"], "exponents": x["exponents"]}
    if x["op"] == "expand":
        src, dst = x["src"].long(), x["dst"].long()
        codes = x["pages"].view(torch.uint8)[src].view(torch.float8_e4m3fn)
        exponents = x["exponents"].view(torch.uint8)[src].view(torch.float8_e8m0fnu)
        x["out"][dst] = _values(codes, exponents).bfloat16()
        return x["out"]
    return _attention(x)


def _attention(x):
    n, most, nkv, hd = x["table"].shape[0], x["drafts"], x["nkv"], x["hd"]
    total, group = x["q"].shape[0], x["nq"] // nkv
    table = x["table"].long()
    if x["format"] == "bf16":
        kv = x["pages"][table].float()
    else:
        kv = _values(x["pages"].view(torch.uint8)[table].view(torch.float8_e4m3fn),
                     x["exponents"].view(torch.uint8)[table].view(torch.float8_e8m0fnu))
    kv = kv.permute(2, 0, 3, 1, 4, 5).reshape(2, n, nkv, -1, hd)          # [2][n][nkv][cached][hd]
    t = torch.arange(most, device="cuda")
    at = x["start"][:-1, None] + t
    live = at < x["start"][1:, None]
    at = at.clamp(max=total - 1)
    q = x["q"][at].float().view(n, most, nkv, group, hd).permute(0, 2, 1, 3, 4).reshape(n, nkv, most * group, hd)
    keys = torch.cat([kv[0], x["k"][at].float().transpose(1, 2)], 2)
    values = torch.cat([kv[1], x["v"][at].float().transpose(1, 2)], 2)
    s = torch.matmul(q, keys.transpose(-1, -2)) / math.sqrt(hd)
    cached = torch.arange(kv.shape[3], device="cuda") < x["lens"][:, None]
    seen = (x["mask"][at][:, :, t // 32] >> (t % 32)) & 1
    keep = torch.cat([cached[:, None].expand(n, most, -1), seen.bool() & live[:, None]], -1)
    s = s.view(n, nkv, most, group, -1).masked_fill_(~keep[:, None, :, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-1e30)
    p = (s - top).exp_()
    whole = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, nkv, most * group, -1), values).view(n, nkv, most, group, hd)
    o = torch.where(whole > 0, o / whole, 0.0).permute(0, 2, 1, 3, 4).reshape(n, most, nkv * group, hd)
    token = torch.arange(total, device="cuda", dtype=torch.int32)
    b = torch.searchsorted(x["start"][1:], token, right=True)
    return o[b, (token - x["start"][b]).long()].bfloat16()


# ---------------------------------------------------------------- the same in 64 bits
def _rotated64(x, freq, y, sign):
    angle = x["positions"].double()[:, None] * torch.tensor(freq, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones_like(angle), sign * angle)[:, None, :]
    y, rd = y.double().clone(), x["rd"]
    pairs = y[..., :rd].unflatten(-1, (-1, 2)) if x["interleaved"] else y[..., :rd].unflatten(-1, (2, -1)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y[..., :rd] = (z if x["interleaved"] else z.transpose(-1, -2)).flatten(-2)
    return y


def _e4m3_64(y):
    """|y| <= 448 to the nearest of e4m3's values (ties to even): steps of 1/8 of the power of two below, from 2^-9 on."""
    step = torch.exp2((torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3))
    return torch.round(y / step) * step


def exact(case, seed):
    c = case
    x = prepare(c, seed)
    hd, nq, nkv = c["hd"], c["nq"], c["nkv"]
    if c["op"] in ("rope", "rope_back"):
        freq = _frequencies(x)
        return [_rotated64(x, freq, y, -1.0 if c["op"] == "rope_back" else 1.0) for y in (x["q"], x["k"])]
    if c["op"] == "write":
        k = _rotated64(x, _frequencies(x), x["k"], 1.0) if c["rotate"] else x["k"].double()
        pages = x["pages"].double()
        exponents = x["exponents"].double() if c["format"] == "e4m3" else None
        used = x["slots"] >= 0
        page, off = x["slots"][used] // PAGE, x["slots"][used] % PAGE
        for i, y in enumerate((k, x["v"].double())):
            y = y[used]
            if c["format"] == "e4m3":
                e = torch.ceil(torch.log2(y.abs().amax(-1, keepdim=True) / 448.0)).clamp(min=-127)
                y = _e4m3_64(y * torch.exp2(-e))
                exponents[page, i, :, off] = torch.exp2(e)[..., 0]
            pages[page, i, :, off] = y
        return {"pages": pages, "exponents": exponents}
    if c["op"] == "expand":
        out = x["out"].double()
        for s, d in zip(x["src"].tolist(), x["dst"].tolist()):
            out[d] = x["pages"][s].double() * x["exponents"][s].double()[..., None]
        return out
    out = torch.zeros((x["q"].shape[0], nq, hd), dtype=torch.float64, device="cuda")
    lens, start, bits = x["lens"].tolist(), x["start"].tolist(), x["mask"].tolist()
    for b, n in enumerate(lens):
        ids = x["table"][b, :(n + PAGE - 1) // PAGE].tolist()
        s0, s1 = start[b], start[b + 1]
        if c["format"] == "bf16":
            rows = [x["pages"][i].double() for i in ids]
        else:
            rows = [x["pages"][i].double() * x["exponents"][i].double()[..., None] for i in ids]
        kv = torch.cat(rows, 2)[:, :, :n] if rows else out.new_zeros(2, nkv, 0, hd)
        see = torch.tensor([[bool(row[j // 32] >> (j % 32) & 1) for j in range(s1 - s0)] for row in bits[s0:s1]],
                           device="cuda").view(s1 - s0, s1 - s0)
        keep = torch.cat([torch.ones((s1 - s0, n), dtype=torch.bool, device="cuda"), see], 1)
        for g in range(nkv):
            keys = torch.cat([kv[0, g], x["k"][s0:s1, g].double()])
            values = torch.cat([kv[1, g], x["v"][s0:s1, g].double()])
            for h in range(g * nq // nkv, (g + 1) * nq // nkv):
                s = x["q"][s0:s1, h].double() @ keys.T / hd ** 0.5
                w = torch.softmax(s.masked_fill(~keep, -math.inf), -1)
                out[s0:s1, h] = w @ values
    return out
