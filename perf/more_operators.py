"""The operators of a search that keeps its candidates in a 4-bit cache: tokens stored in 4 bits and made readable to the
scorer, attention of drafted tokens over 4-bit pages, and the pages' bookkeeping when candidates are dropped, doubled and
extended, or when the pool is to be closed up.

4-bit rows: e2m1 codes (0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign; two in a byte, the first in its low half) with a power of two
(an exponent byte, 127 for one) for every 32 elements.

A case is a dict of plain values.  `op` and what goes with it:
  "store"    tokens, nkv, hd, dtype, fused    keys and values of tokens written in 4 bits, and the pages that they went to
                                              expanded into the scorer's
  "expand"   n pages of a pool of `pool`, nkv, hd: 4-bit pages into the scorer's
  "attend"   n sequences of up to `drafts` drafted tokens each, nq, nkv, hd
             cache                            "equal": len cached tokens each; "ragged": len / 16 .. len, one of them 0
  "fork"     n sequences of which `new` descend, layers, nkv, hd, format ("bf16", "e4m3")
             shared, len, room                tokens of a common beginning, of a sequence's own at most, and to come at most
  "compact"  n sequences of up to len tokens in a pool of `pool` pages, layers, nkv, hd, format
  shape_seed draws lengths and descent (sizes belong to the case, values to the seed)
"""
import math
import random

import torch

own = False

PAGE = 16
BLOCK = 32     # elements that share a power of two

SHAPES = {   # heads of the repository's scorers
    "tiny": dict(nq=4, nkv=2, hd=64),
    "small64": dict(nq=16, nkv=4, hd=64),
    "1p5b": dict(nq=12, nkv=2, hd=128),
    "7b": dict(nq=28, nkv=4, hd=128),
    "8b": dict(nq=32, nkv=8, hd=128),
}
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _store(name, shape, tokens, dtype="bf16", fused=True):
    return dict(name=name, op="store", tokens=tokens, dtype=dtype, fused=fused, **SHAPES[shape])


def _expand(name, shape, n, pool):
    return dict(name=name, op="expand", n=n, pool=pool, **SHAPES[shape])


def _attend(name, shape, n, drafts, cache, len_, shape_seed=1):
    return dict(name=name, op="attend", n=n, drafts=drafts, cache=cache, len=len_, shape_seed=shape_seed, **SHAPES[shape])


def _fork(name, shape, layers, format, n, new, shared, len_, room, shape_seed=1):
    return dict(name=name, op="fork", layers=layers, format=format, n=n, new=new, shared=shared, len=len_, room=room,
                shape_seed=shape_seed, **SHAPES[shape])


def _compact(name, shape, layers, format, n, len_, pool, shape_seed=1):
    return dict(name=name, op="compact", layers=layers, format=format, n=n, len=len_, pool=pool, shape_seed=shape_seed,
                **SHAPES[shape])


def listed():
    return [
        # one decoding step of a 64-wide beam: each candidate's token stored, its page made readable
        _store("store_step_7b", "7b", 64),
        # whole trajectories stored and made readable
        _store("store_prompt_8b", "8b", 30001),
        # a few pages of one candidate made readable to the scorer
        _expand("expand_few_small", "small64", 24, 40),
        # a batch's pages made readable to the scorer
        _expand("expand_batch_8b", "8b", 4099, 4200),
        # the smallest step: four short sequences, one token each
        _attend("attend_tiny", "tiny", 4, 1, "equal", 128),
        # plain decoding of many uneven sequences
        _attend("attend_decode_7b", "7b", 64, 1, "ragged", 9001),
        # a few drafts behind few, long contexts
        _attend("attend_long_8b", "8b", 8, 4, "equal", 32768),
        # wide trees of drafts, uneven contexts
        _attend("attend_wide_7b", "7b", 16, 64, "ragged", 16384),
        # a step of a small search: half of 16 candidates go on, twice each
        _fork("fork_step_small", "small64", 2, "e4m3", 16, 16, 128, 500, 4),
        # a beam after scoring: 256 candidates descend from the best quarter of 64, in all layers
        _fork("fork_beam_7b", "7b", 28, "bf16", 64, 256, 4096, 200, 40),
        # a few pages of a small pool closed up
        _compact("compact_small", "tiny", 2, "bf16", 8, 100, 120),
        # what a search has left behind in a pool of all layers closed up
        _compact("compact_pool_7b", "7b", 28, "e4m3", 48, 600, 2000),
    ]


def draw(rng):
    def logint(lo, hi):
        return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    while True:
        op = rng.choice(["store", "expand", "attend", "attend", "attend", "fork", "compact"])
        shape = rng.choice(["tiny", "small64", "1p5b", "7b", "8b"])
        hd, nkv, nq = SHAPES[shape]["hd"], SHAPES[shape]["nkv"], SHAPES[shape]["nq"]
        if op == "store":
            c = _store("", shape, logint(1, 32768), rng.choice(["bf16", "fp16", "fp32"]), rng.random() < 0.5)
        elif op == "expand":
            n = logint(1, 4096)
            c = _expand("", shape, n, n + logint(1, 64))
        elif op == "attend":
            c = _attend("", shape, logint(1, 64), logint(1, 64), rng.choice(["equal", "ragged"]), logint(1, 65536),
                        rng.randrange(1 << 30))
            cached, longest = sum(_lens(c)), max(_lens(c))
            # no dearer than the largest listed case, and what the plain form holds in 32 bits fits a few GB
            if cached * c["drafts"] * nq > 16 * 64 * 28 * 9000 or cached > 1 << 18:
                continue
            if c["n"] * longest * nkv * hd > 1 << 29 or c["n"] * c["drafts"] * nq * longest > 1 << 30:
                continue
        elif op == "fork":
            c = _fork("", shape, rng.choice([1, 2, 28, 32]), rng.choice(["bf16", "e4m3"]), logint(1, 128), logint(1, 256),
                      logint(1, 8192), logint(1, 1000), logint(1, 64), rng.randrange(1 << 30))
            if _page_elements(c) * _pool_pages(c) > 900 << 20:
                continue
        else:
            n, len_ = logint(1, 128), logint(1, 2000)
            c = _compact("", shape, rng.choice([1, 2, 28, 32]), rng.choice(["bf16", "e4m3"]), n, len_,
                         n * ((len_ + PAGE - 1) // PAGE) + logint(4, 1000), rng.randrange(1 << 30))
            if _page_elements(c) * c["pool"] > 900 << 20:
                continue
        del c["name"]
        return c


# ---------------------------------------------------------------- sizes
def _ceil(n):
    return (n + PAGE - 1) // PAGE


def _lens(c):
    rng = random.Random(c["shape_seed"])
    if c["op"] == "fork":   # a common beginning and something of one's own
        return [c["shared"] + rng.randint(0, c["len"]) for _ in range(c["n"])]
    if c["op"] == "compact":
        return [rng.randint(0, c["len"]) for _ in range(c["n"])]
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


def _descent(c):
    """(parents, room): whom each new sequence continues -- one of the best quarter to half, or nobody -- and for how many tokens
    it wants room."""
    rng = random.Random(c["shape_seed"] + 2)
    best = rng.sample(range(c["n"]), max(1, c["n"] // rng.choice([2, 4])))
    parents = [rng.choice(best) for _ in range(c["new"])]
    if c["new"] > 8:
        parents[c["new"] // 2] = -1   # a request that begins
    return parents, [rng.randint(0, c["room"]) for _ in range(c["new"])]


HELD = 3   # pages of a pool that others hold


def _fork_pages(c):
    """(pages in use before, pages that are copied, pages that are new)."""
    lens, (parents, room) = _lens(c), _descent(c)
    common = c["shared"] // PAGE
    used = common + sum(_ceil(n) - common for n in lens)
    ends, copies, more = set(), 0, 0
    for p, r in zip(parents, room):
        n = lens[p] if p >= 0 else 0
        if n % PAGE:
            copies += p in ends
            ends.add(p)
        more += _ceil(n + r) - _ceil(n)
    return used, copies, more


def _pool_pages(c):
    used, copies, more = _fork_pages(c)
    return used + copies + more + HELD + 5


def _page_elements(c):
    return c["layers"] * 2 * c["nkv"] * PAGE * c["hd"]


def _page_bytes(c):
    e = _page_elements(c)
    return 2 * e if c["format"] == "bf16" else e + e // c["hd"]


def _live(c):
    """Which pages of a pool its sequences and others hold, in the order of their numbers, by the case's own lot."""
    used = sum(_ceil(n) for n in _lens(c)) + HELD
    return random.Random(c["shape_seed"] + 3).sample(range(c["pool"]), used)


def _moves(c):
    live = _live(c)
    return sum(p >= len(live) for p in live)


def work(case):
    c = case
    hd, nq, nkv = c["hd"], c["nq"], c["nkv"]
    row = hd // 2 + hd // BLOCK   # bytes of a 4-bit row
    if c["op"] == "store":
        size, rows = DTYPES[c["dtype"]].itemsize, 2 * c["tokens"] * nkv
        pages = c["tokens"] if c["tokens"] < 256 else _ceil(c["tokens"])
        read = 2 * pages * nkv * PAGE
        return {"bytes": size * rows * hd + rows * row + 8 * c["tokens"] + read * (row + 2 * hd) + 8 * pages,
                "flops": 4 * rows * hd}
    if c["op"] == "expand":
        rows = 2 * c["n"] * nkv * PAGE
        return {"bytes": rows * (row + 2 * hd) + 8 * c["n"], "flops": rows * hd}
    if c["op"] == "fork":
        used, copies, more = _fork_pages(c)
        lens, (parents, room) = _lens(c), _descent(c)
        before = sum(_ceil(n) for n in lens)
        after = sum(_ceil((lens[p] if p >= 0 else 0) + r) for p, r in zip(parents, room))
        return {"bytes": 2 * copies * _page_bytes(c) + 4 * (before + after + 2 * _pool_pages(c) + c["n"] + 3 * c["new"]),
                "flops": 0}
    if c["op"] == "compact":
        return {"bytes": 2 * _moves(c) * _page_bytes(c) + 4 * (3 * c["pool"] + 2 * sum(_ceil(n) for n in _lens(c)) + c["n"]),
                "flops": 0}
    lens, drafts = _lens(c), _drafts(c)
    n = sum(drafts)
    total = 2 * nkv * row * sum(lens) + 2 * n * hd * (2 * nq + 2 * nkv) + 4 * n * ((c["drafts"] + 31) // 32)
    pairs = sum(t * (x + (t + 1) / 2) for t, x in zip(drafts, lens))
    return {"bytes": total + 4 * (sum(_ceil(x) for x in lens) + 2 * c["n"] + 1), "flops": 4 * hd * nq * pairs}


# ---------------------------------------------------------------- inputs
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


def _pool4(pages, nkv, hd, gen):
    """A used 4-bit pool: codes [pages][2][nkv][16][hd / 2], exponents [pages][2][nkv][16][hd / 32]."""
    # codes as quantised N(0, 1) rows have them: the largest of 32 between 3 and 6
    codes = torch.empty((pages, 2, nkv, PAGE, hd // 2), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (2 * nkv * PAGE * hd))
    for a in range(0, pages, step):
        y = _normal((min(step, pages - a), 2, nkv, PAGE, hd), 1.9, gen, torch.float32).clamp_(-6.0, 6.0)
        c = _codes(y)
        codes[a:a + step] = c[..., 0::2] | (c[..., 1::2] << 4)
    exponents = torch.randint(127 - 2, 127 + 1, (pages, 2, nkv, PAGE, hd // BLOCK), dtype=torch.uint8, device="cuda",
                              generator=gen)
    return codes, exponents.view(torch.float8_e8m0fnu)


def _layers(c, pages, gen):
    """Pools of all layers whose pages are moved: [layers][pages][2][nkv][16][hd], and for e4m3 exponents without the hd."""
    shape = (c["layers"], pages, 2, c["nkv"], PAGE, c["hd"])
    if c["format"] == "bf16":
        return [_normal(shape, 1.0, gen, torch.bfloat16)]
    codes = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
    for layer in codes:
        layer.copy_(_normal(layer.shape, 100.0, gen, torch.float32).clamp_(-448.0, 448.0))
    exponents = torch.randint(127 - 8, 127 - 5, shape[:-1], dtype=torch.uint8, device="cuda", generator=gen)
    return [codes, exponents.view(torch.float8_e8m0fnu)]


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


def _table(ids, blocks, width):
    """int32 [sequences][width] with `blocks` page numbers each, taken from `ids` in turn."""
    table, at = torch.zeros((len(blocks), max(1, width)), dtype=torch.int32), 0
    for b, k in enumerate(blocks):
        table[b, :k] = ids[at:at + k]
        at += k
    return table


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cpu = torch.Generator().manual_seed(seed)
    hd, nq, nkv = c["hd"], c["nq"], c["nkv"]
    x = dict(c)
    if c["op"] == "store":
        n = c["tokens"]
        x["k"], x["v"] = _heads(n, (nkv, nkv), hd, (2.0, 0.5), c["fused"], gen, DTYPES[c["dtype"]])
        step = n < 256
        used = n if step else _ceil(n)
        pages = used + 3
        x["pages"], x["exponents"] = _pool4(pages, nkv, hd, gen)
        order = torch.randperm(pages, generator=cpu)
        if step:   # a slot somewhere in a page of its own for each sequence
            slots = order[:n] * PAGE + torch.randint(0, PAGE, (n,), generator=cpu)
        else:      # trajectories: page after page, in no particular order of pages
            slots = order[torch.arange(n) // PAGE] * PAGE + torch.arange(n) % PAGE
        slots[torch.rand(n, generator=cpu) < 0.02] = -1   # padding of the batch: not written
        x["slots"] = slots.cuda()
        x["src"] = order[:used].int().cuda()
        x["dst"] = torch.randperm(used, generator=cpu).int().cuda()
        x["out"] = torch.zeros((used, 2, nkv, PAGE, hd), dtype=torch.bfloat16, device="cuda")
    elif c["op"] == "expand":
        x["pages"], x["exponents"] = _pool4(c["pool"], nkv, hd, gen)
        x["src"] = torch.randperm(c["pool"], generator=cpu)[:c["n"]].int().cuda()
        x["dst"] = torch.randperm(c["n"] + 1, generator=cpu)[:c["n"]].int().cuda()
        x["out"] = torch.zeros((c["n"] + 1, 2, nkv, PAGE, hd), dtype=torch.bfloat16, device="cuda")
    elif c["op"] == "attend":
        lens, drafts = _lens(c), _drafts(c)
        blocks = [_ceil(n) for n in lens]
        total = sum(blocks) + 3
        x["pages"], x["exponents"] = _pool4(total, nkv, hd, gen)
        table = _table(torch.randperm(total, generator=cpu).int(), blocks, max(blocks))
        start = torch.tensor([0] + drafts).cumsum(0).int()
        # scores q.k / sqrt(hd) with a spread of about two, as a trained model's
        x["q"], x["k"], x["v"] = _heads(int(start[-1]), (nq, nkv, nkv), hd, (2.0, 1.0, 1.0), True, gen, torch.bfloat16)
        x.update(table=table.cuda(), lens=torch.tensor(lens, dtype=torch.int32).cuda(), start=start.cuda(),
                 mask=_tree_masks(drafts, (c["drafts"] + 31) // 32, cpu), longest=max(lens))
    elif c["op"] == "fork":
        lens, (parents, room) = _lens(c), _descent(c)
        pages, common = _pool_pages(c), c["shared"] // PAGE
        blocks = [_ceil(n) for n in lens]
        order = torch.randperm(pages, generator=cpu).int()
        mine = _table(order[HELD + common:], [k - common for k in blocks], max(blocks) - common)
        table = torch.cat([order[HELD:HELD + common].expand(c["n"], -1), mine], 1).contiguous()
        refs = torch.zeros(pages, dtype=torch.int32)
        refs[order[:HELD].long()] = 1
        in_use = torch.arange(table.shape[1]) < torch.tensor(blocks)[:, None]
        refs += torch.bincount(table[in_use].long(), minlength=pages).int()
        x["width"] = max(blocks) + _ceil(c["room"])
        x.update(table=table.cuda(), lens=torch.tensor(lens, dtype=torch.int32).cuda(), refs=refs.cuda(),
                 parents=torch.tensor(parents, dtype=torch.int32).cuda(), want=torch.tensor(room, dtype=torch.int32).cuda(),
                 pools=_layers(c, pages, gen))
        # the tables that the next step reads, as a program keeps them in turn with the present ones
        x["out"] = (torch.empty((c["new"], x["width"]), dtype=torch.int32, device="cuda"),
                    torch.empty(c["new"], dtype=torch.int32, device="cuda"), torch.empty_like(x["refs"]),
                    torch.empty(2, dtype=torch.int32, device="cuda"))
    else:
        lens = _lens(c)
        blocks = [_ceil(n) for n in lens]
        live = torch.tensor(_live(c), dtype=torch.int32)[torch.randperm(sum(blocks) + HELD, generator=cpu)]
        table = _table(live[HELD:], blocks, max(blocks))
        refs = torch.zeros(c["pool"], dtype=torch.int32)
        refs[live.long()] = torch.randint(1, 4, (len(live),), generator=cpu, dtype=torch.int32)
        x.update(table=table.cuda(), lens=torch.tensor(lens, dtype=torch.int32).cuda(), refs=refs.cuda(),
                 pools=_layers(c, c["pool"], gen))
        x["out"] = (torch.empty_like(x["table"]), torch.empty_like(x["refs"]), torch.empty_like(x["refs"]),
                    torch.empty(2, dtype=torch.int32, device="cuda"))
    return x


# ---------------------------------------------------------------- one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(x):
    import paper_2607_09153_gb300 as kp
    if x["op"] == "store":
        kp.cache_write(x["pages"], x["slots"], x["k"], x["v"], exponents=x["exponents"])
        return kp.cache_expand(x["pages"], x["exponents"], x["src"], x["out"], x["dst"])
    if x["op"] == "expand":
        return kp.cache_expand(x["pages"], x["exponents"], x["src"], x["out"], x["dst"])
    if x["op"] == "attend":
        return kp.tree_attention(x["q"], x["k"], x["v"], x["pages"], x["table"], x["lens"], x["start"],
                                 max_drafts=x["drafts"], max_len=x["longest"], exponents=x["exponents"], mask=x["mask"])
    if x["op"] == "fork":
        table, lens, refs, counts = kp.cache_fork(x["pools"], x["refs"], x["table"], x["lens"], x["parents"], room=x["want"],
                                                  out=x["out"])
        return {"table": table, "lens": lens, "refs": refs, "counts": counts, "pools": x["pools"]}
    table, refs, moved, counts = kp.cache_compact(x["pools"], x["refs"], x["table"], x["lens"], out=x["out"])
    return {"table": table, "refs": refs, "moved": moved, "counts": counts, "pools": x["pools"]}


def _codes(y):
    """e2m1 codes (uint8) of |y| <= 6: to nearest, ties to the even code."""
    m = y.abs()
    # the values between two neighbours; one that is on the border goes to the even code
    up = (m > 0.25).byte() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)
    return up | (torch.signbit(y).byte() << 3)


def _quantised(y):
    """Codes (a byte each) and exponent bytes of rows in 32 bits: for every 32 elements the smallest power of two that brings
    their largest magnitude to 6 or less, at least 2^-127."""
    y = y.unflatten(-1, (-1, BLOCK))
    most = y.abs().amax(-1)
    m, e = torch.frexp(most)   # most = m 2^e, 1/2 <= m < 1; 6 = 3/4 2^3
    e = torch.where(most == 0, -127, torch.where(m > 0.75, e - 2, e - 3).clamp(min=-127)).int()
    down = ((127 - e) << 23).view(torch.float32)   # 2^-e by its bits: no power function rounds it
    return _codes(y * down[..., None]).flatten(-2), (e + 127).byte()


def _values(codes, exponents):
    """What 4-bit rows stand for, in 32 bits."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    e, m = (c >> 1) & 3, (c & 1).float()
    y = torch.where(e == 0, 0.5 * m, (1.0 + 0.5 * m) * (1 << e.int()).float() * 0.5)
    y = torch.where(c > 7, -y, y)
    return (y.unflatten(-1, (-1, BLOCK)) * exponents.view(torch.float8_e8m0fnu).float()[..., None]).flatten(-2)


def _run_plain(x):
    if x["op"] == "store":
        kv = torch.stack([x["k"].float(), x["v"].float()], 1)   # [tokens][2][nkv][hd]
        used = (x["slots"] >= 0).nonzero()[:, 0]
        page, place = x["slots"][used] // PAGE, x["slots"][used] % PAGE
        codes, exponents = _quantised(kv[used])
        x["pages"][page, :, :, place] = codes[..., 0::2] | (codes[..., 1::2] << 4)
        x["exponents"].view(torch.uint8)[page, :, :, place] = exponents
    if x["op"] in ("store", "expand"):
        src = x["src"].long()
        x["out"][x["dst"].long()] = _values(x["pages"][src], x["exponents"].view(torch.uint8)[src]).bfloat16()
        return x["out"]
    if x["op"] == "attend":
        return _attention(x)
    return _forked(x) if x["op"] == "fork" else _compacted(x)


def _attention(x):
    n, most, nkv, hd = x["table"].shape[0], x["drafts"], x["nkv"], x["hd"]
    total, group = x["q"].shape[0], x["nq"] // nkv
    table = x["table"].long()
    kv = _values(x["pages"][table], x["exponents"].view(torch.uint8)[table])
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


def _bits(pool):
    """A pool as elements that can be indexed whatever they stand for."""
    return pool.view(torch.uint8 if pool.element_size() == 1 else torch.int16)


def _forked(x):
    """New sequences in place of the old ones: full pages shared, a page that ends inside kept by the first of its descendants
    (where nobody else holds it) and copied for the others, pages for what is to come; the lowest free pages in turn."""
    table, lens, refs = x["table"], x["lens"], x["refs"]
    n, w = table.shape
    N, width, m = refs.shape[0], x["width"], x["parents"].shape[0]
    i32 = dict(dtype=torch.int32, device="cuda")
    fresh = (x["parents"] < 0) | (x["parents"] >= n)
    parent = x["parents"].clamp(0, n - 1).long()
    held, full = (lens + PAGE - 1) // PAGE, lens // PAGE
    b, order = torch.arange(w, **i32), torch.arange(m, **i32)
    children = torch.zeros(n, **i32).index_add_(0, parent, (~fresh).int())
    change = torch.where(b < full[:, None], children[:, None] - 1, -1) * (b < held[:, None])
    after = torch.cat([refs, torch.zeros(1, **i32)])   # (one more page, for what has none)
    after.index_add_(0, table.flatten().long(), change.flatten().int())
    len_, h, f = (torch.where(fresh, 0, y[parent]) for y in (lens, held, full))
    rows = table[parent]
    open_ = f < h
    last = torch.where(open_, rows.gather(1, f.clamp(max=w - 1).long()[:, None])[:, 0], N).long()
    first = torch.full((N + 1,), m, **i32).scatter_reduce_(0, last, order, "amin")
    keeps = open_ & (after[last] == 0) & (first[last] == order)
    after.index_add_(0, last, keeps.int())
    copies = (open_ & ~keeps).int()
    need = copies + (len_ + x["want"] + PAGE - 1) // PAGE - h
    at = need.cumsum(0).int() - need
    free = after[:N] <= 0
    rank, total, have = free.cumsum(0) - 1, need.sum(), free.sum()
    pages = torch.full((N + 1,), -1, **i32)
    pages.scatter_(0, torch.where(free, rank, N), torch.arange(N, **i32))
    pages[N] = -1
    after = after[:N] + (free & (rank < total)).int()
    c = torch.arange(width, **i32)
    old = torch.cat([rows, torch.full((m, width), -1, **i32)], 1)[:, :width]
    mine = torch.where((c >= h[:, None]) & (c < (h + need - copies)[:, None]), (at + copies - h)[:, None] + c, -1)
    mine = torch.where((c == f[:, None]) & (copies > 0)[:, None], at[:, None], mine)
    new = torch.where(mine >= 0, pages[mine.clamp(0, N).long()], torch.where(c < h[:, None], old, -1))
    dst = pages[at.clamp(max=N).long()]
    who = ((copies > 0) & (dst >= 0)).nonzero()[:, 0]
    src, dst = last[who], dst[who].long()
    [_bits(p).index_copy_(1, dst, _bits(p).index_select(1, src)) for p in x["pools"]]
    counts = torch.stack([(have - total).clamp(min=0), (total - have).clamp(min=0)]).int()
    return {"table": new, "lens": len_, "refs": after, "counts": counts, "pools": x["pools"]}


def _compacted(x):
    """Pages in use behind the first as many move into the free ones before, in order."""
    refs, N = x["refs"], x["refs"].shape[0]
    page = torch.arange(N, dtype=torch.int32, device="cuda")
    live = refs > 0
    count = live.sum()
    hole, high = ~live & (page < count), live & (page >= count)
    holes = torch.full((N + 1,), -1, dtype=torch.int32, device="cuda")
    holes.scatter_(0, torch.where(hole, hole.cumsum(0) - 1, N), page)
    moved = torch.where(high, holes[(high.cumsum(0) - 1).clamp(min=0)], torch.where(live, page, -1))
    after = torch.zeros(N + 1, dtype=torch.int32, device="cuda").scatter_(0, torch.where(live, moved, N).long(), refs)[:N]
    valid = torch.arange(x["table"].shape[1], device="cuda") < (x["lens"][:, None] + PAGE - 1) // PAGE
    after = torch.where(page < count, after, 0)
    table = torch.where(valid, moved[x["table"].long()], -1)
    src = high.nonzero()[:, 0]
    dst = moved[src].long()
    [_bits(p).index_copy_(1, dst, _bits(p).index_select(1, src)) for p in x["pools"]]
    counts = torch.stack([count, high.sum()]).int()
    return {"table": table, "refs": after, "moved": moved, "counts": counts, "pools": x["pools"]}


# ---------------------------------------------------------------- the same in 64 bits
VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _rows64(codes, exponents):
    """4-bit rows in 64 bits, by a table of the values."""
    table = torch.tensor(VALUES + [-v for v in VALUES], dtype=torch.float64, device="cuda")
    y = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.float64, device="cuda")
    y[..., 0::2], y[..., 1::2] = table[(codes % 16).int()], table[(codes // 16).int()]
    return y * exponents.double().repeat_interleave(BLOCK, -1)


def exact(case, seed):
    c = case
    x = prepare(c, seed)
    hd, nq, nkv = c["hd"], c["nq"], c["nkv"]
    if c["op"] in ("store", "expand"):
        pages = _rows64(x["pages"], x["exponents"])
        if c["op"] == "store":
            used = x["slots"] >= 0
            page, place = x["slots"][used] // PAGE, x["slots"][used] % PAGE
            for i, y in enumerate((x["k"], x["v"])):
                y = y[used].double().unflatten(-1, (-1, BLOCK))
                # of every power of two, the first that 6 times reaches the largest magnitude
                power = torch.tensor([2.0 ** i for i in range(-127, 128)], dtype=torch.float64, device="cuda")
                scale = power[torch.searchsorted(6.0 * power, y.abs().amax(-1, keepdim=True))]
                y = y / scale
                # to the nearest of steps of 1/2 below 2, of 1 below 4, of 2 above, ties to even multiples
                step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
                pages[page, i, :, place] = (torch.round(y / step) * step * scale).flatten(-2)
        out = x["out"].double()
        for s, d in zip(x["src"].tolist(), x["dst"].tolist()):
            out[d] = pages[s]
        return out
    if c["op"] in ("fork", "compact"):
        copies = _fork_copies(x) if c["op"] == "fork" else _compact_copies(x)
        pools = [p.double() for p in x["pools"]]
        for pool in pools:
            for s, d in copies:
                pool[:, d] = pool[:, s]
        names = ("table", "lens", "refs", "counts") if c["op"] == "fork" else ("table", "refs", "moved", "counts")
        return {**{k: None for k in names}, "pools": pools}
    out = torch.zeros((x["q"].shape[0], nq, hd), dtype=torch.float64, device="cuda")
    lens, start, bits = x["lens"].tolist(), x["start"].tolist(), x["mask"].tolist()
    for b, n in enumerate(lens):
        ids = x["table"][b, :_ceil(n)].long()
        s0, s1 = start[b], start[b + 1]
        kv = _rows64(x["pages"][ids], x["exponents"].view(torch.uint8)[ids].view(torch.float8_e8m0fnu))
        kv = kv.permute(1, 2, 0, 3, 4).reshape(2, nkv, -1, hd)[:, :, :n]
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


def _fork_copies(x):
    """(from, to) of the pages that a fork copies, sequence by sequence."""
    table, lens, parents, refs = (x[k].tolist() for k in ("table", "lens", "parents", "refs"))
    for s, n in enumerate(lens):
        for p in table[s][:_ceil(n)]:
            refs[p] -= 1
    for p in parents:
        if p >= 0:
            for page in table[p][:lens[p] // PAGE]:
                refs[page] += 1
    kept, ends = set(), []
    for i, p in enumerate(parents):
        end = table[p][lens[p] // PAGE] if p >= 0 and lens[p] % PAGE else None
        keeps = end is not None and refs[end] == 0 and end not in kept
        if keeps:
            kept.add(end)
        ends.append(None if keeps else end)
    free = iter([p for p, r in enumerate(refs) if r == 0 and p not in kept])
    copies = []
    for p, end, more in zip(parents, ends, x["want"].tolist()):
        n = lens[p] if p >= 0 else 0
        if end is not None:
            copies.append((end, next(free)))
        for _ in range(_ceil(n + more) - _ceil(n)):
            next(free)
    return copies


def _compact_copies(x):
    live = [p for p, r in enumerate(x["refs"].tolist()) if r > 0]
    holes = sorted(set(range(len(live))) - set(live))
    return list(zip([p for p in live if p >= len(live)], holes))
