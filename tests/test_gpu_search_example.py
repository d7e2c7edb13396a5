"""README.md's third example, run as written (random weights, queries, keys and values from torch): a search over a 4-bit cache.
Each step's drafted tokens attend to the pages and are written, the scorer reads the expanded pages, the best half of the
candidates go on twice each, and the pool is closed up at the end.  What every candidate holds after each step is compared with
its own history, quantised apart, and its rewards with those of a cache that was never forked."""
import numpy as np
import pytest

from tests import cache4_util as ref4
from tests import operators_util as ref
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def readme_example(steps=3):
    import torch
    from paper_2607_09153_gb300 import Rope, Scorer, cache_compact, cache_expand, cache_fork, cache_write, tree_attention

    L, d, nq, nkv, hd, ff, n_pages, width = 2, 256, 4, 2, 64, 1024, 64, 8
    torch.manual_seed(0)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    w = lambda *shape: (0.02 * torch.randn(*shape, device="cuda")).to(torch.bfloat16)  # noqa: E731
    weights = {"embed_verify": w(d), "final_norm": torch.ones(d, **bf), "w_plus": w(d), "w_minus": w(d),
               "layers": [{"attn_norm": torch.ones(d, **bf), "w_qkv": w((nq + 2 * nkv) * hd, d), "w_o": w(d, nq * hd),
                           "mlp_norm": torch.ones(d, **bf), "w_gate_up": w(2 * ff, d), "w_down": w(d, ff)}
                          for _ in range(L)]}
    scorer = Scorer(L, d, nq, nkv, hd, ff, weights, max_candidates=8, max_blocks_per_seq=width)
    rope = Rope(hd)                                       # the scorer's rope_base
    ints = lambda x, t=torch.int32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    # the cache: 4-bit pages of all layers, a power of two for each 32 elements, nobody's yet
    pages = torch.zeros(L, n_pages, 2, nkv, 16, hd // 2, dtype=torch.uint8, device="cuda")
    exponents = torch.zeros(L, n_pages, 2, nkv, 16, hd // 32, dtype=torch.uint8, device="cuda")
    pools, refs = [pages, exponents], torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    table, lens = torch.empty((0, width), dtype=torch.int32, device="cuda"), ints([])

    def write(l, seqs, at, k, v):
        """Tokens at position at[i] of sequence seqs[i]; returns their rotated keys."""
        slots = 16 * table[seqs, at // 16].long() + at % 16
        cache_write(pages[l], slots, k, v, exponents[l])

    # four prompts, a candidate each
    prompts = ints([37, 16, 50, 5])
    table, lens, refs, _ = cache_fork(pools, refs, table, lens, ints([-1] * 4), room=prompts)
    seqs = torch.repeat_interleave(torch.arange(4, device="cuda"), prompts)
    at = torch.cat([torch.arange(n, device="cuda") for n in prompts.tolist()])
    history = []                                          # (for the test)
    for l in range(L):
        k, v = torch.randn(len(seqs), nkv, hd, **bf), torch.randn(len(seqs), nkv, hd, **bf)
        (kr,) = rope.rotate(at.int(), k)
        write(l, seqs, at, kr, v)
        history.append([[(kr[seqs == s], v[seqs == s])] for s in range(4)])
    lens = prompts
    outputs, rewards = [], []
    for step in range(steps):
        # the best half go on twice each, with room for a step of 12 tokens (at first: all, twice)
        best = ints(range(4)) if step == 0 else ints(np.argsort(-rewards[-1], kind="stable")[:len(rewards[-1]) // 2])
        parents = best.repeat_interleave(2)
        table, lens, refs, counts = cache_fork(pools, refs, table, lens, parents, room=torch.full_like(parents, 12))
        n = len(parents)
        history = [[list(h[p]) for p in parents.tolist()] for h in history]
        # a step of each candidate: twelve tokens, each seeing those before it
        start, at = ints(range(0, 12 * n + 1, 12)), (lens[:, None] + torch.arange(12, device="cuda")).flatten()
        seqs = torch.arange(n, device="cuda").repeat_interleave(12)
        for l in range(L):
            rows = torch.randn(12 * n, nq + 2 * nkv, hd, **bf)
            qr, kr = rope.rotate(at.int(), rows[:, :nq], rows[:, nq:nq + nkv])
            v = rows[:, nq + nkv:]
            o = tree_attention(qr, kr, v, pages[l], table, lens, start, max_drafts=12, exponents=exponents[l])
            outputs.append((l, o, qr, kr, v, [list(h) for h in history[l]]))
            write(l, seqs, at.long(), kr, v)
            for s in range(n):
                history[l][s].append((kr[12 * s:12 * s + 12], v[12 * s:12 * s + 12]))
        lens = lens + 12
        # the scorer reads bf16
        kv = torch.empty(L, n_pages, 2, nkv, 16, hd, **bf)
        for l in range(L):
            cache_expand(pages[l], exponents[l], ints(range(n_pages)), kv[l])
        rewards.append(scorer.score(kv, table.cpu().numpy(), lens.cpu().numpy()))
    # what is in use to the pool's beginning
    table, refs, moved, counts = cache_compact(pools, refs, table, lens)
    return dict(locals())


def test_search_example():
    torch = require_gpu()
    x = readme_example()
    L, nkv, hd, table, lens, pools = (x[k] for k in ("L", "nkv", "hd", "table", "lens", "pools"))

    def quantised(parts):
        """Keys and values [tokens][nkv][hd] of a history, as 4 bits leave them."""
        return [ref4.values(*ref4.quantise(torch.cat([p[i] for p in parts]).double())) for i in (0, 1)]

    # each step's outputs against the attention over the candidates' own histories
    for l, o, q, k, v, histories in x["outputs"]:
        rows = [quantised(h) for h in histories]
        sizes, n = [len(r[0]) for r in rows], len(rows)
        seen = torch.ones((12, 12), dtype=torch.bool, device="cuda").tril().repeat(n, 1)
        want, a, peak = ref.attention(q, k, v, rows, sizes, list(range(0, 12 * n + 1, 12)), seen, hd ** -0.5)
        bound = ref.attention_bound(want, a, peak, max(sizes) + 12, hd)
        for s, (_, values) in enumerate(rows):   # small fp16 weights: as Tree4.want
            bound[12 * s:12 * s + 12] += 2.0 ** -37 * values.abs().sum(0).repeat_interleave(q.shape[1] // nkv, 0)
        assert bool(((o.double() - want).abs() <= bound).all())
    # what the closed-up pool holds: every candidate's history, bit by bit, in as few pages as it can be
    live = int(x["counts"][0])
    assert x["refs"][:live].min() >= 1 and not bool(x["refs"][live:].any()) and live < x["n_pages"] // 2
    apart = torch.zeros(L, 64, 2, nkv, 16, hd, dtype=torch.bfloat16, device="cuda")
    for l in range(L):
        for s, h in enumerate(x["history"][l]):
            n = int(lens[s])
            ids = table[s, :(n + 15) // 16].long()
            held = ref4.values(pools[0][l, ids], pools[1][l, ids]).permute(1, 0, 3, 2, 4).reshape(2, -1, nkv, hd)[:, :n]
            for i, want in enumerate(quantised(h)):
                assert torch.equal(held[i], want)
                for t in range(n):
                    apart[l, 8 * s + t // 16, i, :, t % 16] = want[t].bfloat16()
    # rewards of a cache without a shared page
    p = x["scorer"].score(apart, np.arange(64, dtype=np.int32).reshape(8, 8)[:len(lens)], lens.cpu().numpy())
    assert np.abs(p - x["rewards"][-1]).max() <= 2e-5, (p, x["rewards"][-1])
    x["scorer"].close()
