"""README.md's second example, run as written (random weights, queries, keys and values from torch): an 8-bit paged cache is
filled, drafted tokens attend to it and to each other, the accepted ones are written, and the scorer reads the cache
expanded to bf16.  Each step is compared with its formula in 64 bits."""
import numpy as np
import pytest

from tests import operators_util as ref
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def readme_example():
    import torch
    from paper_2607_09153_gb300 import Rope, Scorer, cache_expand, cache_write, tree_attention, tree_mask

    L, d, nq, nkv, hd, ff = 2, 256, 4, 2, 64, 1024
    torch.manual_seed(0)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    w = lambda *shape: (0.02 * torch.randn(*shape, device="cuda")).to(torch.bfloat16)  # noqa: E731
    weights = {"embed_verify": w(d), "final_norm": torch.ones(d, **bf), "w_plus": w(d), "w_minus": w(d),
               "layers": [{"attn_norm": torch.ones(d, **bf), "w_qkv": w((nq + 2 * nkv) * hd, d), "w_o": w(d, nq * hd),
                           "mlp_norm": torch.ones(d, **bf), "w_gate_up": w(2 * ff, d), "w_down": w(d, ff)}
                          for _ in range(L)]}
    scorer = Scorer(L, d, nq, nkv, hd, ff, weights, max_candidates=4, max_blocks_per_seq=8)
    ints = lambda x, t=torch.int32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    rope = Rope(hd, base=1e6)
    # the cache: per layer 32 pages of 16 tokens, 8 bits a value and a power of two per row; sequence s has pages 8 s ..
    pages = torch.zeros(L, 32, 2, nkv, 16, hd, device="cuda").to(torch.float8_e4m3fn)
    exponents = torch.zeros(L, 32, 2, nkv, 16, dtype=torch.uint8, device="cuda")
    block_table, lens = ints(np.arange(32).reshape(4, 8)), [120, 64, 17, 0]
    slot = lambda s, at: 128 * s + at                 # 16 * page + place  # noqa: E731
    where = [(s, i) for s in range(4) for i in range(lens[s])]
    prompt = [torch.randn(len(where), 2 * nkv, hd, **bf) for _ in range(L)]      # a layer's keys, then its values
    for l in range(L):
        cache_write(pages[l], ints([slot(*x) for x in where], torch.int64), prompt[l][:, :nkv], prompt[l][:, nkv:], exponents[l],
                    rope=rope, positions=ints([i for _, i in where]))
    # three drafted tokens of each sequence: one, and two that may follow it
    start, depth = [0, 3, 6, 9, 12], [0, 1, 1] * 4
    mask = tree_mask([-1, 0, 0] * 4, start).cuda()
    at = [lens[i // 3] + depth[i] for i in range(12)]
    drafts = [torch.randn(12, nq + 2 * nkv, hd, **bf) for _ in range(L)]         # queries, keys, values
    outputs = []
    for l in range(L):
        q, k, v = drafts[l][:, :nq], drafts[l][:, nq:nq + nkv], drafts[l][:, nq + nkv:]
        qr, kr = rope.rotate(ints(at), q, k)
        outputs.append(tree_attention(qr, kr, v, pages[l], block_table, ints(lens), ints(start), max_drafts=3,
                                      max_len=128, exponents=exponents[l], mask=mask))
        # accepted: the first and the third (-1: not written)
        cache_write(pages[l], ints([slot(i // 3, at[i]) if i % 3 != 1 else -1 for i in range(12)], torch.int64), k, v,
                    exponents[l], rope=rope, positions=ints(at))
    # the scorer reads bf16
    kv = torch.empty(L, 32, 2, nkv, 16, hd, **bf)
    for l in range(L):
        cache_expand(pages[l], exponents[l], ints(range(32)), kv[l])
    p_plus = scorer.score(kv, block_table.cpu().numpy(), np.array(lens, dtype=np.int32) + 2)
    return dict(locals())


def test_drafts_example():
    require_gpu()
    import torch
    x = readme_example()
    L, nq, nkv, hd, lens, start, at = (x[k] for k in ("L", "nq", "nkv", "hd", "lens", "start", "at"))
    freq = ref.frequencies(hd, 1e6)
    seen = ref.unpack_mask(x["mask"], 3)
    assert seen[:3].tolist() == [[True, False, False], [True, True, False], [True, False, True]]
    for l in range(L):
        # what the prompt and the accepted tokens leave in the cache, quantised in 64 bits from the bf16 inputs: e4m3's
        # steps are 2^-4 of a value at most, 2^-10 2^e below the normal range (the row's largest lies above 224 2^e);
        # fp32 rotation before it moves values by 2^-20 of the pair at most
        kv = x["kv"][l].double()
        value = kv.permute(0, 3, 1, 2, 4).reshape(512, 2, nkv, hd)   # [slot][key, value]
        prompt, drafts = x["prompt"][l], x["drafts"][l]
        first = torch.tensor([128 * s + i for s, i in x["where"]]).cuda()
        kept = [i for i in range(12) if i % 3 != 1]
        later = torch.tensor([128 * (i // 3) + at[i] for i in kept]).cuda()
        for rows, k, v, positions in ((first, prompt[:, :nkv], prompt[:, nkv:], [i for _, i in x["where"]]),
                                      (later, drafts[kept][:, nq:nq + nkv], drafts[kept][:, nq + nkv:], [at[i] for i in kept])):
            want = torch.stack([ref.rotate(k, torch.tensor(positions).cuda(), freq), v.double()], 1)
            top = want.abs().amax(-1, keepdim=True)
            assert bool(((value[rows] - want).abs() <= 2.0 ** -4 * want.abs() + (2.0 ** -17 + 2.0 ** -18) * top).all())
        # the drafts' outputs against the attention over that cache, before the accepted tokens came
        q, k = (t.bfloat16() for t in x["rope"].rotate(x["ints"](at), drafts[:, :nq], drafts[:, nq:nq + nkv]))
        rows = [(value[128 * s:128 * s + lens[s], 0], value[128 * s:128 * s + lens[s], 1]) for s in range(4)]
        o, a, peak = ref.attention(q, k, drafts[:, nq + nkv:], rows, lens, start, seen, hd ** -0.5)
        assert bool(((x["outputs"][l].double() - o).abs() <= ref.attention_bound(o, a, peak, 123, hd)).all())
    # the same cache in other pages: the same rewards
    order = torch.randperm(32, device="cuda")
    moved = torch.empty_like(x["kv"])
    moved[:, order] = x["kv"]
    p = x["scorer"].score(moved, order[x["block_table"].long()].int().cpu().numpy(), np.array(lens, dtype=np.int32) + 2)
    assert np.array_equal(p, x["p_plus"]) and np.all((p > 0) & (p < 1)), (p, x["p_plus"])
    x["scorer"].close()
