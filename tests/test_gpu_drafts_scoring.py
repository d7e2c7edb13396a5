"""A cache that the operators wrote, scored: a decoder's keys (not rotated yet) and values are rotated, written page by page,
in bf16 or in 8 bits, and expanded; the scorer's P(+) and read-outs are those of the oracle, which re-encodes the whole
text.  The scorer rotates its query with the base that the keys were rotated with."""
import dataclasses
import os
import re

import numpy as np
import pytest

import kvsynth as ks
import oracle
from oracle.reencode import reencode
from tests import operators_util as ref
from tests.gpu_util import ATTN_RTOL, P_PLUS_ATOL, attn_rel_err, require_gpu

LENS = (40, 17, 0, 100)


class Model:
    """Random weights whose attention is peaked, texts, and what re-encoding them gives."""

    def __init__(self, base, seed=77):
        self.arch = dataclasses.replace(ks.ARCH_TINY, rope_base=base)
        self.weights = ks.host_weights(self.arch, seed, ks.Tables.make(0.2, qkv_std=0.1))
        self.texts = [np.random.default_rng(1000 + n).normal(0, 1, (n, self.arch.d_model)) for n in LENS]
        out = [reencode(self.arch, self.weights, xs, mirror=False) for xs in self.texts]
        self.p = np.array([x[0] for x in out])
        self.attn = np.stack([x[1] for x in out], 1)
        self.cache = [x[2] for x in out]   # [text][layer] (keys rotated, values), bf16 bits [n][n_kv][head_dim]


def test_bases_matter():
    """The check can see a base that differs: the same texts' caches, rotated with another one, move P(+) far beyond the
    tolerance.  (On the CPU, in the oracle.)"""
    for base, other in ((1e4, 1e6), (1e6, 1e4)):
        m, wrong = Model(base), Model(other)
        kv = [[wrong.cache[b][l] for b in range(len(LENS))] for l in range(m.arch.n_layers)]
        r = oracle.score_dense(m.arch, m.weights, kv, mirror=False)
        away = np.abs(r.p_plus - m.p)
        assert all(away[i] > 10 * P_PLUS_ATOL for i, n in enumerate(LENS) if n), away


def test_readme_bases_agree():
    """README's examples: the cache is rotated with the scorer's base."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "README.md")).read()
    (scorer,) = re.findall(r"Scorer\(L,.*?\)", text)
    base = re.search(r"rope_base=([\d.e]+)", scorer)
    for rope in re.findall(r"Rope\(hd.*?\)", text):
        b = re.search(r"base=([\d.e]+)", rope)
        assert float(b.group(1) if b else 1e4) == float(base.group(1) if base else 1e4), (scorer, rope)


@pytest.mark.gpu
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("base", [1e4, 1e6])
def test_scored(base, e4m3):
    torch = require_gpu()
    import paper_2607_09153_gb300 as kp
    m, a = Model(base), dataclasses.replace(ks.ARCH_TINY, rope_base=base)
    L, nkv, hd = a.n_layers, a.n_kv_heads, a.head_dim
    freq, rope = ref.frequencies(hd, base), kp.Rope(hd, base=base)
    bits = lambda x: torch.from_numpy(np.ascontiguousarray(x).view(np.int16)).cuda().view(torch.bfloat16)  # noqa: E731
    W = m.weights
    top, layers = W["top"], W["layers"]
    names = {"attn_norm": 4, "w_qkv": 5, "w_o": 6, "mlp_norm": 7, "w_gate_up": 8, "w_down": 9}
    scorer = kp.Scorer(L, a.d_model, a.n_q_heads, nkv, hd, a.d_ff,
                       {"embed_verify": bits(top[0]), "final_norm": bits(top[1]), "w_plus": bits(top[2]), "w_minus": bits(top[3]),
                        "layers": [{k: bits(layers[l][i]) for k, i in names.items()} for l in range(L)]},
                       max_candidates=len(LENS), max_blocks_per_seq=7, rope_base=base)
    n_pages = 7 * len(LENS)
    table = np.random.default_rng(5).permutation(n_pages).astype(np.int32).reshape(len(LENS), 7)
    kv = torch.full((L, n_pages, 2, nkv, 16, hd), 3.0, dtype=torch.bfloat16, device="cuda")
    dense = []
    # 8-bit pages: a bf16 number lies half way between two codes once in 16 times, where a rotation in 32 bits decides either
    # way; numbers of full length do not
    away = np.random.default_rng(6)
    source = [[tuple(ks.bf16_bits_to_f64(x) * (1 + (0.01 * away.normal(0, 1, x.shape) if e4m3 else 0)) for x in m.cache[b][l])
               for l in range(L)] for b in range(len(LENS))]
    for l in range(L):
        pages = torch.zeros((n_pages, 2, nkv, 16, hd), device="cuda").to(torch.float8_e4m3fn) if e4m3 else kv[l]
        exps = torch.zeros((n_pages, 2, nkv, 16), dtype=torch.uint8, device="cuda") if e4m3 else None
        for b, n in enumerate(LENS):
            # keys as they were before their rotation, in 64 bits and then the call's 32
            pos = torch.arange(n, dtype=torch.int32, device="cuda")
            k, v = (torch.from_numpy(x).cuda() for x in source[b][l])
            k, v = ref.rotate(k, pos, freq, inverse=True).float(), v.float()
            slots = torch.tensor([16 * int(table[b, i // 16]) + i % 16 for i in range(n)], dtype=torch.int64, device="cuda")
            # a prompt, then one token at a time beside a draft that is not accepted
            cut = max(0, n - 3)
            kp.cache_write(pages, slots[:cut], k[:cut], v[:cut], exps, rope=rope, positions=pos[:cut])
            for i in range(cut, n):
                two = lambda x: torch.cat([x[i:i + 1], 9 * x[i:i + 1]])  # noqa: E731
                kp.cache_write(pages, torch.cat([slots[i:i + 1], slots[:1] * 0 - 1]), two(k), two(v), exps, rope=rope,
                               positions=pos[i:i + 1].repeat(2))
        if e4m3:
            kp.cache_expand(pages, exps, torch.arange(n_pages, dtype=torch.int32, device="cuda"), kv[l])
            values = ref.e4m3_values()
            rows = []
            for b in range(len(LENS)):   # the oracle's cache: each row quantised in 64 bits (exact in bf16)
                pair = []
                for x in source[b][l]:
                    x = torch.from_numpy(x)
                    y = torch.zeros_like(x)
                    for i in range(x.shape[0]):
                        for g in range(nkv):
                            c, e = ref.quantise(x[i, g])
                            y[i, g] = values[c.long()] * 2.0 ** (e - 127)
                    pair.append(ks.f64_to_bf16_bits(y.numpy()))
                rows.append(tuple(pair))
            dense.append(rows)
    p, attn = m.p, m.attn
    if e4m3:
        r = oracle.score_dense(a, W, dense, mirror=False)
        p, attn = r.p_plus, r.attn
    kp.kvprm_set_debug(scorer.ctx, 1)
    got = scorer.score(kv, table, np.array(LENS, dtype=np.int32))
    o = torch.empty((L, len(LENS), a.n_q_heads * hd), dtype=torch.float32, device="cuda")
    kp.kvprm_debug_attn_out(scorer.ctx, o.data_ptr())
    torch.cuda.synchronize()
    assert np.abs(got - p).max() <= P_PLUS_ATOL, (got, p)
    assert attn_rel_err(o.cpu().numpy().astype(np.float64), attn).max() <= ATTN_RTOL
    scorer.close()
