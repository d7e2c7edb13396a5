"""Host side of the operators around the cache: the rotary table, tree masks, and what the library refuses before it
touches a device."""
import ctypes
import math
from fractions import Fraction

import pytest

import paper_2607_09153_gb300 as kp
from paper_2607_09153_gb300 import operators as ops
from tests import operators_util as ref


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("base", 2.0), ("ramp", 8.0),
                                            ("smooth", 7.5)])
@pytest.mark.parametrize("rd", [2, 32, 64, 98, 128, 256])
def test_turns(rd, scaling, factor):
    if scaling == "base" and rd == 2:
        pytest.skip("refused")
    r = kp.Rope(rd, base=5e5, scaling=scaling, factor=factor, original_len=8192, low=1.0, high=4.0)
    want = ref.frequencies(rd, 5e5, scaling, factor, 8192, 1.0, 4.0)
    for t, f in zip(r.turns(), want.tolist()):
        # both are 64-bit floating point computations of a few steps; the table's unit is 2^-64
        want = Fraction(f / (2 * math.pi)) * 2 ** 64
        assert abs(t - want) <= 1 + want * Fraction(1e-13)


def test_stretched_frequencies_are_between():
    """Every way of stretching leaves a frequency between the original and its factor-th part, and keeps the order."""
    plain = kp.Rope(128).turns()
    for scaling in ("linear", "base", "ramp", "smooth"):
        t = kp.Rope(128, scaling=scaling, factor=4.0, original_len=4096).turns()
        assert all(a >= b >= a // 4 - 1 for a, b in zip(plain, t)), scaling
        assert all(a > b for a, b in zip(t, t[1:])), scaling
    for scaling in ("ramp", "smooth"):
        t = kp.Rope(128, scaling=scaling, factor=4.0, original_len=4096).turns()
        assert t[0] == plain[0] and abs(t[-1] - plain[-1] / 4) <= 2


@pytest.mark.parametrize("bad", [dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=258), dict(base=1.0),
                                 dict(base=math.nan), dict(base=math.inf), dict(scaling="linear", factor=0.5),
                                 dict(scaling="linear", factor=math.nan), dict(scaling="base", rotary_dim=2),
                                 dict(scaling="ramp", original_len=0), dict(scaling="ramp", original_len=9, low=0.0),
                                 dict(scaling="smooth", original_len=9, low=4.0, high=4.0),
                                 dict(magnitude=math.inf)])
def test_rope_refusals(bad):
    with pytest.raises(kp.KvprmError) as e:
        kp.Rope(**{"rotary_dim": 64, **bad})
    assert e.value.code == kp.KVPRM_EINVAL and "kvprm_rope_create" in str(e.value)


def test_unknown_scaling():
    with pytest.raises(ValueError):
        kp.Rope(64, scaling="other")


def test_tree_mask():
    #        0 -> 1 -> 3,  0 -> 2 ; a second root 4; another sequence of one
    m = kp.tree_mask([-1, 0, 0, 1, -1, -1], [0, 5, 6])
    assert m[:, 0].tolist() == [0b1, 0b11, 0b101, 0b1011, 0b10000, 0b1]
    chain = kp.tree_mask([-1] + list(range(39)), [0, 40])
    assert chain.shape == (40, 2) and chain[39].tolist() == [-1, 0xFF] and chain[31].tolist() == [-1, 0]
    for parents in ([0], [-1, 1], [-2]):
        with pytest.raises(ValueError):
            kp.tree_mask(parents, [0, len(parents)])


# ---------------------------------------------------------------- refusals: addresses that nothing reads
P = 0x10000


def _cache(**kw):
    d = dict(pages=P, exponents=None, n_pages=8, n_kv_heads=2, head_dim=64, format=kp.KVPRM_CACHE_BF16)
    d.update(kw)
    return ops.KvprmCache(*[d[k] for k, _ in ops.KvprmCache._fields_])


def _refused(rc, code=kp.KVPRM_EINVAL):
    assert rc == code
    assert kp.lib().kvprm_operator_error()


BAD_CACHES = [dict(head_dim=96), dict(head_dim=0), dict(n_kv_heads=0), dict(n_pages=-1), dict(pages=None),
              dict(pages=P + 8), dict(format=2), dict(format=kp.KVPRM_CACHE_E4M3),
              dict(format=kp.KVPRM_CACHE_E4M3, exponents=P + 4)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_cache_refusals(bad):
    L, c = ops.lib(), _cache(**bad)
    _refused(L.kvprm_cache_write(ctypes.byref(c), kp.KVPRM_BF16, P, 128, 64, P, 128, 64, P, 1, None, None, None))
    t = _tree()
    n = ctypes.c_int64()
    _refused(L.kvprm_tree_workspace(ctypes.byref(c), ctypes.byref(t), ctypes.byref(n)))
    _refused(L.kvprm_tree_attention(ctypes.byref(c), ctypes.byref(t), P, 1 << 30, None))
    _refused(L.kvprm_cache_expand(ctypes.byref(c), P, P, 1, P, 8, None))


def test_write_refusals():
    L, c = ops.lib(), _cache()
    r = kp.Rope(128)   # more than the cache's head_dim
    half = kp.Rope(32)
    w = lambda dtype=kp.KVPRM_BF16, k=P, v=P, slots=P, n=1, rope=None, pos=None: L.kvprm_cache_write(  # noqa: E731
        ctypes.byref(c), dtype, k, 128, 64, v, 128, 64, slots, n, rope, pos, None)
    for rc in (w(dtype=3), w(k=None), w(v=None), w(slots=None), w(n=-1), w(k=P + 1), w(slots=P + 4), w(rope=half.handle),
               w(pos=P), w(rope=r.handle, pos=P),
               L.kvprm_cache_write(None, kp.KVPRM_BF16, P, 128, 64, P, 128, 64, P, 1, None, None, None)):
        _refused(rc)
    assert w(n=0) == kp.KVPRM_OK


def test_rotate_refusals():
    L, r = ops.lib(), kp.Rope(64)

    def go(handle=r.handle, dtype=kp.KVPRM_F32, hd=64, pos=P, n=1, inverse=0, n_x=1, **row):
        d = dict(in_=P, out=P, n_heads=2, in_token=128, in_head=64, out_token=128, out_head=64)
        d.update(row)
        rows = (ops.KvprmHeads * 5)(*[ops.KvprmHeads(*[d[k] for k, _ in ops.KvprmHeads._fields_]) for _ in range(5)])
        return L.kvprm_rope_rotate(handle, dtype, hd, pos, n, inverse, rows, n_x, None)

    for rc in (go(handle=None), go(dtype=9), go(hd=32), go(hd=1024), go(pos=None), go(n=-1), go(inverse=2), go(n_x=0),
               go(n_x=5), go(in_=None), go(out=None), go(n_heads=-1), go(n_heads=1025), go(n_heads=600, n_x=2),
               go(in_=P + 2)):
        _refused(rc)
    assert go(n=0) == kp.KVPRM_OK and go(n_heads=0) == kp.KVPRM_OK


def test_expand_refusals():
    L, c = ops.lib(), _cache(format=kp.KVPRM_CACHE_E4M3, exponents=P)
    e = lambda src=P, dst=P, n=1, out=P, pages=8: L.kvprm_cache_expand(ctypes.byref(c), src, dst, n, out, pages, None)  # noqa: E731
    for rc in (e(src=None), e(dst=None), e(n=-1), e(out=None), e(out=P + 2), e(pages=-1)):
        _refused(rc)
    assert e(n=0) == kp.KVPRM_OK
    plain = _cache()
    _refused(L.kvprm_cache_expand(ctypes.byref(plain), P, P, 1, P, 8, None))


def _tree(**kw):
    d = dict(q=P, k=P, v=P, out=P, q_token=256, q_head=64, k_token=128, k_head=64, v_token=128, v_head=64,
             out_token=256, out_head=64, block_table=P, lens=P, start=P, mask=P, max_blocks=4, n_seqs=2, n_tokens=4,
             n_q_heads=4, max_drafts=33, max_len=64, mask_words=2, scale=0.125)
    d.update(kw)
    return ops.KvprmTree(*[d[k] for k, _ in ops.KvprmTree._fields_])


@pytest.mark.parametrize("bad", [dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(block_table=None),
                                 dict(lens=None), dict(start=None), dict(q=P + 8), dict(out=P + 2), dict(k_token=130),
                                 dict(q_head=60), dict(n_seqs=-1), dict(n_tokens=-1), dict(max_blocks=-1),
                                 dict(max_len=-1), dict(n_q_heads=3), dict(n_q_heads=0), dict(n_q_heads=2048),
                                 dict(max_drafts=0), dict(max_drafts=1025), dict(mask_words=1),
                                 dict(scale=math.nan), dict(scale=math.inf)])
def test_tree_refusals(bad):
    c, t = _cache(), _tree(**bad)
    _refused(ops.lib().kvprm_tree_attention(ctypes.byref(c), ctypes.byref(t), P, 1 << 30, None))


def test_tree_nothing_to_do():
    c = _cache()
    for kw in (dict(n_seqs=0), dict(n_tokens=0)):
        t = _tree(**kw)
        assert ops.lib().kvprm_tree_attention(ctypes.byref(c), ctypes.byref(t), None, 0, None) == kp.KVPRM_OK
