"""cache_fork and cache_compact where no GPU is needed: the definition that the GPU tests compare with (tests/cache4_util.py) keeps
what sequences hold, and the library refuses what the host can see, before anything is enqueued."""
import ctypes
import random

import pytest

import paper_2607_09153_gb300 as kp
from paper_2607_09153_gb300 import operators as ops
from tests.cache4_util import Pool


@pytest.mark.parametrize("seed", range(20))
def test_definition_keeps_what_sequences_hold(seed):
    """Over random steps of a search every sequence's tokens are what its ancestors wrote, whoever else wrote since; references are
    the tables' own; nothing is lost or held twice."""
    rng = random.Random(seed)
    n_pages, width = rng.choice([40, 80]), 12
    content = {}                                   # slot -> token
    pool, held = Pool([0] * n_pages, [], []), []   # held: each sequence's tokens
    others = rng.sample(range(n_pages), 4)
    for p in others:
        pool.refs[p] = 1
    for step in range(8):
        n = len(held)
        parents = [rng.randrange(-1, n) if n else -1 for _ in range(rng.randint(1, 5))]
        room = [rng.randint(0, 40) if p < 0 or len(held[p]) < 100 else 0 for p in parents]
        table, lens, refs, counts, copies = pool.fork(parents, room, width)
        for a, b in copies:
            for i in range(16):
                content[16 * b + i] = content.get(16 * a + i)
        pool = Pool(refs, table, lens)
        held = [list(held[p]) if p >= 0 else [] for p in parents]
        counted = [0] * n_pages
        for p in others:
            counted[p] += 1
        for s, row in enumerate(table):
            for p in row:
                if p >= 0:
                    counted[p] += 1
            for t in range(room[s]):               # write the step
                at = len(held[s])
                if at // 16 < width and row[at // 16] >= 0:
                    content[16 * row[at // 16] + at % 16] = (step, s, t)
                    held[s].append((step, s, t))
                    pool.lens[s] += 1
                else:
                    break
        assert counted == refs and counts[0] == sum(r == 0 for r in refs)
        for s, tokens in enumerate(held):
            if all(p >= 0 for p in pool.table[s][:-(-len(tokens) // 16)]):   # (a copy that was not to be had aside)
                assert [content[16 * pool.table[s][i // 16] + i % 16] for i in range(len(tokens))] == tokens
    table, refs, moved, (live, moves), copies = pool.compact()
    assert sorted(refs, reverse=True)[:live] == sorted((r for r in pool.refs if r > 0), reverse=True)
    assert all(r > 0 for r in refs[:live]) and not any(refs[live:]) and len(copies) == moves
    assert not {a for a, _ in copies} & {b for _, b in copies}


def _arrays():
    """Host memory in the place of device memory: nothing is launched by a call that is refused."""
    return {k: (ctypes.c_int32 * 256)() for k in ("refs", "block_table", "lens", "parents", "room", "refs_out", "table_out", "lens_out",
                                                  "moved", "counts")}


def _fork(arrays, pools=(), workspace=1 << 20, **kw):
    f = ops.KvprmFork()
    for k in ("refs", "block_table", "lens", "parents", "room", "refs_out", "table_out", "lens_out", "counts"):
        setattr(f, k, ctypes.addressof(arrays[k]))
    f.n_pages, f.n_pools, f.n_seqs, f.max_blocks, f.n_new, f.width = 16, len(pools), 3, 4, 5, 6
    for k, v in kw.items():
        setattr(f, k, v)
    packed = (ops.KvprmPool * max(1, len(pools)))(*pools)
    return ops.lib().kvprm_cache_fork(packed, ctypes.byref(f), None if workspace is None else 256, workspace or 0, None)


def _compact(arrays, pools=(), workspace=1 << 20, **kw):
    f = ops.KvprmCompact()
    for k in ("refs", "block_table", "lens", "refs_out", "table_out", "moved", "counts"):
        setattr(f, k, ctypes.addressof(arrays[k]))
    f.n_pages, f.n_pools, f.n_seqs, f.max_blocks = 16, len(pools), 3, 4
    for k, v in kw.items():
        setattr(f, k, v)
    packed = (ops.KvprmPool * max(1, len(pools)))(*pools)
    return ops.lib().kvprm_cache_compact(packed, ctypes.byref(f), None if workspace is None else 256, workspace or 0, None)


@pytest.mark.parametrize("call", [_fork, _compact])
def test_refusals(call):
    x = _arrays()
    at = {k: ctypes.addressof(v) for k, v in x.items()}
    error = lambda: ops.lib().kvprm_operator_error().decode()  # noqa: E731
    for kw in (dict(n_pages=-1), dict(n_pages=(1 << 30) + 1), dict(n_seqs=-1), dict(max_blocks=-1), dict(n_pools=-1), dict(n_pools=97),
               dict(n_seqs=8193), dict(max_blocks=(1 << 24) + 1), dict(refs=None), dict(lens=None), dict(refs_out=None), dict(counts=None),
               dict(refs=at["refs"] + 2), dict(table_out=at["table_out"] + 1),
               dict(refs_out=at["refs"]), dict(refs_out=at["refs"] + 4 * 15), dict(table_out=at["block_table"] + 4), dict(counts=at["lens"] + 8),
               dict(refs_out=at["table_out"] + 8)):
        assert call(x, **kw) == kp.KVPRM_EINVAL, kw
        assert error().startswith("kvprm_cache_" + call.__name__[1:]), error()
    base = ctypes.addressof(x["moved"]) // 16 * 16 + 16
    pool = lambda **kw: ops.KvprmPool(**{**dict(base=base, layer_stride=256, page_stride=16, page_bytes=16, layers=1), **kw})  # noqa: E731
    for kw in (dict(base=None), dict(base=base + 8), dict(layer_stride=8), dict(page_stride=24), dict(page_bytes=20), dict(page_bytes=-16),
               dict(layers=-1), dict(page_bytes=1 << 31)):
        assert call(x, [pool(), pool(**kw)]) == kp.KVPRM_EINVAL, kw
    assert call(x, [pool(layers=1 << 30, page_bytes=1 << 20)]) == kp.KVPRM_EINVAL
    assert call(x, workspace=None) == kp.KVPRM_EINVAL
    assert call(x, workspace=512) == kp.KVPRM_ECAPACITY and "needed" in error()


def test_fork_refusals():
    x = _arrays()
    for kw in (dict(n_new=-1), dict(width=-1), dict(n_new=8193), dict(width=(1 << 24) + 1), dict(n_new=8000, width=1 << 18), dict(parents=None),
               dict(lens_out=None), dict(room=ctypes.addressof(x["refs_out"])), dict(parents=ctypes.addressof(x["lens_out"]) + 16)):
        assert _fork(x, **kw) == kp.KVPRM_EINVAL, kw


def test_workspaces():
    need, f, c = ctypes.c_int64(), ops.KvprmFork(), ops.KvprmCompact()
    L = ops.lib()
    for n in (0, 1, 1000, 1 << 20):
        f.n_pages = c.n_pages = n
        f.n_new = min(n, 8192)
        assert L.kvprm_fork_workspace(None, ctypes.byref(f), ctypes.byref(need)) == kp.KVPRM_OK and need.value >= 8 * n + 24 * f.n_new
        assert L.kvprm_compact_workspace(None, ctypes.byref(c), ctypes.byref(need)) == kp.KVPRM_OK and need.value >= 16 * n
    assert L.kvprm_fork_workspace(None, None, ctypes.byref(need)) == kp.KVPRM_EINVAL
    assert L.kvprm_compact_workspace(None, ctypes.byref(c), None) == kp.KVPRM_EINVAL
