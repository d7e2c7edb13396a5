"""torch face of the operators around the cache (include/kvprm.h): rotary positions, the paged cache written in bf16
or quantised to 8 bits, quantised pages expanded for the scorer, and the attention of drafted tokens over the pages.

Like kvprm.py this module only marshals arguments: shapes, types and devices are checked here, everything else by the
library, and every step runs in its CUDA kernels.  Calls are enqueued on `stream` (default: torch's current one); a
tensor that belongs to another stream has to be ordered by the caller, as for any torch operation.
"""
from __future__ import annotations

import ctypes
import math

from .kvprm import KVPRM_OK, KvprmError
from .kvprm import lib as _base_lib

KVPRM_F32, KVPRM_BF16, KVPRM_F16 = range(3)
KVPRM_CACHE_BF16, KVPRM_CACHE_E4M3 = range(2)
ROPE_SCALINGS = ("none", "linear", "base", "ramp", "smooth")
PAGE = 16


class KvprmRopeConfig(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("scaling", ctypes.c_int32),
                ("original_len", ctypes.c_int32), ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("low", ctypes.c_double), ("high", ctypes.c_double), ("magnitude", ctypes.c_double)]


class KvprmHeads(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n_heads", ctypes.c_int32),
                ("in_token", ctypes.c_int64), ("in_head", ctypes.c_int64), ("out_token", ctypes.c_int64),
                ("out_head", ctypes.c_int64)]


class KvprmCache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("exponents", ctypes.c_void_p), ("n_pages", ctypes.c_int64),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("format", ctypes.c_int32)]


class KvprmTree(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("q", "k", "v", "out")] +
                [(k, ctypes.c_int64) for k in ("q_token", "q_head", "k_token", "k_head", "v_token", "v_head",
                                               "out_token", "out_head")] +
                [(k, ctypes.c_void_p) for k in ("block_table", "lens", "start", "mask")] +
                [(k, ctypes.c_int32) for k in ("max_blocks", "n_seqs", "n_tokens", "n_q_heads", "max_drafts",
                                               "max_len", "mask_words")] +
                [("scale", ctypes.c_float)])


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L = _base_lib()
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        L.kvprm_operator_error.restype = ctypes.c_char_p
        L.kvprm_rope_create.argtypes = [vp, vp]
        L.kvprm_rope_destroy.argtypes = [vp]
        L.kvprm_rope_destroy.restype = None
        L.kvprm_rope_turns.argtypes = [vp, vp]
        L.kvprm_rope_rotate.argtypes = [vp, i32, i32, vp, i64, i32, vp, i32, vp]
        L.kvprm_cache_write.argtypes = [vp, i32, vp, i64, i64, vp, i64, i64, vp, i64, vp, vp, vp]
        L.kvprm_cache_expand.argtypes = [vp, vp, vp, i64, vp, i64, vp]
        L.kvprm_tree_workspace.argtypes = [vp, vp, vp]
        L.kvprm_tree_attention.argtypes = [vp, vp, vp, i64, vp]
        _lib = L
    return _lib


def _check(rc: int) -> None:
    if rc != KVPRM_OK:
        raise KvprmError(rc, lib().kvprm_operator_error().decode())


def _dtype(t) -> int:
    import torch
    code = {torch.float32: KVPRM_F32, torch.bfloat16: KVPRM_BF16, torch.float16: KVPRM_F16}.get(t.dtype)
    if code is None:
        raise TypeError(f"expected float32, bfloat16 or float16, got {t.dtype}")
    return code


def _heads(name: str, t, device, dtype=None) -> None:
    """[tokens][heads][head_dim] on `device`, the elements of a head side by side."""
    if t.dim() != 3 or (t.stride(2) != 1 and t.shape[2] > 1):
        raise ValueError(f"{name} is [tokens][heads][head_dim] with consecutive elements in a head, got "
                         f"{tuple(t.shape)} with strides {tuple(t.stride())}")
    if t.device != device or t.device.type != "cuda":
        raise ValueError(f"{name} is on {t.device}, expected {device} (a CUDA device)")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, expected {dtype}")


def _ints(name: str, t, dtype, shape, device) -> None:
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name} is a contiguous {dtype} tensor of shape {tuple(shape)} on {device}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")


class _on:
    """Makes the tensors' device current for the call (a no-op where it is) and gives the stream's handle."""

    def __init__(self, device, stream):
        import torch
        self.guard = torch.cuda.device(device) if device.index != torch.cuda.current_device() else None
        self.stream = stream if stream is not None else torch.cuda.current_stream(device)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return self.stream.cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


class Rope:
    """Rotary positions of `rotary_dim` elements per head (kvprm_rope_create; see include/kvprm.h for the layouts and
    the ways the frequencies are stretched)."""

    def __init__(self, rotary_dim: int, base: float = 1e4, interleaved: bool = False, scaling: str = "none",
                 factor: float = 1.0, original_len: int = 0, low: float = 1.0, high: float = 32.0,
                 magnitude: float = 1.0):
        if scaling not in ROPE_SCALINGS:
            raise ValueError(f"scaling is one of {ROPE_SCALINGS}, got {scaling!r}")
        self.handle = ctypes.c_void_p()
        self.rotary_dim = int(rotary_dim)
        cfg = KvprmRopeConfig(self.rotary_dim, int(interleaved), ROPE_SCALINGS.index(scaling), int(original_len),
                              float(base), float(factor), float(low), float(high), float(magnitude))
        _check(lib().kvprm_rope_create(ctypes.byref(cfg), ctypes.byref(self.handle)))

    def turns(self) -> list:
        """Per pair, the turns that one position adds, in units of 2^-64."""
        out = (ctypes.c_uint64 * (self.rotary_dim // 2))()
        _check(lib().kvprm_rope_turns(self.handle, out))
        return list(out)

    def rotate(self, positions, *tensors, out=None, stream=None) -> tuple:
        """Each of up to four tensors [tokens][heads][head_dim] (queries, keys) rotated by its tokens' int32
        positions; `out`: tensors to write instead of new ones (the inputs themselves: in place)."""
        return self._run(positions, tensors, out, 0, stream)

    def rotate_backward(self, positions, *grads, out=None, stream=None) -> tuple:
        """The gradients with respect to rotate's inputs from those with respect to its outputs."""
        return self._run(positions, grads, out, 1, stream)

    def _run(self, positions, tensors, out, inverse, stream):
        import torch
        if not 1 <= len(tensors) <= 4:
            raise ValueError(f"1 to 4 tensors, got {len(tensors)}")
        x0 = tensors[0]
        if out is None:
            # the dense layout of the shape, also where the input is a slice of wider rows
            out = tuple(torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in tensors)
        elif len(out) != len(tensors):
            raise ValueError(f"{len(tensors)} tensors and {len(out)} outputs")
        _ints("positions", positions, torch.int32, x0.shape[:1], x0.device)
        rows = (KvprmHeads * len(tensors))()
        for r, t, o in zip(rows, tensors, out):
            _heads("a tensor", t, x0.device, x0.dtype)
            _heads("an output", o, x0.device, x0.dtype)
            if t.shape[0] != x0.shape[0] or t.shape[2] != x0.shape[2] or o.shape != t.shape:
                raise ValueError("the tensors have different tokens or head_dim, or an output another shape")
            r.in_, r.out, r.n_heads = t.data_ptr(), o.data_ptr(), t.shape[1]
            r.in_token, r.in_head, _ = t.stride()
            r.out_token, r.out_head, _ = o.stride()
        with _on(x0.device, stream) as st:
            _check(lib().kvprm_rope_rotate(self.handle, _dtype(x0), x0.shape[2], positions.data_ptr(), x0.shape[0],
                                           inverse, rows, len(tensors), st))
        return tuple(out)

    def __del__(self):
        try:
            if self.handle:
                lib().kvprm_rope_destroy(self.handle)
                self.handle = None
        except Exception:
            pass


def _cache(pages, exponents) -> KvprmCache:
    """One layer's pages [n_pages][2][n_kv_heads][16][head_dim]: bfloat16, or float8_e4m3fn with exponents
    [n_pages][2][n_kv_heads][16] (uint8 or float8_e8m0fnu)."""
    import torch
    if pages.dim() != 5 or pages.shape[1] != 2 or pages.shape[3] != PAGE or not pages.is_contiguous() or \
            pages.device.type != "cuda":
        raise ValueError(f"pages are a contiguous CUDA tensor [n_pages][2][n_kv_heads][16][head_dim], got "
                         f"{tuple(pages.shape)} on {pages.device}")
    if pages.dtype == torch.bfloat16:
        if exponents is not None:
            raise ValueError("bfloat16 pages have no exponents")
        return KvprmCache(pages.data_ptr(), None, pages.shape[0], pages.shape[2], pages.shape[4], KVPRM_CACHE_BF16)
    if pages.dtype != torch.float8_e4m3fn:
        raise TypeError(f"pages are bfloat16 or float8_e4m3fn, got {pages.dtype}")
    if exponents is None or exponents.dtype not in (torch.uint8, torch.float8_e8m0fnu) or \
            exponents.shape != pages.shape[:4] or not exponents.is_contiguous() or exponents.device != pages.device:
        raise ValueError("float8_e4m3fn pages need contiguous uint8 or float8_e8m0fnu exponents "
                         "[n_pages][2][n_kv_heads][16]")
    return KvprmCache(pages.data_ptr(), exponents.data_ptr(), pages.shape[0], pages.shape[2], pages.shape[4],
                      KVPRM_CACHE_E4M3)


def cache_write(pages, slots, k, v, exponents=None, rope: Rope | None = None, positions=None, stream=None) -> None:
    """Writes tokens' keys and values [tokens][n_kv_heads][head_dim] into their slots (int64: 16 * page + place; below
    zero: not written), quantised where the pages are, the keys rotated on the way with `rope` and int32 `positions`."""
    import torch
    c = _cache(pages, exponents)
    for name, t in (("k", k), ("v", v)):
        _heads(name, t, pages.device, k.dtype)
        if tuple(t.shape[1:]) != (c.n_kv_heads, c.head_dim) or t.shape[0] != k.shape[0]:
            raise ValueError(f"{name} is {tuple(t.shape)}, expected [tokens][{c.n_kv_heads}][{c.head_dim}]")
    _ints("slots", slots, torch.int64, k.shape[:1], pages.device)
    if (rope is None) != (positions is None):
        raise ValueError("rope and positions come together")
    if positions is not None:
        _ints("positions", positions, torch.int32, k.shape[:1], pages.device)
    with _on(pages.device, stream) as st:
        _check(lib().kvprm_cache_write(ctypes.byref(c), _dtype(k), k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(),
                                       v.stride(0), v.stride(1), slots.data_ptr(), k.shape[0],
                                       rope.handle if rope is not None else None,
                                       positions.data_ptr() if positions is not None else None, st))


def cache_expand(pages, exponents, src, out, dst=None, stream=None):
    """Quantised pages src[i] as bf16 pages dst[i] (default: i) of `out`, a layer that the scoring calls read; returns
    `out`."""
    import torch
    c = _cache(pages, exponents)
    if out.dtype != torch.bfloat16 or out.dim() != 5 or out.shape[1:] != pages.shape[1:] or not out.is_contiguous() or \
            out.device != pages.device:
        raise ValueError(f"out is a contiguous bfloat16 tensor [pages]{list(pages.shape[1:])} on {pages.device}")
    if dst is None:
        dst = torch.arange(src.shape[0], dtype=torch.int32, device=pages.device)
    _ints("src", src, torch.int32, src.shape[:1], pages.device)
    _ints("dst", dst, torch.int32, src.shape[:1], pages.device)
    with _on(pages.device, stream) as st:
        _check(lib().kvprm_cache_expand(ctypes.byref(c), src.data_ptr(), dst.data_ptr(), src.shape[0], out.data_ptr(),
                                        out.shape[0], st))
    return out


def tree_mask(parents, start):
    """The mask of drafted tokens that form trees: parents[i] is the index, within its sequence, of the parent of
    token i (one before it), or -1 for a child of the cached tokens' end; start [n_seqs + 1] as in tree_attention
    (both host sequences).  Returns a host int32 tensor [tokens][ceil(longest / 32)]: each token sees its ancestors
    and itself."""
    import numpy as np
    import torch
    parents, start = np.asarray(parents, np.int64), np.asarray(start, np.int64)
    longest = int(np.max(np.diff(start), initial=1))
    words = (longest + 31) // 32
    mask = np.zeros((int(start[-1]), words), np.uint32)
    for s0, s1 in zip(start[:-1], start[1:]):
        for i in range(s0, s1):
            p = parents[i]
            if not -1 <= p < i - s0:
                raise ValueError(f"token {i - s0} of its sequence has parent {p}")
            if p >= 0:
                mask[i] = mask[s0 + p]
            mask[i, (i - s0) // 32] |= np.uint32(1 << ((i - s0) % 32))
    return torch.from_numpy(mask.view(np.int32))


_workspaces: dict = {}


def _workspace(need: int, device, stream):
    """Scratch of tree_attention, kept per device and stream: calls on one stream follow one another, so they can
    share it, and each leaves its counters at zero.  A call that is being captured gets scratch of its own (the
    graph's, zeroed by it): the graph may be replayed on any stream."""
    import torch
    if torch.cuda.is_current_stream_capturing():
        with torch.cuda.stream(stream):
            return torch.zeros(need, dtype=torch.uint8, device=device)
    key = (device, stream.cuda_stream)
    w = _workspaces.get(key)
    if w is None or w.numel() < need:
        with torch.cuda.stream(stream):
            w = _workspaces[key] = torch.zeros(need, dtype=torch.uint8, device=device)
    return w


def tree_attention(q, k, v, pages, block_table, lens, start, max_drafts: int, max_len: int | None = None,
                   exponents=None, mask=None, scale: float | None = None, out=None, workspace=None, stream=None):
    """Attention of drafted tokens over their sequences' cached tokens and over each other.

    q [tokens][n_q_heads][head_dim], k and v [tokens][n_kv_heads][head_dim]: bfloat16, rotated; sequence s has the
    drafted tokens start[s] .. start[s + 1] - 1 (int32 [n_seqs + 1], at most max_drafts each) and lens[s] (int32)
    cached ones in pages block_table[s][0 ..] (int32).  mask: int32 [tokens][words], bit j of a token's row: it sees
    drafted token j of its sequence (tree_mask); None: those up to itself.  max_len sizes the launch (default: the
    block table's width).  Returns [tokens][n_q_heads][head_dim]."""
    import torch
    c = _cache(pages, exponents)
    dev = pages.device
    for name, t, heads in (("q", q, q.shape[1]), ("k", k, c.n_kv_heads), ("v", v, c.n_kv_heads)):
        _heads(name, t, dev, torch.bfloat16)
        if t.shape[0] != q.shape[0] or t.shape[1] != heads or t.shape[2] != c.head_dim:
            raise ValueError(f"{name} is {tuple(t.shape)}, expected [{q.shape[0]}][{heads}][{c.head_dim}]")
    n = lens.shape[0]
    if block_table.dim() != 2:
        raise ValueError("block_table is [n_seqs][max_blocks]")
    _ints("block_table", block_table, torch.int32, (n, block_table.shape[1]), dev)
    _ints("lens", lens, torch.int32, (n,), dev)
    _ints("start", start, torch.int32, (n + 1,), dev)
    if mask is not None:
        if mask.dim() != 2:
            raise ValueError("mask is [tokens][words]")
        _ints("mask", mask, torch.int32, (q.shape[0], mask.shape[1]), dev)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=dev)
    else:
        _heads("out", out, dev, torch.bfloat16)
        if out.shape != q.shape:
            raise ValueError(f"out is {tuple(out.shape)}, expected {tuple(q.shape)}")
    t = KvprmTree(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), q.stride(0), q.stride(1), k.stride(0),
                  k.stride(1), v.stride(0), v.stride(1), out.stride(0), out.stride(1), block_table.data_ptr(),
                  lens.data_ptr(), start.data_ptr(), mask.data_ptr() if mask is not None else None,
                  block_table.shape[1], n, q.shape[0], q.shape[1], int(max_drafts),
                  PAGE * block_table.shape[1] if max_len is None else int(max_len),
                  mask.shape[1] if mask is not None else 0,
                  1.0 / math.sqrt(c.head_dim) if scale is None else float(scale))
    on = _on(dev, stream)
    with on as st:
        if workspace is None:
            need = ctypes.c_int64()
            _check(lib().kvprm_tree_workspace(ctypes.byref(c), ctypes.byref(t), ctypes.byref(need)))
            workspace = _workspace(need.value, dev, on.stream)
        _check(lib().kvprm_tree_attention(ctypes.byref(c), ctypes.byref(t), workspace.data_ptr(), workspace.numel(), st))
    return out
