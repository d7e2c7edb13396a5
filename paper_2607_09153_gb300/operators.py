"""torch face of the operators around the cache (include/kvprm.h): rotary positions, the paged cache written in bf16
or quantised to 8 bits, quantised pages expanded for the scorer, and the attention of drafted tokens over the pages.

Like kvprm.py this module only marshals arguments: shapes, types and devices are checked here, everything else by the
library, and every step runs in its CUDA kernels.  Calls are enqueued on `stream` (default: torch's current one), and the
tensors that they return belong to it; a tensor that belongs to another stream has to be ordered by the caller, as for
any torch operation.

A decoding step's calls take a few microseconds on the GPU, so what is spent here counts: arguments are read once, and
the C structs are packed as bytes (a ctypes structure takes about 0.2 us a field).
"""
from __future__ import annotations

import ctypes
import math
import struct
import threading

from .kvprm import KVPRM_ECAPACITY, KVPRM_OK, KvprmError
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
        L.kvprm_tree_attention.argtypes = L.kvprm_tree_attention_filled.argtypes = [vp, vp, vp, i64, vp]
        _lib = L
    return _lib


def _check(rc: int) -> None:
    if rc != KVPRM_OK:
        raise KvprmError(rc, lib().kvprm_operator_error().decode())


class _Torch:
    """What the calls need of torch, looked up once (the package imports without it)."""

    def __init__(self):
        import torch
        self.torch = torch
        self.codes = {torch.float32: KVPRM_F32, torch.bfloat16: KVPRM_BF16, torch.float16: KVPRM_F16}
        self.bf16, self.i32, self.i64 = torch.bfloat16, torch.int32, torch.int64
        self.e4m3, self.bytes = torch.float8_e4m3fn, (torch.uint8, torch.float8_e8m0fnu)
        self.raw_stream = torch._C._cuda_getCurrentRawStream   # the handle alone: 0.1 us against 2 us for the object
        self.device = torch._C._cuda_getDevice                  # the calls' tensors have initialised CUDA
        self.capturing = torch.cuda.is_current_stream_capturing
        self.empty = torch.empty   # 1.8 us; Tensor.new_empty takes 3.3
        self.grad_enabled = torch.is_grad_enabled
        self.rotation, self.attention = _functions(torch)


def _functions(torch):
    """What autograd is told of the calls: the rotation's gradient, and that the attention has none."""

    class Rotation(torch.autograd.Function):
        @staticmethod
        def forward(ctx, rope, positions, inverse, *tensors):
            ctx.rope, ctx.inverse = rope, inverse
            ctx.save_for_backward(positions)
            out = rope._run(positions, tensors, None, inverse, None)
            ctx.mark_non_differentiable(*[o for o, need in zip(out, ctx.needs_input_grad[3:]) if not need])
            return out

        @staticmethod
        def backward(ctx, *grads):
            (positions,) = ctx.saved_tensors
            need = [i for i, n in enumerate(ctx.needs_input_grad[3:]) if n]
            dense = [g if g.stride(2) == 1 else g.contiguous() for g in (grads[i] for i in need)]
            result = [None] * (3 + len(grads))
            for i, g in zip(need, ctx.rope._run(positions, dense, None, 1 - ctx.inverse, None)):
                result[3 + i] = g
            return tuple(result)

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, call, *tensors):
            return call()

        @staticmethod
        def backward(ctx, grad):
            raise RuntimeError("tree_attention has no gradient: call it under torch.no_grad(), or on detached tensors")

    return Rotation, Attention


_t = None


def _torch() -> _Torch:
    global _t
    if _t is None:
        _t = _Torch()
    return _t


# struct layouts of the C ABI (the trailing 0q pads to the alignment, as C does)
_HEADS = struct.Struct("@PPiqqqq")
_CACHE = struct.Struct("@PPqiii0q")
_TREE = struct.Struct("@PPPPqqqqqqqqPPPPiiiiiiif0q")
assert _HEADS.size == ctypes.sizeof(KvprmHeads) and _CACHE.size == ctypes.sizeof(KvprmCache)
assert _TREE.size == ctypes.sizeof(KvprmTree)


def _heads(name: str, t, shape, dtype, device: int) -> tuple:
    """Strides (token, head) of a tensor [tokens][heads][head_dim] whose heads' elements are side by side."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        if t.dtype is not dtype:
            raise TypeError(f"{name} is {t.dtype}, expected {dtype}")
        raise ValueError(f"{name} is {tuple(t.shape)} on {t.device}, expected {tuple(shape)} on CUDA device {device}")
    st = t.stride()
    if st[2] != 1 and shape[2] > 1 and t.numel() > 0:
        raise ValueError(f"the elements of a head of {name} are not side by side: strides {st}")
    return st


def _rows(name: str, t) -> tuple:
    """(shape, device index) of the tensor that the others of a call are compared with."""
    shape, device = t.shape, t.get_device()
    if len(shape) != 3 or device < 0:
        raise ValueError(f"{name} is a CUDA tensor [tokens][heads][head_dim], got {tuple(shape)} on {t.device}")
    return shape, device


def _ints(name: str, t, dtype, shape: tuple, device: int) -> int:
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name} is a contiguous {dtype} tensor of shape {tuple(shape)} on CUDA device {device}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _call(T, device: int, stream, function, *args) -> int:
    """function(*args, stream handle) with the tensors' device current; the status."""
    handle = T.raw_stream(device) if stream is None else stream.cuda_stream
    if T.device() == device:
        return function(*args, handle)
    with T.torch.cuda.device(device):
        return function(*args, handle)


def _result(T, shape, dtype, device, stream):
    """A tensor of the stream that the call writes it on (one of another stream might still be in use there)."""
    with T.torch.cuda.stream(stream):
        return T.empty(shape, dtype=dtype, device=device)


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
        L = lib()
        self._rotate = L.kvprm_rope_rotate
        _check(L.kvprm_rope_create(ctypes.byref(cfg), ctypes.byref(self.handle)))

    def turns(self) -> list:
        """Per pair, the turns that one position adds, in units of 2^-64."""
        out = (ctypes.c_uint64 * (self.rotary_dim // 2))()
        _check(lib().kvprm_rope_turns(self.handle, out))
        return list(out)

    def rotate(self, positions, *tensors, out=None, stream=None) -> tuple:
        """Each of up to four tensors [tokens][heads][head_dim] (queries, keys) rotated by its tokens' int32
        positions; `out`: tensors to write instead of new ones (the inputs themselves: in place).  Differentiable."""
        return self._run(positions, tensors, out, 0, stream)

    def rotate_backward(self, positions, *grads, out=None, stream=None) -> tuple:
        """The gradients with respect to rotate's inputs from those with respect to its outputs."""
        return self._run(positions, grads, out, 1, stream)

    def _run(self, positions, tensors, out, inverse, stream):
        T = _t or _torch()
        if not 1 <= len(tensors) <= 4:
            raise ValueError(f"1 to 4 tensors, got {len(tensors)}")
        x0 = tensors[0]
        (n, _, hd), dev = _rows("a tensor", x0)
        dtype = x0.dtype
        code = T.codes.get(dtype)
        if code is None:
            raise TypeError(f"expected float32, bfloat16 or float16, got {dtype}")
        if out is not None and len(out) != len(tensors):
            raise ValueError(f"{len(tensors)} tensors and {len(out)} outputs")
        result, packed = [], b""
        for i, x in enumerate(tensors):
            shape = x.shape
            if len(shape) != 3 or shape[0] != n or shape[2] != hd:
                raise ValueError(f"a tensor is {tuple(shape)}, expected [{n}][heads][{hd}]")
            if x.requires_grad and T.grad_enabled():
                return self._differentiable(T, positions, tensors, out, inverse, stream)
            st = _heads("a tensor", x, shape, dtype, dev)
            if out is None:   # dense, also where x is a slice of wider rows
                o = T.empty(shape, dtype=dtype, device=x.device) if stream is None else _result(T, shape, dtype, x.device, stream)
                so = (shape[1] * hd, hd)
            else:
                o = out[i]
                so = _heads("an output", o, shape, dtype, dev)
            result.append(o)
            packed += _HEADS.pack(x.data_ptr(), o.data_ptr(), shape[1], st[0], st[1], so[0], so[1])
        at = _ints("positions", positions, T.i32, (n,), dev)
        rc = _call(T, dev, stream, self._rotate, self.handle, code, hd, at, n, inverse, packed, len(result))
        if rc != KVPRM_OK:
            _check(rc)
        return tuple(result)

    def _differentiable(self, T, positions, tensors, out, inverse, stream):
        if out is not None:
            raise ValueError("out= has no gradient: leave it away, or call under torch.no_grad()")
        with T.torch.cuda.stream(stream):   # (autograd orders the backward pass by the current stream)
            return T.rotation.apply(self, positions, inverse, *tensors)

    def __del__(self):
        try:
            if self.handle:
                lib().kvprm_rope_destroy(self.handle)
                self.handle = None
        except Exception:
            pass


def _cache(T, pages, exponents) -> tuple:
    """(C struct, kv heads, head_dim, device index) of one layer's pages [n_pages][2][n_kv_heads][16][head_dim]:
    bfloat16, or float8_e4m3fn with exponents [n_pages][2][n_kv_heads][16] (uint8 or float8_e8m0fnu)."""
    shape, device = pages.shape, pages.get_device()
    if len(shape) != 5 or shape[1] != 2 or shape[3] != PAGE or device < 0 or not pages.is_contiguous():
        raise ValueError(f"pages are a contiguous CUDA tensor [n_pages][2][n_kv_heads][16][head_dim], got "
                         f"{tuple(shape)} on {pages.device}")
    if pages.dtype is T.bf16:
        if exponents is not None:
            raise ValueError("bfloat16 pages have no exponents")
        return _CACHE.pack(pages.data_ptr(), 0, shape[0], shape[2], shape[4], KVPRM_CACHE_BF16), shape[2], shape[4], device
    if pages.dtype is not T.e4m3:
        raise TypeError(f"pages are bfloat16 or float8_e4m3fn, got {pages.dtype}")
    if exponents is None or exponents.dtype not in T.bytes or exponents.shape != shape[:4] or \
            exponents.get_device() != device or not exponents.is_contiguous():
        raise ValueError("float8_e4m3fn pages need contiguous uint8 or float8_e8m0fnu exponents "
                         "[n_pages][2][n_kv_heads][16]")
    return (_CACHE.pack(pages.data_ptr(), exponents.data_ptr(), shape[0], shape[2], shape[4], KVPRM_CACHE_E4M3),
            shape[2], shape[4], device)


def cache_write(pages, slots, k, v, exponents=None, rope: Rope | None = None, positions=None, stream=None) -> None:
    """Writes tokens' keys and values [tokens][n_kv_heads][head_dim] into their slots (int64: 16 * page + place; below
    zero: not written; one token each), quantised where the pages are, the keys rotated on the way with `rope` and int32
    `positions`.  No gradient passes through the pages."""
    T = _t or _torch()
    c, heads, hd, dev = _cache(T, pages, exponents)
    n, dtype = k.shape[0], k.dtype
    code = T.codes.get(dtype)
    if code is None:
        raise TypeError(f"k is {dtype}, expected float32, bfloat16 or float16")
    sk, sv = _heads("k", k, (n, heads, hd), dtype, dev), _heads("v", v, (n, heads, hd), dtype, dev)
    if (rope is None) != (positions is None):
        raise ValueError("rope and positions come together")
    handle = at = None
    if rope is not None:
        handle, at = rope.handle, _ints("positions", positions, T.i32, (n,), dev)
    rc = _call(T, dev, stream, lib().kvprm_cache_write, c, code, k.data_ptr(), sk[0], sk[1], v.data_ptr(), sv[0], sv[1],
               _ints("slots", slots, T.i64, (n,), dev), n, handle, at)
    if rc != KVPRM_OK:
        _check(rc)


def cache_expand(pages, exponents, src, out, dst=None, stream=None):
    """Quantised pages src[i] (int32) as bf16 pages dst[i] (int32, none twice; default: i) of `out`, a layer that the
    scoring calls read; returns `out`."""
    T = _t or _torch()
    c, _, _, dev = _cache(T, pages, exponents)
    shape = out.shape
    if out.dtype is not T.bf16 or len(shape) != 5 or shape[1:] != pages.shape[1:] or out.get_device() != dev or \
            not out.is_contiguous():
        raise ValueError(f"out is a contiguous bfloat16 tensor [pages]{list(pages.shape[1:])} on {pages.device}")
    n = src.shape[0]
    if dst is None:
        with T.torch.cuda.stream(stream):
            dst = T.torch.arange(n, dtype=T.i32, device=out.device)
    rc = _call(T, dev, stream, lib().kvprm_cache_expand, c, _ints("src", src, T.i32, (n,), dev),
               _ints("dst", dst, T.i32, (n,), dev), n, out.data_ptr(), shape[0])
    if rc != KVPRM_OK:
        _check(rc)
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


class _Stream:
    """Scratch of the calls on one stream.  They follow one another there, so they can share it; `lock` is held while one
    of them enqueues its launches, for those of two host threads must not be mixed."""
    __slots__ = ("lock", "scratch", "address", "bytes")

    def __init__(self):
        self.lock, self.scratch, self.address, self.bytes = threading.RLock(), None, 0, 0


_streams: dict = {}   # by device and stream handle


def _scratch(T, need: int, device: int, stream):
    with T.torch.cuda.stream(stream):   # (None: the current one)
        return T.torch.empty(need, dtype=T.torch.uint8, device=T.torch.device("cuda", device))


def _workspace_bytes(c: bytes, t: bytes) -> int:
    need = ctypes.c_int64()
    _check(lib().kvprm_tree_workspace(c, t, ctypes.byref(need)))
    return need.value


def _attend(T, go, c: bytes, t: bytes, device: int, stream) -> int:
    """`go`, an attention entry point, with scratch of the stream's, the tensors' device being current; the status."""
    if stream is None:
        handle, capturing = T.raw_stream(device), T.capturing()
    else:
        handle = stream.cuda_stream
        with T.torch.cuda.stream(stream):
            capturing = T.capturing()
    if capturing:   # scratch of the graph's own, for the graph may be replayed on any stream
        w = _scratch(T, _workspace_bytes(c, t), device, stream)
        return go(c, t, w.data_ptr(), w.numel(), handle)
    key = (device, handle)
    mine = _streams.get(key) or _streams.setdefault(key, _Stream())
    with mine.lock:
        rc = go(c, t, mine.address, mine.bytes, handle) if mine.bytes else KVPRM_ECAPACITY
        if rc == KVPRM_ECAPACITY:
            w = mine.scratch = _scratch(T, _workspace_bytes(c, t), device, stream)
            mine.address, mine.bytes = w.data_ptr(), w.numel()
            rc = go(c, t, mine.address, mine.bytes, handle)
    return rc


def _attend_without_gradient(T, args):
    """tree_attention(*args) on tensors that require gradients."""
    *_, out, _, stream = args
    if out is not None:
        raise ValueError("out= has no gradient: call under torch.no_grad()")
    with T.torch.cuda.stream(stream):
        return T.attention.apply(lambda: tree_attention(*args), *args[:4])


def tree_attention(q, k, v, pages, block_table, lens, start, max_drafts: int, max_len: int | None = None,
                   exponents=None, mask=None, scale: float | None = None, out=None, workspace=None, stream=None):
    """Attention of drafted tokens over their sequences' cached tokens and over each other.

    q [tokens][n_q_heads][head_dim], k and v [tokens][n_kv_heads][head_dim]: bfloat16, rotated; sequence s has the
    drafted tokens start[s] .. start[s + 1] - 1 (int32 [n_seqs + 1], at most max_drafts each) and lens[s] (int32)
    cached ones in pages block_table[s][0 ..] (int32).  mask: int32 [tokens][words], bit j of a token's row: it sees
    drafted token j of its sequence (tree_mask); None: those up to itself.  max_len sizes the launch (default: the
    block table's width).  Returns [tokens][n_q_heads][head_dim]: `out`, where rows of tokens that no sequence has, or one
    with more than max_drafts, are left as they are, or a new tensor, where they are zeros and NaN.  There is no gradient: a
    backward pass that reaches the call raises.  Scratch is kept for each stream, as large as its largest call wanted;
    workspace: a contiguous tensor to use instead (one that is too small is refused with the bytes that are needed)."""
    T = _t or _torch()
    if (q.requires_grad or k.requires_grad or v.requires_grad or pages.requires_grad) and T.grad_enabled():
        return _attend_without_gradient(T, (q, k, v, pages, block_table, lens, start, max_drafts, max_len, exponents, mask, scale,
                                            out, workspace, stream))
    c, heads, hd, dev = _cache(T, pages, exponents)
    shape, _ = _rows("q", q)
    tokens, nq, _ = shape
    bf16, i32 = T.bf16, T.i32
    sq = _heads("q", q, (tokens, nq, hd), bf16, dev)
    sk, sv = _heads("k", k, (tokens, heads, hd), bf16, dev), _heads("v", v, (tokens, heads, hd), bf16, dev)
    n = lens.shape[0]
    if block_table.dim() != 2:
        raise ValueError("block_table is [n_seqs][max_blocks]")
    width = block_table.shape[1]
    bits, words = 0, 0
    if mask is not None:
        if mask.dim() != 2:
            raise ValueError("mask is [tokens][words]")
        words = mask.shape[1]
        bits = _ints("mask", mask, i32, (tokens, words), dev)
    if out is None:
        out = T.empty(shape, dtype=bf16, device=q.device) if stream is None else _result(T, shape, bf16, q.device, stream)
        so = (nq * hd, hd)
        go = lib().kvprm_tree_attention_filled
    else:
        so = _heads("out", out, shape, bf16, dev)
        go = lib().kvprm_tree_attention
    t = _TREE.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), sq[0], sq[1], sk[0], sk[1], sv[0], sv[1],
                   so[0], so[1], _ints("block_table", block_table, i32, (n, width), dev),
                   _ints("lens", lens, i32, (n,), dev), _ints("start", start, i32, (n + 1,), dev), bits, width, n,
                   tokens, nq, max_drafts, PAGE * width if max_len is None else max_len, words,
                   1.0 / math.sqrt(hd) if scale is None else scale)
    if workspace is not None:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace is a contiguous tensor on CUDA device {dev}, got one on {workspace.device}")
        rc = _call(T, dev, stream, go, c, t, workspace.data_ptr(),
                   workspace.numel() * workspace.element_size())
    elif T.device() == dev:
        rc = _attend(T, go, c, t, dev, stream)
    else:
        with T.torch.cuda.device(dev):
            rc = _attend(T, go, c, t, dev, stream)
    if rc != KVPRM_OK:
        _check(rc)
    return out
