"""What the operators' torch face asks of torch and hands to the library, with both replaced by stand-ins that keep a record:
which stream a tensor is made on, who holds scratch when.  (No GPU.)"""
import contextlib
import itertools
import threading
import time

import pytest
import torch

from paper_2607_09153_gb300 import operators as ops


class Tensor:
    """As much of a contiguous CUDA tensor as the calls look at."""
    addresses = itertools.count(1 << 20, 1 << 20)

    def __init__(self, shape, dtype, stream=None, device=0):
        self.address = next(Tensor.addresses)
        self.shape, self.dtype, self.made_on, self.index = torch.Size(shape), dtype, stream, device
        self.device, self.requires_grad = f"cuda:{device}", False

    def get_device(self):
        return self.index

    def stride(self):
        out = [1]
        for n in reversed(self.shape[1:]):
            out.insert(0, out[0] * n)
        return tuple(out)

    def dim(self):
        return len(self.shape)

    def element_size(self):
        return self.dtype.itemsize

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.address


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Cuda:
    """torch.cuda with one current stream and device."""

    def __init__(self):
        self.current, self.index = threading.local(), 0

    def handle(self):
        return getattr(self.current, "handle", 1)

    @contextlib.contextmanager
    def stream(self, stream):
        before = self.handle()
        if stream is not None:
            self.current.handle = stream.cuda_stream
        yield
        self.current.handle = before

    @contextlib.contextmanager
    def device(self, index):
        before, self.index = self.index, index
        yield
        self.index = before


class Torch:
    """What _Torch offers."""

    def __init__(self):
        self.cuda, self.uint8 = Cuda(), torch.uint8
        self.torch = self
        self.codes = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
        self.bf16, self.i32, self.i64 = torch.bfloat16, torch.int32, torch.int64
        self.e4m3, self.bytes = torch.float8_e4m3fn, (torch.uint8, torch.float8_e8m0fnu)
        self.made = []
        self.grad_enabled = torch.is_grad_enabled

    def raw_stream(self, device):
        return self.cuda.handle()

    def device(self, kind=None, index=None):   # _Torch.device() and torch.device("cuda", i)
        return self.cuda.index if kind is None else index

    def capturing(self):
        return False

    def empty(self, shape, dtype, device):
        t = Tensor((shape,) if isinstance(shape, int) else shape, dtype, self.cuda.handle())
        self.made.append(t)
        return t


class Library:
    """Entry points that succeed; `calls` keeps their arguments."""

    def __init__(self):
        self.calls = []
        self.need = 4096

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call

    def kvprm_tree_workspace(self, c, t, need):
        need._obj.value = self.need
        return 0

    def kvprm_tree_attention(self, c, t, workspace, size, stream):
        self.calls.append(("kvprm_tree_attention", (workspace, size, stream)))
        return 0 if size >= self.need else ops.KVPRM_ECAPACITY

    def kvprm_tree_attention_filled(self, *args):
        return self.kvprm_tree_attention(*args)


@pytest.fixture
def face(monkeypatch):
    T, L = Torch(), Library()
    monkeypatch.setattr(ops, "_t", T)
    monkeypatch.setattr(ops, "lib", lambda: L)
    monkeypatch.setattr(ops, "_streams", {})
    return T, L


def attend(tokens=3, n=2, device=0, **kw):
    t = lambda *shape: Tensor(shape, torch.bfloat16, device=device)  # noqa: E731
    i = lambda *shape: Tensor(shape, torch.int32, device=device)  # noqa: E731
    return ops.tree_attention(t(tokens, 4, 64), t(tokens, 2, 64), t(tokens, 2, 64), t(8, 2, 2, 16, 64), i(n, 4), i(n), i(n + 1),
                              max_drafts=2, **kw)


def test_results_belong_to_the_stream_that_writes_them(face):
    """A tensor made on another stream may be in use there when the call writes it, and goes back to that stream's callers
    while this one still uses it."""
    T, L = face
    rope, side = ops.Rope(64), Stream(77)
    for stream, handle in ((side, 77), (None, 1)):
        L.calls.clear()
        out = rope.rotate(Tensor((3,), torch.int32), Tensor((3, 2, 64), torch.bfloat16), stream=stream)
        out += rope.rotate_backward(Tensor((3,), torch.int32), Tensor((3, 2, 64), torch.float32), stream=stream)
        out += (attend(stream=stream),)
        assert [x.made_on for x in out] == [handle] * 3
        assert all(x.made_on == handle for x in T.made[-4:])
        assert [c[1][-1] for c in L.calls if "create" not in c[0]] == [handle] * 3
    assert T.cuda.handle() == 1


def test_threads_share_a_streams_scratch_in_turn(face, monkeypatch):
    """A call enqueues several launches that leave and read partial results: another thread's on the same stream and scratch
    must not come between them.  Calls on other streams have scratch of their own and need not wait."""
    T, L = face
    held, overlaps, together, lock = {}, [], [], threading.Lock()

    def enqueue(c, t, workspace, size, stream):
        if size < L.need:
            return ops.KVPRM_ECAPACITY
        with lock:
            if held.get(workspace):
                overlaps.append(workspace)
            together.append(sum(held.values()))
            held[workspace] = 1
        time.sleep(0.002)   # as long as ctypes holds no lock of Python's
        with lock:
            held[workspace] = 0
        return 0

    monkeypatch.setattr(L, "kvprm_tree_attention", enqueue, raising=False)
    barrier = threading.Barrier(6)

    def work(i):
        barrier.wait()
        for k in range(20):
            if i == 0:
                L.need = 4096 * (1 + k // 4)   # scratch that is outgrown meanwhile
            attend(stream=Stream(5) if i < 4 else None)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(6)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    assert not overlaps
    assert max(together) == 1   # the two streams' calls did run beside each other


def test_scratch_of_another_device(face, monkeypatch):
    """With another device current: whether a call is being captured, and what scratch it needs, are the tensors' device's
    to say."""
    T, L = face
    capturing, asked = set(), []
    monkeypatch.setattr(T, "capturing", lambda: T.cuda.index in capturing)

    def workspace(c, t, need):
        asked.append(T.cuda.index)
        need._obj.value = L.need
        return 0

    monkeypatch.setattr(L, "kvprm_tree_workspace", workspace, raising=False)
    capturing.add(1)
    attend(device=1)
    assert ops._streams == {} and asked == [1]   # the graph's own scratch
    capturing.clear()
    capturing.add(0)
    attend(device=1)
    assert list(ops._streams) == [(1, 1)] and asked == [1, 1] and T.cuda.index == 0


def test_workspace_of_the_callers(face):
    """Scratch that the caller passes: on the tensors' device and contiguous, as its address alone is handed on; its size is
    counted in bytes."""
    T, L = face
    good = Tensor((1024,), torch.float32)
    attend(workspace=good)
    assert L.calls[-1][1][:2] == (good.address, 4096)
    host = Tensor((4096,), torch.uint8, device=-1)
    other = Tensor((4096,), torch.uint8, device=1)
    gaps = Tensor((4096,), torch.uint8)
    gaps.is_contiguous = lambda: False
    calls = len(L.calls)
    for bad in (host, other, gaps):
        with pytest.raises(ValueError, match="workspace"):
            attend(workspace=bad)
    assert len(L.calls) == calls
