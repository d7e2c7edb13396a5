"""The operators' calls as torch's allocator, threads and gradients meet them."""
import threading

import pytest

from tests import operators_util as ref
from tests.gpu_util import require_gpu
from tests.test_gpu_operators import Tree

pytestmark = pytest.mark.gpu


def test_results_of_a_side_stream():
    """What a call on a side stream returned and its caller dropped is not handed to the current stream, where nothing waits
    for the call."""
    torch = require_gpu()
    import paper_2607_09153_gb300 as kp
    side, rope = torch.cuda.Stream(), kp.Rope(64)
    x = torch.zeros((777, 3, 64), device="cuda")
    pos = torch.zeros(777, dtype=torch.int32, device="cuda")
    t = Tree(torch, 4, 2, 64, [40, 10], [3, 2], seed=1)
    t.run(stream=side)
    torch.cuda.synchronize()
    for call in (lambda: rope.rotate(pos, x, stream=side)[0], lambda: rope.rotate_backward(pos, x, stream=side)[0],
                 lambda: t.run(stream=side)):
        y = call()
        torch.cuda.synchronize()
        at, shape, dtype = y.data_ptr(), y.shape, y.dtype
        del y
        kept = [torch.empty(shape, dtype=dtype, device="cuda") for _ in range(8)]
        assert at not in [z.data_ptr() for z in kept]


def test_threads_on_one_stream():
    """Host threads that call on one stream, each with sequences of its own that several CTAs share: what each call gives
    alone, bit for bit."""
    torch = require_gpu()
    trees = [Tree(torch, 8, 2, 128, [9000 + 1000 * i, 5000], [1 + 3 * i, 2], i % 2 == 1, seed=i) for i in range(4)]
    args = [dict(lens=torch.tensor(t.lens, dtype=torch.int32).cuda(), start=torch.tensor(t.start, dtype=torch.int32).cuda())
            for t in trees]
    alone = [t.run(**a) for t, a in zip(trees, args)]
    torch.cuda.synchronize()
    results, barrier = [None] * 4, threading.Barrier(4)

    def work(i):
        barrier.wait()
        results[i] = [trees[i].run(**args[i]) for _ in range(100)]

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    torch.cuda.synchronize()
    for a, many in zip(alone, results):
        assert all(torch.equal(a, o) for o in many)


def _rope_inputs(torch, n=19):
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k = (torch.randn((n, h, 64), generator=gen, device="cuda").requires_grad_() for h in (3, 2))
    return q, k, torch.randint(0, 9999, (n,), generator=gen, device="cuda", dtype=torch.int32), gen


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_is_differentiable(interleaved, inverse):
    """Against autograd of the definition in 64 bits: the map is linear with factors of at most `magnitude`, so a gradient is
    off by what the call itself may be (6e-7 of two magnitudes), here through one rotation more."""
    torch = require_gpu()
    import paper_2607_09153_gb300 as kp
    q, k, pos, gen = _rope_inputs(torch)
    rope = kp.Rope(32, interleaved=interleaved, magnitude=1.25)
    call = rope.rotate_backward if inverse else rope.rotate
    plain = lambda x: ref.rotate(x, pos, ref.frequencies(32), interleaved, 1.25, inverse)  # noqa: E731
    dq, dk = (torch.randn(x.shape, generator=gen, device="cuda") for x in (q, k))
    yq, yk = call(pos, q, k)
    assert yq.requires_grad and yk.requires_grad
    got = torch.autograd.grad(((yq * dq).sum(), (yk * dk).sum()), (q, k))
    want = torch.autograd.grad(((plain(q) * dq).sum(), (plain(k) * dk).sum()), (q, k))
    for g, w, d in zip(got, want, (dq, dk)):
        assert bool(((g.double() - w.double()).abs() <= 3e-6 * d.abs().amax(-1, keepdim=True)).all())
    # a gradient that is not dense, a tensor that wants none, and the gradient's own gradient
    (g,) = torch.autograd.grad(call(pos, q, k.detach())[0].sum(), (q,))
    (w,) = torch.autograd.grad(plain(q).sum(), (q,))
    assert bool(((g.double() - w.double()).abs() <= 3e-6).all())
    assert not call(pos, q, k.detach())[1].requires_grad
    (g,) = torch.autograd.grad((call(pos, q)[0] ** 3).sum(), (q,), create_graph=True)
    (gg,) = torch.autograd.grad((g * dq).sum(), (q,))
    (w,) = torch.autograd.grad((plain(q) ** 3).sum(), (q,), create_graph=True)
    (ww,) = torch.autograd.grad((w * dq).sum(), (q,))
    assert bool(((gg.double() - ww.double()).abs() <= 1e-4 * ww.double().abs().amax()).all())


def test_rotation_gradient_of_a_side_stream():
    torch = require_gpu()
    import paper_2607_09153_gb300 as kp
    q, _, pos, _ = _rope_inputs(torch)
    rope, side = kp.Rope(64), torch.cuda.Stream()
    rope.rotate(pos, q)[0].sum().backward()
    want, q.grad = q.grad, None
    side.wait_stream(torch.cuda.current_stream())
    y = rope.rotate(pos, q, stream=side)[0]
    with torch.cuda.stream(side):
        loss = y.sum()
    loss.backward()
    torch.cuda.synchronize()
    assert torch.equal(q.grad, want)


def test_gradients_that_there_are_not():
    """No gradient is dropped without a word: outputs of the caller's and the attention."""
    torch = require_gpu()
    import paper_2607_09153_gb300 as kp
    q, _, pos, _ = _rope_inputs(torch)
    rope = kp.Rope(64)
    with pytest.raises(ValueError):
        rope.rotate(pos, q, out=(torch.empty_like(q),))
    with torch.no_grad():
        y = torch.empty_like(q)
        assert rope.rotate(pos, q, out=(y,))[0] is y
        assert not rope.rotate(pos, q)[0].requires_grad
    t = Tree(torch, 4, 2, 64, [40, 10], [3, 2], seed=1)
    plain = t.run()
    for name in ("q", "k", "v"):
        x = getattr(t, name)
        setattr(t, name, x.detach().clone().requires_grad_())
        out = t.run()
        assert torch.equal(out, plain)
        with pytest.raises(RuntimeError, match="tree_attention"):
            out.float().sum().backward()
        with pytest.raises(ValueError):
            t.run(out=torch.empty_like(plain))
        with torch.no_grad():
            assert not t.run().requires_grad
        setattr(t, name, x)
