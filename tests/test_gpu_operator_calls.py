"""The operators' calls as torch's allocator, threads and gradients meet them."""
import threading

import pytest

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
