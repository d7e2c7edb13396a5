"""The operators' calls as torch's allocator, threads and gradients meet them."""
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
