"""Calls without tokens: nothing of theirs has an address (an empty tensor's is NULL), and there is nothing to refuse."""
import ctypes

import paper_2607_09153_gb300 as kp
from paper_2607_09153_gb300 import operators as ops

P = 0x10000


def test_write_nothing_rotated():
    c = ops.KvprmCache(P, None, 8, 2, 64, kp.KVPRM_CACHE_BF16)
    rope = kp.Rope(32)
    go = lambda n, pos, handle=rope.handle: ops.lib().kvprm_cache_write(  # noqa: E731
        ctypes.byref(c), kp.KVPRM_BF16, None, 128, 64, None, 128, 64, None, n, handle, pos, None)
    assert go(0, None) == kp.KVPRM_OK and go(0, P) == kp.KVPRM_OK and go(0, None, None) == kp.KVPRM_OK
    assert go(1, None) == kp.KVPRM_EINVAL
    too_wide = kp.Rope(128)
    assert go(0, None, too_wide.handle) == kp.KVPRM_EINVAL
