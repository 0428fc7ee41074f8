"""Limits of the calls around the cache, on the host: sizes past which a kernel's
32-bit indices would wrap, and buffers that may not overlap.  Nothing is
launched and no pointer is followed."""
import ctypes

import pytest

from paper_2606_20474_amd import uq

INVALID, UNSUPPORTED = uq.UQ_ERR_INVALID_ARGUMENT, uq.UQ_ERR_UNSUPPORTED


def at(address):
    return ctypes.c_void_p(address)


def desc(**kw):
    d = dict(num_kv_heads=2, head_dim=128, page_size=16, group_size=32, num_pages=10, c=0.156, rotate_v=1)
    d.update(kw)
    return uq.uq_cache_desc(**d)


@pytest.mark.parametrize("window", [0, 100])
def test_longest_context(window):
    """Pages ahead of the walk are counted in 32 bits: contexts end well below 2^31 tokens."""
    P, D = at(0x10000), desc()

    def extend(max_context):   # without queries, so that a context in range is refused for that
        return uq.lib.uq_extend_attention(ctypes.byref(D), None, 1, 512, 2, P, 2, 4, P, P, P, 1 << 27, P, max_context,
                                          window, 0, 0.1, P, 0, P, 1, None)

    for n in ((1 << 30) + 1, (1 << 31) - 16):
        assert extend(n) == UNSUPPORTED
        assert uq.lib.uq_extend_workspace_bytes(ctypes.byref(D), 2, 2, 4, n, window, 0) == 0
    assert extend(1 << 30) == INVALID
    if window == 0:
        assert uq.lib.uq_extend_workspace_bytes(ctypes.byref(D), 2, 2, 4, 1 << 30, 0, 0) > 0
