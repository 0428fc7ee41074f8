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


def plan(**kw):
    """Two sequences over rows of 4 pages, 4 free pages, 8 token rows; every array has its own memory unless named."""
    a = {n: 0x10000 * (i + 1) for i, n in enumerate(("cached", "new", "free", "table", "context", "cu", "seq", "pos",
                                                     "slots", "result"))}
    a.update(kw)
    p = {n: at(x) for n, x in a.items()}
    return uq.lib.uq_plan_tokens(2, p["cached"], p["new"], p["free"], 4, p["table"], 4, 8, p["context"], p["cu"], p["seq"],
                                 p["pos"], p["slots"], p["result"], None)


SIZES = dict(cached=8, new=8, free=16, table=32, context=8, cu=12, seq=32, pos=32, slots=64, result=12)


@pytest.mark.parametrize("out", ["table", "context", "cu", "seq", "pos", "slots", "result"])
@pytest.mark.parametrize("other", list(SIZES))
def test_plan_outputs_stand_alone(out, other):
    """An output is written by one block while others still read the inputs."""
    if out == other:
        return
    for first, second in ((out, other), (other, out)):      # the same start, and the last bytes of either
        assert plan(**{first: 0x200000, second: 0x200000}) == INVALID
        assert plan(**{first: 0x200000, second: 0x200000 + SIZES[first] - 4}) == INVALID
