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


def spec():
    return uq.uq_norm_rope_desc(None, None, 1e-6, None, None, 0, 0, 0)


# one token row: 4 query heads and 2 KV heads of 128, BF16; 6 tokens
T, Q, KV = 6, 4 * 128 * 2, 2 * 128 * 2
BF16, F16, F32, FP8 = uq.UQ_BF16, uq.UQ_F16, uq.UQ_F32, uq.UQ_FP8_E4M3


def rope(q, k, qo, ko, qs=512, ks=256, odt=BF16, dt=BF16, tokens=T):
    s = spec()
    return uq.lib.uq_norm_rope(ctypes.byref(s), 128, at(q), qs, 4, at(k), ks, 2, dt, tokens, at(qo), at(ko), odt, None)


def write(q, k, v, qo, qs=512, ks=256, odt=FP8):
    s, D, P = spec(), desc(), at(0x900000)
    return uq.lib.uq_norm_rope_write(ctypes.byref(D), ctypes.byref(s), at(q), qs, 4, at(k), at(v), ks, BF16, T, at(qo), odt,
                                     None, 0, 0, P, P, P, None)


def test_row_outputs_stand_alone():
    """A vector's lanes write its place after they have read it; another vector's input there may not be read yet."""
    A, B, C, E = 0x100000, 0x200000, 0x300000, 0x400000
    for kw in (dict(q=A, k=B, qo=A, ko=C, odt=F32), dict(q=A, k=B, qo=A, ko=C, odt=F16),      # another type
               dict(q=A, k=B, qo=A, ko=C, qs=1024), dict(q=A, k=B, qo=A + 64, ko=C),          # other places of q
               dict(q=A, k=B, qo=A + T * Q - 16, ko=C), dict(q=A, k=B, qo=A - T * Q + 16, ko=C),
               dict(q=A, k=B, qo=C, ko=B, odt=F32), dict(q=A, k=B, qo=C, ko=B, ks=512),
               dict(q=A, k=B, qo=B, ko=C), dict(q=A, k=B, qo=C, ko=A), dict(q=A, k=B, qo=C, ko=C),
               dict(q=A, k=B, qo=C, ko=C + T * Q - 16), dict(q=A, k=B, qo=C + T * KV - 16, ko=C),
               # rows of one buffer: the output in the middle of it
               dict(q=A, k=A + Q, qo=A + 3 * (Q + 2 * KV), ko=C, qs=1024, ks=1024)):
        assert rope(**kw) == INVALID, kw
    for kw in (dict(qo=A), dict(qo=A, odt=F16), dict(qo=A, odt=BF16, qs=1024), dict(qo=A + 16), dict(qo=B), dict(qo=C),
               dict(qo=C + T * KV - 16), dict(qo=A + T * Q - 16)):
        assert write(**{**dict(q=A, k=B, v=C), **kw}) == INVALID, kw


@pytest.mark.parametrize("d", [64, 128, 256])
def test_one_workspace_for_every_step(d):
    """The bound holds over batches, heads and contexts, and is within 4 times the largest need met here."""
    bound = uq.extend_workspace_bound(d)
    largest, grows_down = 0, False
    for hkv, group in ((1, 1), (1, 16), (2, 5), (4, 8), (8, 8), (8, 16), (3, 12), (128, 1), (600, 1)):
        D = desc(head_dim=d, num_kv_heads=hkv)
        for batch in (1, 2, 3, 16, 63, 64, 65, 300, 5000):
            last = 0
            for tokens in sorted({1, 2, 5, batch, 2 * batch, 5 * batch, 64 * batch // group + 1, 64, 128, 333, 512, 1024, 2048,
                                  8191, 8192, 100000, 1 << 23}):
                for context in (0, 16, 600, 5000, 131072, 1 << 30):
                    for window in (0, 300, 40000):
                        need = uq.lib.uq_extend_workspace_bytes(ctypes.byref(D), tokens, batch, hkv * group, context, window, 4)
                        assert need <= bound, (hkv, group, batch, tokens, context, window)
                        largest = max(largest, need)
                grows_down = grows_down or need < last
                last = need
    assert grows_down and largest * 4 >= bound


def test_the_header_states_the_same_bound(tmp_path):
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "bound.c"
    src.write_text('#include "uq.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu\\n", '
                   "UQ_EXTEND_WORKSPACE_BOUND(64), UQ_EXTEND_WORKSPACE_BOUND(128), UQ_EXTEND_WORKSPACE_BOUND(256)); return 0; }\n")
    subprocess.run([cc, "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "bound")], check=True)
    got = subprocess.run([str(tmp_path / "bound")], check=True, capture_output=True, text=True).stdout.split()
    assert [int(x) for x in got] == [uq.extend_workspace_bound(d) for d in (64, 128, 256)]
