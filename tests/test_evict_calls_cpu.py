"""Refusals of the calls for positions with several axes, cross attention and
eviction, on the host: the C ABI's argument checks (nothing is launched, pointers
are never followed) and the binding's."""
import ctypes

import pytest
import torch

from paper_2606_20474_amd import uq

FAKE, ODD = 0x10000, 0x10004
OK, INVALID, UNSUPPORTED, SMALL = uq.UQ_OK, uq.UQ_ERR_INVALID_ARGUMENT, uq.UQ_ERR_UNSUPPORTED, uq.UQ_ERR_WORKSPACE_TOO_SMALL
NAN, INF = float("nan"), float("inf")


def at(i):
    """Distinct addresses, far apart."""
    return 0x100000000 * (i + 1)


def desc(**kw):
    d = dict(num_kv_heads=2, head_dim=128, page_size=16, group_size=32, num_pages=10, c=0.156, rotate_v=1)
    d.update(kw)
    return uq.uq_cache_desc(**d)


def spec(**kw):
    d = dict(q_weight=FAKE, k_weight=FAKE, eps=1e-6, positions=FAKE, cos_sin=FAKE, max_position=8, rot_dim=128, interleaved=0)
    d.update(kw)
    return uq.uq_norm_rope_desc(**d)


def axes(n=3, stride=8, pairs=bytes([0, 1, 2, 0] * 16)):
    return uq.uq_rope_axes(n, stride, pairs)


def rope(a, s=None, T=0, d=128):
    s = spec() if s is None else s
    return uq.lib.uq_norm_rope_axes(ctypes.byref(s), None if a is None else ctypes.byref(a), d, at(0), 512, 4, at(1), 256,
                                    2, 1, T, at(2), at(3), 1, None)


def rope_write(a, s=None, T=0, D=None):
    s, D = spec() if s is None else s, desc() if D is None else D
    return uq.lib.uq_norm_rope_axes_write(ctypes.byref(D), ctypes.byref(s), None if a is None else ctypes.byref(a), at(0),
                                          512, 4, at(1), at(2), 256, 1, T, at(3), 3, None, 0, 0, at(4), at(5), at(6), None)


@pytest.mark.parametrize("call", [rope, rope_write])
def test_rope_axes(call):
    assert call(axes()) == OK
    assert call(axes(4, 0)) == OK   # no tokens
    for a in (None, axes(0), axes(-1), axes(5), axes(pairs=None), axes(2), axes(pairs=bytes([0] * 63 + [3])),
              axes(pairs=bytes([255] * 64)), axes(stride=-1)):
        assert call(a) == INVALID
    assert call(axes(stride=2), T=3) == INVALID
    assert call(axes(), spec(rot_dim=0)) == INVALID
    assert call(axes(), spec(rot_dim=96)) == UNSUPPORTED
    assert call(axes(), spec(cos_sin=None)) == INVALID
    assert call(axes(), spec(positions=None), T=3) == INVALID


def test_pair_axes_of():
    assert uq.pair_axes_of((2, 1, 3)) == (0, 0, 1, 2, 2, 2)
    assert uq.pair_axes_of((4, 2, 2), in_turns=True) == (0, 1, 2, 0, 1, 2, 0, 0)
    assert uq.pair_axes_of((3, 1), in_turns=True) == (0, 1, 0, 0)
    for sections in ((24, 20, 20), (16, 24, 24), (11, 11, 10)):
        if sections != (16, 24, 24):
            got = uq.pair_axes_of(sections, in_turns=True)
            assert [got.count(a) for a in range(3)] == list(sections)
        assert [uq.pair_axes_of(sections).count(a) for a in range(3)] == list(sections)
    with pytest.raises(ValueError):
        uq.pair_axes_of((16, 24, 24), in_turns=True)   # the third axis would end behind the last pair


def cross(D=None, q=at(0), dt=1, stride=512, T=8, cu=at(1), B=2, hq=4, codes=at(2), scales=at(3), table=at(4), mpps=4,
          lens=at(5), bound=64, scale=0.1, ws=at(6), wsb=1 << 30, out=at(7), odt=1):
    D = desc() if D is None else D
    return uq.lib.uq_cross_attention(ctypes.byref(D), q, dt, stride, T, cu, B, hq, codes, scales, table, mpps, lens, bound,
                                     scale, ws, wsb, out, odt, None)


def test_cross_attention():
    assert cross(T=0) == OK and cross(B=0) == OK
    for kw in (dict(q=None), dict(cu=None), dict(codes=None), dict(scales=None), dict(table=None), dict(lens=None),
               dict(out=None), dict(q=ODD), dict(out=ODD), dict(ws=ODD), dict(stride=504), dict(stride=511), dict(T=-1),
               dict(B=-1), dict(hq=0), dict(hq=3), dict(bound=-1), dict(bound=65), dict(mpps=0), dict(scale=0.0),
               dict(scale=NAN), dict(scale=INF), dict(scale=-1.0), dict(D=desc(num_pages=0)), dict(D=desc(c=0.0))):
        assert cross(**kw) == INVALID, kw
    for kw in (dict(dt=4), dict(odt=2), dict(hq=34), dict(T=1 << 24), dict(B=65536), dict(D=desc(head_dim=96)),
               dict(D=desc(page_size=32))):
        assert cross(**kw) == UNSUPPORTED, kw
    assert cross(bound=65000, mpps=5000, wsb=16) == SMALL
    assert cross(bound=65000, mpps=5000, ws=None) == INVALID
    D = desc()
    n = uq.lib.uq_cross_workspace_bytes(ctypes.byref(D), 8, 2, 4, 65000)
    assert 0 < n <= uq.extend_workspace_bound(128)
    assert uq.lib.uq_cross_workspace_bytes(ctypes.byref(D), -1, 2, 4, 65000) == 0


def weights(D=None, q=at(0), dt=3, stride=512, T=8, cu=at(1), B=2, hq=4, codes=at(2), scales=at(3), table=at(4), mpps=4,
            lens=at(5), bound=64, last=0, causal=1, scale=0.1, w=at(6), width=64, ws=at(7), wsb=1 << 30):
    D = desc() if D is None else D
    return uq.lib.uq_token_weights(ctypes.byref(D), q, dt, stride, T, cu, B, hq, codes, scales, table, mpps, lens, bound,
                                   last, causal, scale, w, width, ws, wsb, None)


def test_token_weights():
    assert weights(T=0) == OK and weights(B=0) == OK and weights(bound=0) == OK
    for kw in (dict(q=None), dict(cu=None), dict(codes=None), dict(scales=None), dict(table=None), dict(lens=None),
               dict(w=None), dict(ws=None), dict(q=ODD), dict(ws=ODD), dict(codes=ODD), dict(stride=511), dict(stride=504),
               dict(T=-1), dict(B=-1), dict(hq=0), dict(hq=3), dict(bound=-1), dict(bound=65), dict(mpps=0),
               dict(scale=0.0), dict(scale=NAN), dict(scale=INF), dict(last=-1), dict(width=63), dict(D=desc(num_pages=0)),
               # weights or workspace over an input or each other
               dict(w=at(0)), dict(w=at(1)), dict(w=at(2) + 64), dict(w=at(5) + 4), dict(w=at(7)), dict(ws=at(3)),
               dict(ws=at(4) - 256), dict(ws=at(0))):
        assert weights(**kw) == INVALID, kw
    for kw in (dict(dt=4), dict(hq=34), dict(T=1 << 24), dict(B=65536), dict(D=desc(head_dim=96)),
               dict(bound=(1 << 30) + 1), dict(D=desc(group_size=16)), dict(stride=1 << 26),
               dict(T=1 << 23, hq=128, D=desc(num_kv_heads=128), stride=128 * 128)):
        assert weights(**kw) == UNSUPPORTED, kw
    assert weights(wsb=1 << 20) == SMALL


def test_token_weights_workspace_does_not_fall():
    """The size for the largest step is enough for the smaller ones."""
    for d in (64, 128, 256):
        D = desc(head_dim=d, num_kv_heads=4)

        def size(T, B, bound, last, dt=3):
            return uq.lib.uq_token_weights_workspace_bytes(ctypes.byref(D), dt, T, B, 32, bound, last)

        most = size(8192, 64, 131072, 0)
        for T in (1, 7, 64, 1000, 8192):
            for B in (1, 5, 64):
                for bound in (1, 500, 131072):
                    for last in (0, 1, 64):
                        assert 0 < size(T, B, bound, last) <= most
        assert size(100, 1, 100, 0, 1) > size(100, 1, 100, 0)   # rows are prepared there
        assert size(-1, 1, 1, 0) == size(1, 1, 1, -1) == size(1, 1, -1, 0) == 0


def select(w=at(0), width=100, B=2, H=3, lens=at(1), bound=100, budget=10, sinks=2, recent=3, kept=at(2), kl=at(3),
           ws=at(4), wsb=1 << 30):
    return uq.lib.uq_select_tokens(w, width, B, H, lens, bound, budget, sinks, recent, kept, kl, ws, wsb, None)


def test_select_tokens():
    assert select(B=0) == OK
    for kw in (dict(w=None), dict(lens=None), dict(kept=None), dict(kl=None), dict(B=-1), dict(H=0), dict(bound=-1),
               dict(budget=0), dict(budget=-1), dict(sinks=-1), dict(recent=-1), dict(sinks=8), dict(recent=9),
               dict(sinks=1 << 30, recent=1 << 30), dict(width=99), dict(kl=at(1)), dict(kl=at(1) + 4), dict(kept=at(0)),
               dict(kept=at(3) - 8), dict(kl=at(0) + 400)):
        assert select(**kw) == INVALID, kw
    for kw in (dict(B=65536), dict(H=65536), dict(B=2000, H=5000), dict(B=(1 << 15) - 1, H=64 + 1), dict(bound=(1 << 30) + 1, width=1 << 31),
               dict(budget=(1 << 30) + 1), dict(B=1000, H=8, bound=1 << 26, width=1 << 26)):
        assert select(**kw) == UNSUPPORTED, kw
    assert uq.select_workspace_bytes(2, 3, 16384, 10) == 0 and uq.select_workspace_bytes(2, 3, 1 << 20, 1 << 20) == 0
    n = uq.select_workspace_bytes(2, 3, 40000, 10)
    assert n > 0 and select(bound=40000, width=40000, wsb=n - 1) == SMALL
    for kw in (dict(ws=None), dict(ws=at(4) + 4), dict(ws=at(0)), dict(ws=at(2) + 16)):
        assert select(bound=40000, width=40000, **kw) == INVALID, kw


def compact(D=None, kept=at(0), budget=10, kl=at(1), lens=at(2), B=2, codes=at(3), scales=at(4), table=at(5), mpps=4, w=at(6),
            width=64, freed=at(7), count=at(8), ws=at(9), wsb=1 << 30):
    D = desc() if D is None else D
    return uq.lib.uq_compact_kv(ctypes.byref(D), kept, budget, kl, lens, B, codes, scales, table, mpps, w, width, freed,
                                count, ws, wsb, None)


def test_compact_kv():
    for kw in (dict(kept=None), dict(kl=None), dict(lens=None), dict(codes=None), dict(scales=None), dict(table=None),
               dict(codes=ODD), dict(scales=ODD), dict(B=-1), dict(budget=0), dict(mpps=0), dict(width=-1),
               dict(freed=None), dict(count=None), dict(D=desc(num_pages=0)),
               # outputs over inputs or each other
               dict(w=at(0)), dict(w=at(3) + 128), dict(freed=at(5)), dict(freed=at(2)), dict(count=at(1)),
               dict(count=at(7) + 8), dict(scales=at(3) + 64)):
        assert compact(**kw) == INVALID, kw
    for kw in (dict(B=65536), dict(mpps=1 << 27), dict(budget=(1 << 30) + 1), dict(D=desc(head_dim=96)),
               dict(B=32, mpps=1 << 26)):
        assert compact(**kw) == UNSUPPORTED, kw
    assert compact(B=0, freed=None, count=None) == OK
    D = desc()
    n = uq.lib.uq_compact_kv_workspace_bytes(ctypes.byref(D), 2, 10)
    assert n > 0 and compact(wsb=n - 1) == SMALL
    for kw in (dict(ws=None), dict(ws=at(9) + 8), dict(ws=at(3)), dict(ws=at(0))):
        assert compact(**kw) == INVALID, kw
    assert uq.lib.uq_compact_kv_workspace_bytes(ctypes.byref(D), 32, 10) == 0   # 64 pairs: in place


def test_binding_wants_gpu_tensors():
    D = uq.CacheDesc(num_kv_heads=2, num_pages=4)
    codes, scales = torch.zeros(D.codes_bytes(), dtype=torch.uint8), torch.zeros(D.scales_bytes(), dtype=torch.uint8)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q, cu, table, lens, w = torch.zeros((3, 4, 128)), i(3), i(2, 2), i(2), torch.zeros((2, 2, 32))
    for call in (lambda: uq.cross_attention(D, q, cu, codes, scales, table, lens, 32),
                 lambda: uq.token_weights(D, q, cu, codes, scales, table, lens, 32, w),
                 lambda: uq.select_tokens(w, lens, 32, 8),
                 lambda: uq.compact_kv(D, i(2, 2, 8), lens, lens, codes, scales, table),
                 lambda: uq.norm_rope(uq.NormRope(i(3, 3), torch.zeros((4, 128)), pair_axes=[0] * 64), q)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_pair_axes_from_sequences():
    sp = uq.NormRope(torch.zeros((3, 5), dtype=torch.int32), torch.zeros(8, 16), pair_axes=(0, 0, 1, 1, 2, 2, 0, 1))
    want = sp.axes_struct().pair_axes
    for axes in (list(sp.pair_axes), bytes(sp.pair_axes), torch.tensor(sp.pair_axes), torch.tensor(sp.pair_axes).numpy()):
        sp.pair_axes = axes
        a = sp.axes_struct()
        assert (a.num_axes, a.position_stride, a.pair_axes) == (3, 5, want)
    for axes in (8, (0,) * 7, (0,) * 7 + (256,), (0,) * 7 + (-1,), (0,) * 7 + (0.5,)):
        sp.pair_axes = axes
        with pytest.raises((TypeError, ValueError)):
            sp.axes_struct()
