"""Refusals of the calls around the cache, on the host: the C ABI's argument
checks (nothing is launched, pointers are never followed) and the binding's."""
import ctypes

import pytest
import torch

from paper_2606_20474_amd import uq

FAKE = ctypes.c_void_p(0x10000)
ODD = ctypes.c_void_p(0x10004)
OK, INVALID, UNSUPPORTED, SMALL = uq.UQ_OK, uq.UQ_ERR_INVALID_ARGUMENT, uq.UQ_ERR_UNSUPPORTED, uq.UQ_ERR_WORKSPACE_TOO_SMALL


def desc(**kw):
    d = dict(num_kv_heads=2, head_dim=128, page_size=16, group_size=32, num_pages=10, c=0.156, rotate_v=1)
    d.update(kw)
    return uq.uq_cache_desc(**d)


def spec(**kw):
    d = dict(q_weight=0x10000, k_weight=0x10000, eps=1e-6, positions=0x10000, cos_sin=0x10000, max_position=8,
             rot_dim=128, interleaved=0)
    d.update(kw)
    return uq.uq_norm_rope_desc(**d)


def plan(batch=2, cached=FAKE, free=FAKE, nfree=4, table=FAKE, mpps=4, T=8, ctx=FAKE, cu=FAKE, slots=FAKE, result=FAKE):
    return uq.lib.uq_plan_tokens(batch, cached, FAKE, free, nfree, table, mpps, T, ctx, cu, FAKE, FAKE, slots, result, None)


def test_plan_tokens():
    for kw in (dict(batch=-1), dict(nfree=-1), dict(T=-1), dict(mpps=0), dict(cached=None), dict(table=None),
               dict(ctx=None), dict(cu=None), dict(slots=None), dict(result=None), dict(free=None)):
        assert plan(**kw) == INVALID, kw
    for kw in (dict(batch=4097), dict(T=1 << 29), dict(nfree=1 << 29), dict(mpps=1 << 27)):
        assert plan(**kw) == UNSUPPORTED, kw


def rope(s=None, d=128, q=FAKE, qs=512, hq=4, k=FAKE, ks=256, hkv=2, dt=1, T=3, qo=FAKE, ko=FAKE, odt=1):
    s = spec() if s is None else s
    return uq.lib.uq_norm_rope(ctypes.byref(s), d, q, qs, hq, k, ks, hkv, dt, T, qo, ko, odt, None)


def test_norm_rope():
    assert uq.lib.uq_norm_rope(None, 128, FAKE, 512, 4, FAKE, 256, 2, 1, 3, FAKE, FAKE, 1, None) == INVALID
    for kw in (dict(q=None), dict(q=ODD), dict(qo=None), dict(qo=ODD), dict(qs=511), dict(qs=516), dict(hq=0), dict(T=-1),
               dict(k=None), dict(ko=None), dict(hkv=0), dict(hkv=-1), dict(ks=255), dict(ko=ODD), dict(k=ODD),
               dict(s=spec(eps=-1.0)), dict(s=spec(eps=float("nan"))), dict(s=spec(positions=None)),
               dict(s=spec(cos_sin=None)), dict(s=spec(max_position=0)), dict(s=spec(q_weight=0x10004)),
               dict(s=spec(cos_sin=0x10008)), dict(s=spec(rot_dim=-64))):
        assert rope(**kw) == INVALID, kw
    for kw in (dict(d=96), dict(dt=3), dict(odt=3), dict(s=spec(rot_dim=96)), dict(s=spec(rot_dim=192)),
               dict(s=spec(rot_dim=8)), dict(T=1 << 30)):
        assert rope(**kw) == UNSUPPORTED, kw
    assert rope(T=0, q=None, qo=None, k=None, ko=None) == OK
    assert rope(T=0, s=spec(positions=None)) == OK


def write(D=None, s=None, q=FAKE, k=FAKE, v=FAKE, ks=256, dt=1, T=3, qo=FAKE, odt=3, pt=None, ns=0, mpps=0, slots=FAKE,
          codes=FAKE):
    D, s = desc() if D is None else D, spec() if s is None else s
    return uq.lib.uq_norm_rope_write(ctypes.byref(D), ctypes.byref(s), q, 512, 4, k, v, ks, dt, T, qo, odt, pt, ns, mpps,
                                     slots, codes, FAKE, None)


def test_norm_rope_write():
    for kw in (dict(k=None), dict(v=ODD), dict(ks=248), dict(slots=None), dict(codes=None), dict(codes=ODD), dict(T=-1),
               dict(pt=FAKE, ns=0, mpps=4), dict(pt=FAKE, ns=2, mpps=0), dict(D=desc(c=0.0)), dict(D=desc(num_pages=0))):
        assert write(**kw) == INVALID, kw
    for kw in (dict(dt=3), dict(odt=4), dict(D=desc(head_dim=96)), dict(D=desc(page_size=32)), dict(s=spec(rot_dim=80))):
        assert write(**kw) == UNSUPPORTED, kw
    assert write(T=0, q=None, k=None, v=None, slots=None, qo=None) == OK


def read(D=None, codes=FAKE, slots=FAKE, T=3, k=FAKE, v=FAKE, dt=1, pt=None, ns=0, mpps=0):
    D = desc() if D is None else D
    return uq.lib.uq_read_kv(ctypes.byref(D), codes, FAKE, pt, ns, mpps, slots, T, k, v, dt, None)


def test_read_kv():
    for kw in (dict(codes=None), dict(slots=None), dict(T=-1), dict(k=None, v=None), dict(k=ODD), dict(v=ODD),
               dict(pt=FAKE, ns=0, mpps=1)):
        assert read(**kw) == INVALID, kw
    for kw in (dict(dt=3), dict(D=desc(head_dim=32)), dict(D=desc(group_size=16))):
        assert read(**kw) == UNSUPPORTED, kw
    assert read(T=0, slots=None, k=None, v=None) == OK


def extend(D=None, q=FAKE, dt=1, qs=512, T=64, cu=FAKE, B=2, hq=4, codes=FAKE, pt=FAKE, mpps=400, ctx=FAKE, maxctx=6400,
           window=0, sinks=0, scale=0.1, ws=FAKE, wsb=1 << 40, out=FAKE, odt=1):
    D = desc() if D is None else D
    return uq.lib.uq_extend_attention(ctypes.byref(D), q, dt, qs, T, cu, B, hq, codes, FAKE, pt, mpps, ctx, maxctx, window,
                                      sinks, scale, ws, wsb, out, odt, None)


def test_extend_attention():
    for kw in (dict(q=None), dict(q=ODD), dict(qs=504), dict(qs=516), dict(dt=3, qs=520), dict(cu=None), dict(B=-1),
               dict(T=-1), dict(hq=3), dict(hq=0), dict(codes=None), dict(codes=ODD), dict(pt=None), dict(mpps=0),
               dict(ctx=None), dict(maxctx=6401), dict(maxctx=-1), dict(window=-1), dict(sinks=-1), dict(scale=0.0),
               dict(scale=float("inf")), dict(ws=None), dict(ws=ODD), dict(out=None), dict(out=ODD)):
        assert extend(**kw) == INVALID, kw
    for kw in (dict(dt=4), dict(odt=2), dict(hq=34), dict(D=desc(head_dim=96)), dict(T=1 << 24), dict(B=65536)):
        assert extend(**kw) == UNSUPPORTED, kw
    D = desc()
    need = uq.lib.uq_extend_workspace_bytes(ctypes.byref(D), 64, 2, 4, 6400, 0, 0)
    assert need > 0 and extend(wsb=need - 1) == SMALL
    assert extend(T=0, q=None, out=None) == OK
    assert extend(B=0, cu=None) == OK
    for bad in ((-1, 2, 4, 64, 0, 0), (64, -1, 4, 64, 0, 0), (64, 2, 3, 64, 0, 0), (64, 2, 4, -1, 0, 0),
                (64, 2, 4, 64, -1, 0), (64, 2, 4, 64, 4, -1)):
        assert uq.lib.uq_extend_workspace_bytes(ctypes.byref(D), *bad) == 0


def window(D=None, q=FAKE, dt=1, k=None, v=None, ndt=0, B=2, hq=4, mpps=400, maxctx=6400, w=100, sinks=4, part=0, ws=FAKE,
           wsb=1 << 40, scale=0.1):
    D = desc() if D is None else D
    return uq.lib.uq_decode_window(ctypes.byref(D), q, dt, k, v, ndt, B, hq, FAKE, FAKE, FAKE, mpps, FAKE, maxctx, w, sinks,
                                   scale, part, ws, wsb, FAKE, 1, None)


def test_decode_window():
    for kw in (dict(w=0), dict(w=-5), dict(sinks=-1), dict(maxctx=-1), dict(maxctx=6401), dict(mpps=0), dict(q=None),
               dict(k=FAKE), dict(v=FAKE), dict(k=ODD, v=FAKE), dict(part=8), dict(hq=3), dict(B=0), dict(ws=None),
               dict(scale=-1.0)):
        assert window(**kw) == INVALID, kw
    for kw in (dict(dt=4), dict(hq=34), dict(k=FAKE, v=FAKE, ndt=3), dict(D=desc(head_dim=64), k=FAKE, v=FAKE),
               dict(D=desc(head_dim=256), dt=3), dict(D=desc(head_dim=96))):
        assert window(**kw) == UNSUPPORTED, kw
    D = desc()
    need = uq.lib.uq_decode_window_workspace_bytes(ctypes.byref(D), 2, 4, 6400, 100, 4, 16)
    assert need > 0 and window(part=16, wsb=need - 1) == SMALL
    # the walk is bounded by the window: less than the whole context needs
    assert need < uq.lib.uq_decode_workspace_bytes(ctypes.byref(D), 2, 4, 6400, 16)
    for bad in ((2, 4, 6400, 0, 4, 0), (2, 4, 6400, 10, -1, 0), (2, 4, -1, 10, 0, 0), (0, 4, 64, 10, 0, 0)):
        assert uq.lib.uq_decode_window_workspace_bytes(ctypes.byref(D), *bad) == 0


def test_host_tensors_and_wrong_shapes_are_rejected():
    d = uq.CacheDesc(num_kv_heads=2, num_pages=4)
    q, k = torch.zeros(3, 4, 128), torch.zeros(3, 2, 128)
    u8, i32, i64 = torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    pt = torch.zeros((1, 4), dtype=torch.int32)
    sp = uq.NormRope(torch.zeros(3, dtype=torch.int32), torch.zeros(8, 128))
    calls = [
        lambda: uq.plan_tokens(i32, i32, i32, pt, uq.TokenPlan.alloc(2, 4, "cpu")),
        lambda: uq.norm_rope(sp, q, k),
        lambda: uq.norm_rope_write(d, sp, q, k, k, i64, u8, u8),
        lambda: uq.read_kv(d, i64, u8, u8),
        lambda: uq.extend_attention(d, q, i32, u8, u8, pt, i32[:1], 64),
        lambda: uq.decode_window(d, q[:1], u8, u8, pt, i32[:1], 64, 16),
    ]
    for call in calls:
        with pytest.raises(ValueError, match="on the GPU"):
            call()


def test_more_blocks_than_a_grid_holds():
    """A grid has fewer than 2^32 threads; larger calls are refused before the launch."""
    one = spec(rot_dim=0)
    assert rope(s=one, d=64, qs=64, hq=1, k=None, ko=None, hkv=0, T=1 << 30) == UNSUPPORTED
    assert rope(s=one, d=64, qs=64, hq=1, ks=64, hkv=1, T=1 << 29) == UNSUPPORTED
    assert write(T=1 << 28) == UNSUPPORTED
    D = desc(head_dim=64, num_kv_heads=1)
    assert read(D=D, T=1 << 30) == UNSUPPORTED
    assert extend(D=desc(num_kv_heads=1024, head_dim=64), hq=1024, qs=65536, T=1 << 23, B=65535) == UNSUPPORTED
