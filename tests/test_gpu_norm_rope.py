"""Norm and position rotation of queries and keys (uq_norm_rope), the same with
the cache behind it (uq_norm_rope_write), and reading the cache back
(uq_read_kv) against their formulas in 64 bits.

Tolerances, u = 2^-24: the mean square is a sum of d products, at most d / 4 + 4
roundings deep, its reciprocal root 2 u, the products with the weight 2 u, the
rotation 3 u of |a| + |b|: (d / 4 + 20) u of the pair.  A 16-bit output adds half a step.
"""
import math

import pytest
import torch

import serving_ref as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_STEP = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def uq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_20474_amd import uq as mod
    return mod


DEV = "cuda:0"


def table(rot, rows=4000):
    angle = torch.outer(torch.arange(rows, dtype=torch.float64),
                        10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot))
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(DEV)


def inputs(T, hq, hkv, d, dtype, seed, fused):
    g = torch.Generator(device=DEV).manual_seed(seed)
    buf = torch.randn((T, hq + 2 * hkv, d), generator=g, device=DEV)
    buf[:, hq:, 3] *= 20
    buf = buf.to(dtype)
    rows = buf[:, :hq], buf[:, hq:hq + hkv], buf[:, hq + hkv:]
    rows = rows if fused else [x.contiguous() for x in rows]
    w = [torch.rand(d, generator=g, device=DEV) + 0.5 for _ in range(2)]
    pos = torch.randint(0, 4000, (T,), generator=g, device=DEV, dtype=torch.int32)
    return (*rows, w, pos)


def check_rows(got, x, w, pos, cs, inter, d):
    want = ref.norm_rope(x, w, 1e-6, pos, cs, inter)
    plain = ref.norm_rope(x, w, 1e-6, pos, None, inter)
    top = plain.abs().amax(-1, keepdim=True)   # |a| + |b| of any pair is at most twice this
    err = (got.double() - want).abs()
    tol = 2 * (d / 4 + 20) * U * top + HALF_STEP[got.dtype] * want.abs() + 2.0 ** -25 * (got.dtype == torch.float16)
    worst = float((err / tol.clamp(min=1e-300)).max())
    print(f"  worst error {worst:.3f} of its bound", flush=True)
    assert worst <= 1


@pytest.mark.parametrize("d,rot", [(64, 64), (64, 32), (64, 16), (64, 0), (128, 128), (128, 64), (128, 32), (128, 16),
                                   (256, 256), (256, 192), (256, 128), (256, 64), (256, 32), (256, 0)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_rows(uq, d, rot, inter, norm):
    for T, hq, hkv, dtype, fused in ((1, 1, 1, torch.float32, False), (37, 6, 3, torch.float32, True),
                                     (70, 5, 1, torch.bfloat16, True), (33, 16, 2, torch.float16, False)):
        print(f"d {d} rot {rot} interleaved {inter} norm {norm} T {T} heads {hq}/{hkv} {dtype} fused {fused}", flush=True)
        q, k, _, w, pos = inputs(T, hq, hkv, d, dtype, T + d, fused)
        cs = table(rot) if rot else None
        spec = uq.NormRope(positions=pos, cos_sin=cs, q_weight=w[0] if norm else None, k_weight=w[1] if norm else None,
                           interleaved=inter)
        qo, ko = uq.norm_rope(spec, q, k)
        check_rows(qo, q, spec.q_weight, pos, cs, inter, d)
        check_rows(ko, k, spec.k_weight, pos, cs, inter, d)


def test_output_types_and_queries_alone(uq):
    q, k, _, w, pos = inputs(19, 4, 2, 128, torch.bfloat16, 1, True)
    cs = table(128)
    spec = uq.NormRope(pos, cs, w[0], None)
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        qo, ko = uq.norm_rope(spec, q, k, out_dtype=dt)
        assert qo.dtype == ko.dtype == dt
        check_rows(qo, q, w[0], pos, cs, False, 128)
        check_rows(ko, k, None, pos, cs, False, 128)
    qo, none = uq.norm_rope(spec, q)
    assert none is None
    check_rows(qo, q, w[0], pos, cs, False, 128)


def test_in_place(uq):
    q, k, _, w, pos = inputs(50, 4, 2, 128, torch.bfloat16, 2, False)
    spec = uq.NormRope(pos, table(128), w[0], w[1])
    want = uq.norm_rope(spec, q.clone(), k.clone())
    uq.norm_rope(spec, q, k, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_positions_are_clamped_and_zero_rows_are_zero(uq):
    q, k, _, w, pos = inputs(8, 2, 1, 128, torch.float32, 3, False)
    cs = table(128, 10)
    pos = torch.tensor([-5, 0, 9, 10, 1 << 30, 3, -(1 << 31), 7], dtype=torch.int32, device=DEV)
    q[5] = 0
    spec = uq.NormRope(pos, cs, w[0], w[1])
    qo, _ = uq.norm_rope(spec, q, k)
    check_rows(qo, q, w[0], pos, cs, False, 128)
    assert torch.all(qo[5] == 0)


def slots_of(T, pages, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randperm(pages * 16, generator=g)[:T].to(DEV)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rotate_v", [True, False])
def test_write_is_norm_rope_then_quantize(uq, d, dtype, rotate_v):
    for T, hq, hkv, fused in ((1, 8, 1, False), (16, 4, 4, True), (100, 6, 3, True)):
        print(f"d {d} {dtype} rotate_v {rotate_v} T {T} heads {hq}/{hkv}", flush=True)
        q, k, v, w, pos = inputs(T, hq, hkv, d, dtype, T, fused)
        k[T // 2] = 0
        v[T // 2] = 0
        spec = uq.NormRope(pos, table(64), w[0], w[1])
        desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=9, rotate_v=rotate_v, head_dim=d)
        slots = slots_of(T, 9, d)
        if T > 2:
            slots[1], slots[2] = -1, 16 * 9
        pools, want = desc.alloc_pools(DEV, fill=0x5A), desc.alloc_pools(DEV, fill=0x5A)
        q8 = uq.norm_rope_write(desc, spec, q, k, v, slots, *pools)
        qf, kf = uq.norm_rope(spec, q, k, out_dtype=torch.float32)
        uq.quantize_kv(desc, kf, v.float().contiguous(), slots, *want)
        assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1])
        if d == 128:
            assert torch.equal(q8, uq.prepare_query(desc, qf))
        want8 = ref.e4m3(ref.walsh(qf.double()))
        got8 = q8.view(torch.float8_e4m3fn).double()
        off = got8 != want8     # a value at a border may round the other way
        assert float(off.float().mean()) <= 1e-4 + 1.5 / off.numel()
        assert torch.all((got8 - want8).abs() <= 2.0 ** -3 * want8.abs() + 2.0 ** -9)
        for dt in (torch.float32, torch.bfloat16, torch.float16):
            rows = uq.norm_rope_write(desc, spec, q, k, v, slots, *pools, q_out_dtype=dt)
            assert torch.equal(rows, uq.norm_rope(spec, q, k, out_dtype=dt)[0])


def test_write_through_a_page_table(uq):
    q, k, v, w, pos = inputs(40, 4, 2, 128, torch.bfloat16, 4, True)
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=12)
    pt = torch.tensor([[5, 1, 9], [0, 11, 3]], dtype=torch.int32, device=DEV)
    logical = torch.cat([torch.arange(0, 25), torch.arange(48, 63)]).to(DEV)
    physical = pt.reshape(-1).long()[logical // 16] * 16 + logical % 16
    spec = uq.NormRope(pos, table(128), w[0], w[1])
    a, b = desc.alloc_pools(DEV, fill=1), desc.alloc_pools(DEV, fill=1)
    uq.norm_rope_write(desc, spec, q, k, v, logical, *a, page_table=pt)
    uq.norm_rope_write(desc, spec, q, k, v, physical, *b)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ka, va = uq.read_kv(desc, logical, *a, page_table=pt)
    kb, vb = uq.read_kv(desc, physical, *a)
    assert torch.equal(ka, kb) and torch.equal(va, vb)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rotate_v", [True, False])
@pytest.mark.parametrize("T,hkv", [(1, 1), (17, 3), (160, 8)])
def test_read(uq, d, dtype, rotate_v, T, hkv):
    desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=11, rotate_v=rotate_v, head_dim=d)
    codes, scales = ref.fill_pools(desc, DEV, d + T)
    slots = slots_of(T, 11, T)
    if T > 2:
        slots[0], slots[2] = -4, 11 * 16 + 3
    valid = (slots >= 0) & (slots < 11 * 16)
    shape = (T, hkv, d)
    k, v = torch.full(shape, 3.0, dtype=dtype, device=DEV), torch.full(shape, 3.0, dtype=dtype, device=DEV)
    uq.read_kv(desc, slots, codes, scales, k_out=k, v_out=v)
    assert torch.all(k[~valid] == 3) and torch.all(v[~valid] == 3)
    ks, vs = ref.pool_values(desc, codes, scales)
    for got, stored, rotate in ((k, ks, True), (v, vs, rotate_v)):
        x = stored[slots[valid]]
        want = ref.walsh(x) if rotate else x
        # log2 d additions and one product, each half a step of at most the sum of magnitudes
        tol = (math.log2(d) + 1) * U * x.abs().sum(-1, keepdim=True) / math.sqrt(d) + HALF_STEP[dtype] * want.abs()
        assert torch.all((got[valid].double() - want).abs() <= tol + 2.0 ** -25 * (dtype == torch.float16))
    only, none = uq.read_kv(desc, slots, codes, scales, v_out=torch.full(shape, 3.0, dtype=dtype, device=DEV))[::-1]
    assert none is None and torch.equal(only, v)


def test_read_then_write_again_keeps_the_bytes(uq):
    """Values on the grid quantise to themselves when the scale the rule picks is theirs: here, whatever
    the scale, the decoded values after one round trip are those of a second one."""
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=8, rotate_v=False)
    g = torch.Generator(device=DEV).manual_seed(7)
    v = torch.randn((100, 2, 128), generator=g, device=DEV)
    slots = slots_of(100, 8, 7)
    pools = desc.alloc_pools(DEV, fill=0)
    uq.quantize_kv(desc, v, v, slots, *pools)
    _, back = uq.read_kv(desc, slots, *pools, out_dtype=torch.float32)
    _, stored = ref.pool_values(desc, *pools)
    assert torch.equal(back.double(), stored[slots])


def test_no_tokens(uq):
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=2)
    pools = desc.alloc_pools(DEV, fill=3)
    e = torch.empty((0, 2, 128), device=DEV)
    s = torch.empty(0, dtype=torch.int64, device=DEV)
    pos = torch.empty(0, dtype=torch.int32, device=DEV)
    spec = uq.NormRope(pos, table(128))
    assert uq.norm_rope(spec, e, e)[0].shape == (0, 2, 128)
    assert uq.norm_rope_write(desc, spec, e, e, e, s, *pools).shape == (0, 2, 128)
    assert uq.read_kv(desc, s, *pools)[0].shape == (0, 2, 128)
