"""Rotary positions with several axes (uq_norm_rope_axes, uq_norm_rope_axes_write)
against their formula in 64 bits, with the tolerances of test_gpu_norm_rope.py:
(d / 4 + 20) u of the pair, u = 2^-24, and half a step of a 16-bit output.  What
equal axes give, and the cache's bytes, have to be those of the calls with one
position.
"""
import pytest
import torch

import serving_ref as ref
from test_gpu_norm_rope import DEV, HALF_STEP, U, inputs, table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def uq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_20474_amd import uq as mod
    return mod


def rotated(x, w, pos, axes, cs, inter):
    """[T, H, d] in 64 bits; pos [A, T], an axis for each pair."""
    x = ref.norm_rope(x, w, 1e-6, pos[0], None, inter)
    half = cs.shape[1] // 2
    y = x.clone()
    for j, a in enumerate(axes):
        row = cs.double()[pos[a].long().clamp(0, cs.shape[0] - 1)]
        c, s = row[:, j, None], row[:, half + j, None]
        i, k = (2 * j, 2 * j + 1) if inter else (j, j + half)
        y[..., i], y[..., k] = x[..., i] * c - x[..., k] * s, x[..., k] * c + x[..., i] * s
    return y


def check(got, x, w, pos, axes, cs, inter):
    want = rotated(x, w, pos, axes, cs, inter)
    top = ref.norm_rope(x, w, 1e-6, pos[0], None, inter).abs().amax(-1, keepdim=True)
    d = x.shape[-1]
    tol = 2 * (d / 4 + 20) * U * top + HALF_STEP[got.dtype] * want.abs() + 2.0 ** -25 * (got.dtype == torch.float16)
    worst = float(((got.double() - want).abs() / tol.clamp(min=1e-300)).max())
    print(f"  worst error {worst:.3f} of its bound", flush=True)
    assert worst <= 1


def places(n_axes, T, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(0, 4000, (n_axes, T), generator=g, device=DEV, dtype=torch.int32)


# sections in runs of 8 pairs, of 4, of any length, and axes in turns
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 32), (64, 16), (128, 128), (128, 64), (256, 256), (256, 192), (128, 32)])
@pytest.mark.parametrize("how", ["eights", "fours", "odd", "turns", "four axes", "one axis"])
@pytest.mark.parametrize("inter", [False, True])
def test_axes(uq, d, rot, how, inter):
    half = rot // 2
    if how == "eights":
        axes = [(j // 8) % 3 for j in range(half)]
    elif how == "fours":
        axes = [(j // 4 * 2 + 1) % 3 for j in range(half)]
    elif how == "odd":
        axes = uq.pair_axes_of((half - half // 2 - half // 3, half // 2, half // 3))
    elif how == "turns":
        axes = uq.pair_axes_of((half - 2 * (half // 4), half // 4, half // 4), in_turns=True)
    elif how == "four axes":
        g = torch.Generator().manual_seed(rot)
        axes = torch.randint(0, 4, (half,), generator=g).tolist()
    else:
        axes = [0] * half
    T, n = 37, max(axes) + 1
    q, k, v, w, _ = inputs(T, 6, 2, d, torch.bfloat16, seed=d + rot, fused=True)
    pos, cs = places(n, T, rot), table(rot)
    spec = uq.NormRope(pos, cs, w[0], w[1], interleaved=inter, pair_axes=axes)
    qo, ko = uq.norm_rope(spec, q, k, out_dtype=torch.float32)
    check(qo, q, w[0], pos, axes, cs, inter)
    check(ko, k, w[1], pos, axes, cs, inter)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_types(uq, dtype, d):
    T = 130
    q, k, v, w, _ = inputs(T, 5, 1, d, dtype, seed=d, fused=False)
    axes = uq.pair_axes_of((d // 2 - 2 * (d // 8) - 1, d // 8 + 1, d // 8))
    pos, cs = places(3, T, d), table(d)
    qo, ko = uq.norm_rope(uq.NormRope(pos, cs, w[0], w[1], pair_axes=axes), q, k)
    assert qo.dtype == dtype
    check(qo, q, w[0], pos, axes, cs, False)
    check(ko, k, w[1], pos, axes, cs, False)
    # in place, without a norm
    mine = q.clone()
    uq.norm_rope(uq.NormRope(pos, cs, pair_axes=axes), mine, q_out=mine)
    check(mine, q, None, pos, axes, cs, False)


@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 32), (256, 256), (64, 16)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("turns", [False, True])
def test_equal_axes_are_one_position(uq, d, rot, inter, turns):
    """The bits of the call with one position, whatever the axes are."""
    T, half = 50, rot // 2
    q, k, v, w, pos = inputs(T, 6, 2, d, torch.bfloat16, seed=rot, fused=True)
    axes = uq.pair_axes_of((half - 2 * (half // 4), half // 4, half // 4), in_turns=turns)
    cs = table(rot)
    one = uq.norm_rope(uq.NormRope(pos, cs, w[0], w[1], interleaved=inter), q, k)
    more = uq.norm_rope(uq.NormRope(pos.expand(3, T).contiguous(), cs, w[0], w[1], interleaved=inter, pair_axes=axes), q, k)
    assert all(torch.equal(a, b) for a, b in zip(one, more))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("fp8", [True, False])
def test_write(uq, d, fp8):
    """The cache bytes are those of the rows in F32, quantised; FP8 queries those of the
    rows, prepared."""
    T, hkv = 75, 2
    q, k, v, w, _ = inputs(T, 6, hkv, d, torch.bfloat16, seed=d, fused=True)
    axes = uq.pair_axes_of((d // 2 - 2 * (d // 6), d // 6, d // 6), in_turns=True)
    pos, cs = places(3, T, d), table(d)
    spec = uq.NormRope(pos, cs, w[0], w[1], pair_axes=axes)
    desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=8, head_dim=d)
    slots = torch.randperm(128, device=DEV)[:T].long()
    slots[3] = -1
    a, b = desc.alloc_pools(DEV, fill=0x33), desc.alloc_pools(DEV, fill=0x33)
    q8 = uq.norm_rope_write(desc, spec, q, k, v, slots, *a, q_out_dtype=torch.uint8 if fp8 else torch.float32)
    qo, ko = uq.norm_rope(spec, q, k, out_dtype=torch.float32)
    uq.quantize_kv(desc, ko, v.float().contiguous(), slots, *b)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    if not fp8:
        assert torch.equal(q8, qo)
    else:
        kv = torch.zeros((T, hkv, d), device=DEV)
        none = torch.full((T,), -1, dtype=torch.int64, device=DEV)
        assert torch.equal(q8, uq.norm_rope_write(desc, uq.NormRope(), qo, kv, kv, none, *b))


def test_positions_are_clamped_on_every_axis(uq):
    q, k, v, w, _ = inputs(9, 4, 1, 128, torch.float32, seed=1, fused=False)
    pos = places(3, 9, 1)
    pos[0, 2], pos[1, 3], pos[2, 4] = -5, 4000, 2 ** 31 - 1
    axes, cs = uq.pair_axes_of((16, 24, 24)), table(128)
    qo, _ = uq.norm_rope(uq.NormRope(pos, cs, w[0], w[1], pair_axes=axes), q)
    check(qo, q, w[0], pos, axes, cs, False)


def test_graph_and_stream(uq):
    q, k, v, w, _ = inputs(40, 4, 2, 128, torch.bfloat16, seed=2, fused=False)
    spec = uq.NormRope(places(3, 40, 2), table(128), w[0], w[1], pair_axes=uq.pair_axes_of((24, 20, 20), in_turns=True))
    want = uq.norm_rope(spec, q, k)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        uq.norm_rope(spec, q, k, q_out=qo, k_out=ko)
    for _ in range(3):
        qo.zero_(), ko.zero_()
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = uq.norm_rope(spec, q, k, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
