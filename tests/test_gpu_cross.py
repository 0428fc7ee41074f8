"""uq_cross_attention against a plain 64-bit form on the same cache bytes, with the
tolerances of test_gpu_extend.py: 1e-3 in the 2-norm of the result, BF16 output half
a step, 2^-8, more."""
import math

import pytest
import torch

import serving_ref as ref

pytestmark = pytest.mark.gpu

REL = 1e-3
DEV = "cuda:0"


@pytest.fixture(scope="module")
def uq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_20474_amd import uq as mod
    return mod


def plain(desc, kv, q8, cu, table, lens, scale):
    k_all, v_all = kv
    d, hkv = desc.head_dim, desc.num_kv_heads
    out = torch.zeros(q8.shape, dtype=torch.float64, device=DEV)
    g = q8.shape[1] // hkv
    for b, n in enumerate(lens):
        m = cu[b + 1] - cu[b]
        if m <= 0 or n <= 0:
            continue
        t = torch.arange(n, device=DEV)
        slot = table[b].long()[t // 16] * 16 + t % 16
        for h in range(hkv):
            qh = q8[cu[b]:cu[b + 1], h * g:(h + 1) * g].reshape(-1, d)
            p = torch.softmax(qh @ k_all[slot, h].t().contiguous() * scale, -1)
            out[cu[b]:cu[b + 1], h * g:(h + 1) * g] = (p @ v_all[slot, h]).reshape(m, g, d)
    return ref.walsh(out) if desc.rotate_v else out


def case(uq, lens, news, hq, hkv, d, seed, dtype=torch.float32, rotate_v=True, bound=0, out_dtype=torch.float32, pad=0,
         stride_pad=0, prepared=False, poison=True):
    print(f"lens {lens[:8]} news {news[:8]} heads {hq}/{hkv} d {d} {dtype} seed {seed}", flush=True)
    bound = max(bound, *lens)
    table, pages = ref.tables(lens, DEV, seed, width=max(1, -(-bound // 16)))
    desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=pages, rotate_v=rotate_v, head_dim=d)
    codes, scales = ref.fill_pools(desc, DEV, seed)
    kv = ref.pool_values(desc, codes, scales)
    if poison:   # slots behind a context
        sc = scales.view(pages, hkv, 2, d // 32, 16)
        for b, n in enumerate(lens):
            if n % 16:
                sc[table[b, n // 16].long(), :, :, :, n % 16:] = 255
    cu = [0]
    for m in news:
        cu.append(cu[-1] + m)
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    q = torch.randn((cu[-1] + pad, hq + stride_pad, d), generator=g, device=DEV).to(dtype)[:, :hq]
    q8 = ref.e4m3(ref.walsh(q.double()))
    q_in = q8.float().to(torch.float8_e4m3fn).view(torch.uint8).contiguous() if prepared else q
    out = torch.full((cu[-1] + pad, hq, d), 7.0, dtype=out_dtype, device=DEV)
    uq.cross_attention(desc, q_in, torch.tensor(cu, dtype=torch.int32, device=DEV), codes, scales, table,
                       torch.tensor(lens, dtype=torch.int32, device=DEV), bound, out=out)
    torch.cuda.synchronize()
    want = plain(desc, kv, q8, cu, table, lens, d ** -0.5)[:cu[-1]]
    assert torch.all(out[cu[-1]:] == 7.0), "rows behind the last sequence were written"
    got = out[:cu[-1]].double()
    assert torch.isfinite(got).all()
    tol = REL + (2.0 ** -8 if out_dtype == torch.bfloat16 else 0.0)
    rel = float((got - want).norm() / want.norm().clamp(min=1e-300))
    worst = float(((got - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1).clamp(min=1e-3)).max())
    print(f"  rel {rel:.2e} worst token row {worst:.2e}", flush=True)
    assert rel <= tol and worst <= 20 * tol
    return out


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(8, 1), (16, 2), (6, 3), (5, 5), (32, 2), (12, 1)])
def test_ragged(uq, d, hq, hkv):
    case(uq, [1, 16, 70, 300, 129, 5], [3, 16, 300, 7, 65, 200], hq, hkv, d, seed=d + hq)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("m", [1, 5, 17, 100])
def test_few_queries_over_a_long_context(uq, d, m):
    """Split over blocks and joined."""
    case(uq, [9001], [m], 8, 1, d, seed=m)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_shares_of_one_length(uq, d):
    case(uq, [5000, 40, 900, 2000, 1, 0], [5, 5, 3, 1, 5, 2], 8, 2, d, seed=d)


@pytest.mark.parametrize("d", [64, 128])
def test_more_blocks_than_run_at_once(uq, d):
    """Sequences of different lengths, the longest first."""
    case(uq, [900, 3000, 31, 0, 1700], [800, 400, 1200, 9, 1100], 64, 8, d, seed=d)


def test_empty_contexts_and_no_queries(uq):
    case(uq, [0, 40, 0, 20], [3, 0, 0, 40], 8, 2, 128, seed=2, pad=5, bound=64)


def test_many_sequences(uq):
    case(uq, [(37 * i) % 150 for i in range(150)], [i % 4 for i in range(150)], 6, 2, 128, seed=6, pad=9)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_types_strides_and_padding(uq, dtype, d):
    case(uq, [90, 40], [30, 111], 8, 2, d, seed=3, dtype=dtype, out_dtype=torch.bfloat16, pad=9, stride_pad=4)
    case(uq, [90, 40], [30, 111], 8, 2, d, seed=3, dtype=dtype, rotate_v=False, bound=700)
    case(uq, [90, 40], [30, 111], 8, 2, d, seed=3, dtype=dtype, prepared=True)


def test_one_query_each_is_decode_attention(uq):
    """The same result as uq_decode_attention, within both calls' bar."""
    lens = [333, 1500, 16]
    table, pages = ref.tables(lens, DEV, 4)
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=pages)
    codes, scales = ref.fill_pools(desc, DEV, 4)
    q = torch.randn((3, 16, 128), device=DEV)
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    a = uq.cross_attention(desc, q, torch.arange(4, dtype=torch.int32, device=DEV), codes, scales, table, lens_t, 1500,
                           out_dtype=torch.float32)
    b = uq.decode_attention(desc, q, codes, scales, table, lens_t, 1500)
    assert float((a - b).norm() / b.norm()) <= 2 * REL


def test_graph_shared_workspace_and_stream(uq):
    lens, news = [4000, 300], [5, 40]
    table, pages = ref.tables(lens, DEV, 5)
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=pages)
    codes, scales = ref.fill_pools(desc, DEV, 5)
    q = torch.randn((45, 16, 128), device=DEV)
    cu = torch.tensor([0, 5, 45], dtype=torch.int32, device=DEV)
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ws = torch.full((uq.extend_workspace_bound(128),), 0xFF, dtype=torch.uint8, device=DEV)
    args = (desc, q, cu, codes, scales, table, lens_t, 4000)
    want, causal = uq.cross_attention(*args), uq.extend_attention(*args)
    out, out2 = torch.empty_like(want), torch.empty_like(want)
    graphs = []
    for call, o, w in ((uq.cross_attention, out, want), (uq.extend_attention, out2, causal)):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            call(*args, workspace=ws, out=o)
        graphs.append((gr, o, w))
    for _ in range(3):
        for gr, o, w in graphs:
            o.zero_()
            gr.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = uq.cross_attention(*args, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_scale_and_magnitudes(uq):
    """Scores of large magnitude stay finite and pick the largest."""
    lens = [100]
    table, pages = ref.tables(lens, DEV, 6)
    desc = uq.CacheDesc(num_kv_heads=1, num_pages=pages)
    codes, scales = ref.fill_pools(desc, DEV, 6)
    kv = ref.pool_values(desc, codes, scales)
    q = torch.randn((20, 8, 128), device=DEV)
    out = uq.cross_attention(desc, q, torch.tensor([0, 20], dtype=torch.int32, device=DEV), codes, scales, table,
                             torch.tensor(lens, dtype=torch.int32, device=DEV), 100, softmax_scale=1e16, out_dtype=torch.float32)
    want = plain(desc, kv, ref.e4m3(ref.walsh(q.double())), [0, 20], table, lens, 1e16)
    assert float((out.double() - want).norm() / want.norm()) <= REL
    assert math.isfinite(float(out.abs().max()))
