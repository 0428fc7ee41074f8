"""Attention of several new queries per sequence over the FP4 cache
(uq_extend_attention) against a plain 64-bit form on the same cache bytes.

Tolerances, relative to the 2-norm of the result, with F32 output: P is cut to
FP16, a loss of 0 to 2^-10 of each weight, of which the kernel gives the mean over
significands, 3.5e-4, back: at most 6.3e-4 either way; the query's FP8 rounding is the
reference's too (a value at a border may round the other way: 2^-24-sized
differences, about one in 10^6 elements, a step of 2^-3 of one channel of 64 or
more), and the QK instruction itself is off by up to 1e-4 of a row's scores
(tests/test_gpu_qk_precision_bound.py).  6.3e-4 + 1e-4 < 1e-3, the library's bar.  BF16
output adds half a step, 2^-8, elementwise.
"""
import math

import pytest
import torch

import serving_ref as ref

pytestmark = pytest.mark.gpu

REL = 1e-3


@pytest.fixture(scope="module")
def uq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_20474_amd import uq as mod
    return mod


def log(msg):
    print(msg, flush=True)


def case(uq, lens, news, hq, hkv, d, seed, window=0, sinks=0, dtype=torch.float32, rotate_v=True, bound=0,
         out_dtype=torch.float32, pad=0, v_scale=1.0, stride_pad=0, q_gain=1.0, prepared=False, poison=None):
    """Runs one batch and compares every row; returns (out, reference)."""
    dev = torch.device("cuda:0")
    log(f"lens {lens} news {news} heads {hq}/{hkv} d {d} window {window} sinks {sinks} {dtype} seed {seed}")
    table, pages = ref.tables(lens, dev, seed, width=max(1, -(-max(bound, *lens) // 16)))
    desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=pages, rotate_v=rotate_v, head_dim=d)
    codes, scales = ref.fill_pools(desc, dev, seed, v_scale)
    kv = ref.pool_values(desc, codes, scales)
    if poison is not None:
        poison(desc, codes, scales, table)
    cu = [0]
    for m in news:
        cu.append(cu[-1] + m)
    T = cu[-1] + pad
    g = torch.Generator(device=dev).manual_seed(seed + 1)
    q = (torch.randn((T, hq + stride_pad, d), generator=g, device=dev) * q_gain).to(dtype)[:, :hq]
    q_in = q
    if prepared:
        q_in = ref.walsh(q.float()).clamp(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8).contiguous()
    out = torch.full((T, hq, d), 7.0, dtype=out_dtype, device=dev)
    uq.extend_attention(desc, q_in, torch.tensor(cu, dtype=torch.int32, device=dev), codes, scales, table,
                        torch.tensor(lens, dtype=torch.int32, device=dev), max(bound, *lens, 0), window=window,
                        sinks=sinks, out=out)
    torch.cuda.synchronize()
    want = ref.attend(desc, kv, q_in if prepared else q, cu, table, lens, window, sinks, prepared=prepared)
    assert torch.all(out[cu[-1]:] == 7.0), "rows behind the last sequence were written"
    got, want = out[:cu[-1]].double(), want[:cu[-1]]
    assert torch.isfinite(got).all()
    tol = REL + (2.0 ** -8 if out_dtype == torch.bfloat16 else 0.0)
    if got.numel():
        rel = float((got - want).norm() / want.norm().clamp(min=1e-300)) if want.norm() > 0 else float(got.abs().max())
        worst = ((got - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1).clamp(min=1e-30)).max()
        log(f"  rel {rel:.2e} worst token row {worst:.2e}")
        assert rel <= tol
        # one token's heads: a border case of the query's rounding moves a few rows, not the whole
        assert worst <= 20 * tol
    return out, want


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(8, 1), (16, 2), (6, 3), (5, 5), (32, 2), (12, 1)])
def test_ragged(uq, d, hq, hkv):
    case(uq, [1, 16, 70, 300, 129, 5], [1, 16, 3, 300, 65, 2], hq, hkv, d, seed=d + hq)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (17, 0), (64, 4), (100, 200), (33, 16), (4096, 7)])
def test_windows(uq, d, window, sinks):
    case(uq, [700, 64, 333, 1], [300, 64, 1, 1], 8, 2, d, seed=window + d, window=window, sinks=sinks)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("news", [[1], [5], [17]])
@pytest.mark.parametrize("n", [3001, 9000])
def test_few_queries_over_a_long_context(uq, d, news, n):
    """Split over blocks and joined."""
    case(uq, [n] * len(news), news, 8, 1, d, seed=n + d)


@pytest.mark.parametrize("window,sinks", [(2500, 4), (2500, 600), (5000, 0)])
def test_split_windows(uq, window, sinks):
    case(uq, [9000, 4000, 100], [7, 1, 100], 8, 2, 128, seed=window, window=window, sinks=sinks)


def test_long_prompt(uq):
    case(uq, [2048], [2048], 8, 1, 128, seed=1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_types_strides_and_padding(uq, dtype, d):
    case(uq, [90, 40], [30, 11], 8, 2, d, seed=3, dtype=dtype, out_dtype=torch.bfloat16, pad=9, stride_pad=4)
    case(uq, [90, 40], [30, 11], 8, 2, d, seed=3, dtype=dtype, rotate_v=False)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_prepared_queries(uq, d):
    case(uq, [90, 140], [30, 11], 8, 2, d, seed=4, prepared=True)


def test_empty_sequences_and_contexts(uq):
    out, _ = case(uq, [40, 0, 20, 33], [10, 0, 0, 33], 8, 2, 128, seed=5)
    # more queries than context: the first rows see nothing and are 0
    out, want = case(uq, [3, 0, 20], [5, 4, 20], 8, 2, 128, seed=6)
    assert torch.all(out[:2] == 0) and torch.all(out[5:9] == 0)
    assert torch.all(want[:2] == 0)
    case(uq, [3000, 0, 20], [5, 4, 20], 2, 1, 128, seed=7, bound=8000)


@pytest.mark.parametrize("v_scale", [2.0 ** -40, 2.0 ** -24, 2.0 ** 15, 2.0 ** 60])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_values_outside_fp16(uq, v_scale, d):
    case(uq, [300, 64], [70, 2], 8, 2, d, seed=8, v_scale=v_scale)


def test_one_far_scale_in_a_tile(uq):
    """Tiles with and without a wide scale next to each other."""
    dev = torch.device("cuda:0")
    lens, news = [400], [50]
    table, pages = ref.tables(lens, dev, 9)
    desc = uq.CacheDesc(num_kv_heads=1, num_pages=pages, rotate_v=False, head_dim=128)
    codes, scales = ref.fill_pools(desc, dev, 9)
    s = scales.view(pages, 1, 2, 4, 16)
    for page, group, tok, byte in ((2, 1, 3, 144), (9, 3, 15, 150), (17, 0, 0, 90), (24, 2, 8, 141)):
        s[int(table[0, page]), 0, 1, group, tok] = byte
    kv = ref.pool_values(desc, codes, scales)
    q = torch.randn((50, 8, 128), generator=torch.Generator(device=dev).manual_seed(9), device=dev)
    out = uq.extend_attention(desc, q, torch.tensor([0, 50], dtype=torch.int32, device=dev), codes, scales, table,
                              torch.tensor(lens, dtype=torch.int32, device=dev), 400, out_dtype=torch.float32)
    want = ref.attend(desc, kv, q, [0, 50], table, lens)
    got = out.double()
    for c in range(0, 128, 32):   # the groups differ by many powers of two: each has to be right by itself
        rel = float((got[..., c:c + 32] - want[..., c:c + 32]).norm() / want[..., c:c + 32].norm())
        log(f"channels {c}: rel {rel:.2e}")
        assert rel <= REL


@pytest.mark.parametrize("first,later", [(0, 124), (0, 254), (124, 254), (254, 120), (100, 113), (100, 114), (1, 140)])
def test_scales_that_grow_and_shrink_along_the_context(uq, first, later):
    """A context whose first 100 tokens have one V scale and whose others another: scores are equal (a zero
    query), so that both weigh in.  Against the sums themselves, at the larger scale's precision."""
    dev = torch.device("cuda:0")
    n = 333
    table, pages = ref.tables([n], dev, 21)
    desc = uq.CacheDesc(num_kv_heads=1, num_pages=pages, rotate_v=False, head_dim=128)
    codes, scales = ref.fill_pools(desc, dev, 21)
    s = scales.view(pages, 1, 2, 4, 16)
    for t in range(n):
        s[int(table[0, t // 16]), 0, 1, :, t % 16] = first if t < 100 else later
    kv = ref.pool_values(desc, codes, scales)
    q = torch.zeros((3, 4, 128), device=dev)
    out = uq.extend_attention(desc, q, torch.tensor([0, 3], dtype=torch.int32, device=dev), codes, scales, table,
                              torch.tensor([n], dtype=torch.int32, device=dev), n, out_dtype=torch.float32)
    want = ref.attend(desc, kv, q, [0, 3], table, [n])
    assert float((out.double() - want).norm() / want.norm()) <= REL


@pytest.mark.parametrize("gain", [0.0, 30.0, 1e4])
def test_score_ranges(uq, gain):
    case(uq, [200, 64], [80, 2], 8, 2, 128, seed=10, q_gain=gain)


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_unwritten_tokens_stay_out(uq, d, window, sinks):
    """Everything no query sees is set to codes and scales of NaN and infinity."""
    lens, news = [200, 77], [20, 3]

    def poison(desc, codes, scales, table):
        c = codes.view(desc.num_pages, desc.num_kv_heads, 2, 8 * d)
        s = scales.view(desc.num_pages, desc.num_kv_heads, 2, d // 32, 16)
        keep = torch.zeros((desc.num_pages, 16), dtype=torch.bool, device=codes.device)
        for b, n in enumerate(lens):
            for i in range(news[b]):
                for t in ref.visible(n, n - news[b] + i, window, sinks):
                    keep[int(table[b, t // 16]), t % 16] = True
        s.masked_fill_(~keep[:, None, None, None, :], 255)
        whole = ~keep.any(1)
        c[whole] = 0x77
    case(uq, lens, news, 8, 2, d, seed=11, window=window, sinks=sinks, poison=poison)


def test_against_decode_attention(uq):
    """One query per sequence is decode attention."""
    dev = torch.device("cuda:0")
    lens = [5, 200, 1000, 17]
    table, pages = ref.tables(lens, dev, 12)
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=pages)
    codes, scales = ref.fill_pools(desc, dev, 12)
    q = torch.randn((4, 16, 128), device=dev)
    n = torch.tensor(lens, dtype=torch.int32, device=dev)
    a = uq.decode_attention(desc, q, codes, scales, table, n, 1000)
    b = uq.extend_attention(desc, q, torch.arange(5, dtype=torch.int32, device=dev), codes, scales, table, n, 1000,
                            out_dtype=torch.float32)
    assert float((a - b).norm() / a.norm()) <= REL


def test_bad_device_indices_stay_in_bounds(uq):
    """Page ids outside the pool read page 0; lengths above the bound and descending offsets are clamped."""
    dev = torch.device("cuda:0")
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=8)
    codes, scales = ref.fill_pools(desc, dev, 13)
    table = torch.tensor([[0, 9, -5, 1 << 30], [3, 2, 1, 0]], dtype=torch.int32, device=dev)
    q = torch.randn((12, 8, 128), device=dev)
    for cu in ([0, 6, 12], [0, 60, 12], [-4, 6, 99], [9, 3, 12]):
        out = uq.extend_attention(desc, q, torch.tensor(cu, dtype=torch.int32, device=dev), codes, scales, table,
                                  torch.tensor([1000, -3], dtype=torch.int32, device=dev), 64, window=20, sinks=1)
        torch.cuda.synchronize()
        assert torch.isfinite(out).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("batch", [2, 40, 64, 65])
def test_more_blocks_than_run_at_once(uq, d, batch):
    """Ragged sequences, also empty ones and ones with more queries than context: their blocks run
    longest first up to 64 sequences, in order beyond."""
    g = torch.Generator().manual_seed(batch)
    lens = [int(x) for x in torch.randint(0, 400, (batch,), generator=g)]
    news = [int(x) for x in torch.randint(0, 5000 if batch == 2 else 200, (batch,), generator=g)]
    news = [n if i % 7 == 0 or batch == 2 else min(n, m) for i, (n, m) in enumerate(zip(news, lens))]
    lens[1], news[1] = (3500, 3400) if batch == 2 else (0, 0)
    case(uq, lens, news, 32 if batch > 2 else 256, 16, d, seed=batch + d)
