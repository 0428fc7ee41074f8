"""Decode attention under a sliding window with visible first tokens
(uq_decode_window) against a plain 64-bit form, at the library's bar
(relative L2 1e-3 of the result, F32 output)."""
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


def case(uq, lens, hq, hkv, d, window, sinks, seed, partition=0, bound=0, dtype=torch.float32, rotate_v=True,
         poison=False, out_dtype=torch.float32, fp8=False):
    print(f"lens {lens} heads {hq}/{hkv} d {d} window {window} sinks {sinks} partition {partition} seed {seed}",
          flush=True)
    B = len(lens)
    table, pages = ref.tables(lens, DEV, seed, width=max(1, -(-max(bound, *lens) // 16)))
    desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=pages, rotate_v=rotate_v, head_dim=d)
    codes, scales = ref.fill_pools(desc, DEV, seed)
    kv = ref.pool_values(desc, codes, scales)
    view = table.clone()
    if poison:
        # hidden tokens: NaN scales; hidden pages: handed back, their table entries anything
        s = scales.view(pages, hkv, 2, d // 32, 16)
        keep = torch.zeros((pages, 16), dtype=torch.bool, device=DEV)
        for b, n in enumerate(lens):
            seen = ref.visible(n, n - 1, window, sinks)
            for t in seen:
                keep[int(table[b, t // 16]), t % 16] = True
            for pg in set(range(table.shape[1])) - {t // 16 for t in seen}:
                view[b, pg] = 1 << 30
        s.masked_fill_(~keep[:, None, None, None, :], 255)
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = torch.randn((B, hq, d), generator=g, device=DEV).to(dtype)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    want = ref.attend(desc, kv, q, list(range(B + 1)), table, lens, window, sinks)
    q_in = uq.prepare_query(desc, q) if fp8 else q
    out = uq.decode_window(desc, q_in, codes, scales, view, n, max(bound, *lens), window, sinks=sinks,
                           partition_tokens=partition, out_dtype=out_dtype)
    torch.cuda.synchronize()
    got = out.double()
    assert torch.isfinite(got).all()
    tol = REL + (2.0 ** -8 if out_dtype == torch.bfloat16 else 0)
    for b in range(B):
        top = float(want[b].norm())
        rel = float((got[b] - want[b]).norm()) / top if top else float(got[b].abs().max())
        # a border case of the query's FP8 rounding moves one row by a step of one channel
        assert rel <= tol, (b, lens[b], rel)


LENS = [1, 16, 17, 100, 333, 1000, 0, 64]


@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 1), (128, 32, 2), (128, 5, 5), (64, 16, 2), (64, 8, 1), (64, 24, 3),
                                      (64, 16, 1), (256, 8, 2), (256, 3, 3)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (15, 4), (16, 16), (33, 0), (128, 1), (100, 40), (50, 500),
                                          (900, 3), (5000, 4), (2147483647, 2147483647)])
def test_windows(uq, d, hq, hkv, window, sinks):
    case(uq, LENS, hq, hkv, d, window, sinks, seed=window % 1000 + d + hq)


@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 1), (64, 16, 2), (64, 8, 1), (64, 16, 1), (256, 8, 2)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (20, 3), (65, 17), (130, 0)])
def test_hidden_tokens_and_pages_may_hold_anything(uq, d, hq, hkv, window, sinks):
    case(uq, LENS, hq, hkv, d, window, sinks, seed=d + window, poison=True)


@pytest.mark.parametrize("partition", [16, 48, 128, 1024])
@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 1), (64, 16, 2), (64, 8, 1), (256, 8, 2)])
def test_partitions(uq, partition, d, hq, hkv):
    case(uq, [2000, 3, 700, 0, 1499], hq, hkv, d, 600, 20, seed=partition, partition=partition)
    case(uq, [2000, 3, 700, 0, 1499], hq, hkv, d, 600, 20, seed=partition, partition=partition, poison=True)


def test_bounds_types_and_outputs(uq):
    case(uq, [300, 20000, 7], 16, 2, 128, 4096, 4, seed=1, bound=40000)
    case(uq, [300, 2000, 7], 16, 2, 128, 100, 4, seed=2, bound=2500, dtype=torch.bfloat16, out_dtype=torch.bfloat16)
    case(uq, [300, 2000, 7], 16, 2, 128, 100, 4, seed=3, dtype=torch.float16, rotate_v=False)
    case(uq, [300, 2000, 7], 16, 2, 128, 100, 4, seed=4, fp8=True)
    case(uq, [900] * 300, 8, 8, 128, 256, 4, seed=5)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_wide_window_is_decode_attention(uq, d):
    lens = [5, 200, 1000, 17]
    table, pages = ref.tables(lens, DEV, 12)
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=pages, head_dim=d)
    codes, scales = ref.fill_pools(desc, DEV, 12)
    q = torch.randn((4, 16, d), device=DEV)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    a = uq.decode_attention(desc, q, codes, scales, table, n, 1000, partition_tokens=256)
    b = uq.decode_window(desc, q, codes, scales, table, n, 1000, 1000, partition_tokens=256)
    assert torch.equal(a, b)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (40, 3), (600, 16), (5000, 0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_step(uq, window, sinks, dtype):
    """The new token is written as decode_step writes it and attended to."""
    lens = [1, 16, 17, 100, 1333, 64, 0]
    B = len(lens)
    table, pages = ref.tables(lens, DEV, window)
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=pages)
    codes, scales = ref.fill_pools(desc, DEV, window)
    g = torch.Generator(device=DEV).manual_seed(window)
    q, k, v = (torch.randn((B, h, 128), generator=g, device=DEV).to(dtype) for h in (16, 2, 2))
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    want = codes.clone(), scales.clone()
    live = n > 0
    slots = torch.where(live, torch.arange(B, device=DEV) * (table.shape[1] * 16) + n.long() - 1, -1)
    uq.quantize_kv(desc, k, v, slots, *want, page_table=table)
    out = uq.decode_window(desc, q, codes, scales, table, n, max(lens), window, sinks=sinks, k_new=k, v_new=v)
    torch.cuda.synchronize()
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
    kv = ref.pool_values(desc, codes, scales)
    exact = ref.attend(desc, kv, q, list(range(B + 1)), table, lens, window, sinks)
    for b in range(B):
        top = float(exact[b].norm())
        assert (float((out[b].double() - exact[b]).norm()) <= REL * top) if top else torch.all(out[b] == 0)
