"""uq_select_tokens and uq_compact_kv against plain indexing: indices, codes,
scale bytes and weights are equal, nothing is rounded."""
import math

import pytest
import torch

import serving_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def uq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_20474_amd import uq as mod
    return mod


def log(msg):
    print(msg, flush=True)


def chosen(w, n, budget, sinks, recent):
    """Indices that stay of one row (list of floats)."""
    if n <= budget:
        return list(range(n))
    fixed = list(range(sinks)) + list(range(n - recent, n))
    rank = sorted(range(sinks, n - recent), key=lambda t: (-(w[t] if not math.isnan(w[t]) else -math.inf),
                                                           math.isnan(w[t]), t))
    return sorted(fixed + rank[:budget - sinks - recent])


def check_select(uq, weights, lens, budget, sinks=0, recent=0, bound=None):
    log(f"select {tuple(weights.shape)} lens {lens[:8]} budget {budget} sinks {sinks} recent {recent}")
    bound = weights.shape[2] if bound is None else bound
    kept, kl = uq.select_tokens(weights, torch.tensor(lens, dtype=torch.int32, device=DEV), bound, budget, sinks=sinks,
                                recent=recent)
    kept, kl, w = kept.tolist(), kl.tolist(), weights.tolist()
    for b, n in enumerate(lens):
        n = min(n, bound)
        assert kl[b] == min(n, budget)
        for h in range(weights.shape[1]):
            want = chosen(w[b][h], n, budget, sinks, recent)
            assert kept[b][h] == want + [-1] * (budget - len(want)), (b, h)


@pytest.mark.parametrize("n", [2, 63, 64, 65, 1000, 1024, 1025, 5000])
def test_random_weights(uq, n):
    g = torch.Generator(device=DEV).manual_seed(n)
    w = torch.exp(3 * torch.randn((3, 2, n), generator=g, device=DEV))
    for budget in {1, 2, n // 3 + 1, n - 1, n, n + 5}:
        check_select(uq, w, [n, n - 1, n // 2], budget)
        check_select(uq, w, [n, n - 1, n // 2], budget, sinks=budget // 3, recent=budget // 4)
        check_select(uq, w, [n, n - 1, n // 2], budget, sinks=budget // 2, recent=budget - budget // 2)


def test_equal_weights_go_to_the_lowest_index(uq):
    g = torch.Generator(device=DEV).manual_seed(1)
    w = torch.randint(0, 4, (2, 3, 2000), generator=g, device=DEV).float() / 8
    for budget in (1, 10, 700, 1999):
        check_select(uq, w, [2000, 1500], budget, sinks=min(4, budget // 2), recent=min(64, budget // 2))
    check_select(uq, torch.zeros_like(w), [2000, 1500], 100, sinks=4, recent=9)


def test_unusual_values(uq):
    """Zeros of both signs are equal, negatives, infinities, denormals; a NaN comes last."""
    g = torch.Generator(device=DEV).manual_seed(2)
    vals = torch.tensor([0.0, -0.0, 1e-45, -1e-45, 1.0, -1.0, math.inf, -math.inf, math.nan, 3e38, 1e-38], device=DEV)
    w = vals[torch.randint(0, len(vals), (2, 2, 700), generator=g, device=DEV)]
    w[0, 0, 5] = -math.nan
    for budget in (1, 50, 128, 300, 500, 650, 699):
        check_select(uq, w, [700, 640], budget)
    check_select(uq, torch.full((1, 1, 300), math.nan, device=DEV), [300], 100)


def test_close_weights(uq):
    """Neighbouring floats: every bit of a key counts."""
    base = torch.tensor([1.0], device=DEV).view(torch.int32)
    g = torch.Generator(device=DEV).manual_seed(3)
    w = (base + torch.randint(0, 3000, (1, 2, 4000), generator=g, device=DEV).int()).view(torch.float32)
    for budget in (7, 2000, 3990):
        check_select(uq, w, [4000], budget)


def test_long_row_and_wide_array(uq):
    g = torch.Generator(device=DEV).manual_seed(4)
    w = torch.exp(2 * torch.randn((1, 2, 140001), generator=g, device=DEV))
    check_select(uq, w, [140000], 30011, sinks=4, recent=1000)
    check_select(uq, w, [70000], 30011, sinks=4, recent=1000, bound=66001)
    check_select(uq, w, [33000], 1000)


@pytest.mark.parametrize("n", [16384, 16385, 17000, 32768, 40001])
def test_rows_of_several_slices(uq, n):
    g = torch.Generator(device=DEV).manual_seed(n)
    w = torch.exp(2.5 * torch.randn((2, 2, n + 3), generator=g, device=DEV))
    w[torch.rand(w.shape, generator=g, device=DEV) < 0.1] = 0.0
    for budget, sinks, recent in ((1, 0, 0), (1000, 4, 64), (16390, 0, 16390), (n - 1, 5, n // 2), (12000, 12000, 0)):
        check_select(uq, w, [n, 16383], budget, sinks=min(sinks, budget), recent=min(recent, budget), bound=n)


def test_slices_of_equal_and_close_weights(uq):
    """More keys with the same first bits than a list holds, and ties over slices."""
    g = torch.Generator(device=DEV).manual_seed(6)
    n = 50000
    w = torch.randint(0, 3, (1, 2, n), generator=g, device=DEV).float()
    for budget in (1, 100, 16000, 33000, 49999):
        check_select(uq, w, [n], budget, sinks=min(7, budget), recent=min(20, budget) // 2)
    check_select(uq, torch.zeros_like(w), [n], 20000, sinks=4, recent=100)
    base = torch.tensor([1.0], device=DEV).view(torch.int32)
    w = (base + torch.randint(0, 30000, (1, 1, n), generator=g, device=DEV).int()).view(torch.float32)
    for budget in (5, 25000):
        check_select(uq, w, [n], budget)
    # one slice with nothing but ties, the others mixed
    w = torch.rand((1, 1, n), generator=g, device=DEV)
    w[:, :, 16384:32768] = 0.5
    for budget in (20000, 26000, 40000):
        check_select(uq, w, [n], budget)


def test_short_rows_beside_long_ones(uq):
    g = torch.Generator(device=DEV).manual_seed(7)
    w = torch.rand((6, 1, 60000), generator=g, device=DEV)
    check_select(uq, w, [60000, 0, 5, 16384, 900, 33000], 900, sinks=1, recent=30)


def test_lengths_of_zero_and_negative(uq):
    w = torch.rand((3, 2, 40), device=DEV)
    kept, kl = uq.select_tokens(w, torch.tensor([0, -3, 40], dtype=torch.int32, device=DEV), 40, 8)
    assert kl.tolist() == [0, 0, 8] and (kept[:2] == -1).all()


def test_many_rows(uq):
    g = torch.Generator(device=DEV).manual_seed(5)
    w = torch.rand((70, 3, 90), generator=g, device=DEV)
    check_select(uq, w, [(31 * i) % 91 for i in range(70)], 40, sinks=2, recent=5)


# ---------------------------------------------------------------------------


def compact_plain(desc, kept, kl, lens, codes, scales, table, weights):
    """In place, token after token of copies; returns the freed pages."""
    H, d = desc.num_kv_heads, desc.head_dim
    kc = codes.view(-1, H, 2, d // 32, 16, 16)
    vc = codes.view(-1, H, 2, 4, d // 8, 4, 4)
    sc = scales.view(-1, H, 2, d // 32, 16)
    k0, v0, s0, w0 = kc.clone(), vc.clone(), sc.clone(), weights.clone()
    freed = []
    for b, n in enumerate(lens):
        m = kl[b]
        to = torch.arange(m, device=DEV)
        p2, o2 = table[b].long()[to // 16], to % 16
        for h in range(H):
            frm = kept[b, h, :m].long()
            p1, o1 = table[b].long()[frm // 16], frm % 16
            kc[p2, h, 0, :, o2] = k0[p1, h, 0, :, o1]
            vc[p2, h, 1, o2 // 4, :, o2 % 4] = v0[p1, h, 1, o1 // 4, :, o1 % 4]
            sc[p2, h, :, :, o2] = s0[p1, h, :, :, o1]
            weights[b, h, :m] = w0[b, h, frm]
            weights[b, h, m:n] = 0
        freed += table[b, (m + 15) // 16:(max(n, 0) + 15) // 16].tolist()
    return freed


def check_compact(uq, lens, budget, hkv, d, seed, sinks=1, recent=3, same_heads=False, width_pad=3):
    log(f"compact lens {lens[:8]} budget {budget} heads {hkv} d {d} seed {seed}")
    table, pages = ref.tables(lens, DEV, seed, width=max(1, -(-max(lens) // 16)) + 2)
    desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=pages, head_dim=d)
    codes, scales = ref.fill_pools(desc, DEV, seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = torch.rand((len(lens), hkv, max(max(lens), 1) + width_pad), generator=g, device=DEV)
    if same_heads:
        w = w[:, :1].expand(-1, hkv, -1).contiguous()
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s, r = min(sinks, budget // 2), min(recent, budget // 2)
    kept, kl = uq.select_tokens(w, lens_t, max(lens), budget, sinks=s, recent=r)
    c2, s2, w2 = codes.clone(), scales.clone(), w.clone()
    freed = torch.full((table.numel(),), -7, dtype=torch.int32, device=DEV)
    count = torch.zeros(1, dtype=torch.int32, device=DEV)
    uq.compact_kv(desc, kept, kl, lens_t, codes, scales, table, weights=w, freed_pages=freed, freed_count=count)
    torch.cuda.synchronize()
    want = compact_plain(desc, kept, kl.tolist(), lens, c2, s2, table, w2)
    assert torch.equal(codes, c2) and torch.equal(scales, s2) and torch.equal(w, w2)
    assert count.item() == len(want) and freed[:len(want)].tolist() == want and (freed[len(want):] == -7).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hkv", [1, 3])
def test_compact(uq, d, hkv):
    for lens, budget in (([50], 20), ([16, 17, 33], 16), ([200, 3, 0, 129], 64), ([1000, 640], 333), ([70], 69),
                         ([5], 1), ([700], 17)):
        check_compact(uq, lens, budget, hkv, d, seed=d + hkv + budget)


def test_compact_keeps_what_fits(uq):
    check_compact(uq, [50, 90], 100, 2, 128, seed=3)


def test_compact_long(uq):
    check_compact(uq, [20000, 9000, 15011], 4099, 2, 128, seed=4, sinks=4, recent=500)
    check_compact(uq, [40000], 20000, 1, 64, seed=5, sinks=64, recent=500)
    check_compact(uq, [9001], 8999, 8, 256, seed=6)


def test_compact_many_sequences(uq):
    check_compact(uq, [(53 * i) % 300 for i in range(300)], 60, 2, 64, seed=7)


def test_compact_without_weights_and_freed(uq):
    table, pages = ref.tables([300], DEV, 1)
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=pages)
    codes, scales = ref.fill_pools(desc, DEV, 1)
    w = torch.rand((1, 2, 300), device=DEV)
    lens = torch.tensor([300], dtype=torch.int32, device=DEV)
    kept, kl = uq.select_tokens(w, lens, 300, 77)
    c2, s2 = codes.clone(), scales.clone()
    uq.compact_kv(desc, kept, kl, lens, codes, scales, table)
    compact_plain(desc, kept, kl.tolist(), [300], c2, s2, table, w)
    assert torch.equal(codes, c2) and torch.equal(scales, s2)


def test_compact_in_place_and_through_the_workspace(uq):
    """64 and more (sequence, KV head) pairs are moved in place, fewer through the workspace."""
    for d in (64, 128, 256):
        check_compact(uq, [700 + 37 * i for i in range(16)], 500, 4, d, seed=d, sinks=16, recent=100)
        check_compact(uq, [(97 * i) % 1200 for i in range(70)], 513, 1, d, seed=d + 1)
        check_compact(uq, [3000, 1100], 1030, 32, d, seed=d + 2, sinks=0, recent=0)


def test_compact_nothing(uq):
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=4)
    codes, scales = desc.alloc_pools(DEV, fill=1)
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    count = torch.full((1,), 9, dtype=torch.int32, device=DEV)
    uq.compact_kv(desc, torch.empty((0, 2, 8), dtype=torch.int32, device=DEV), none, none,
                  codes, scales, torch.empty((0, 4), dtype=torch.int32, device=DEV), freed_pages=none, freed_count=count)
    assert count.item() == 0 and (codes == 1).all()


def test_compact_leaves_shared_front_pages(uq):
    """Pages that keep all their tokens are not written: two sequences share one."""
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=12)
    codes, scales = ref.fill_pools(desc, DEV, 2)
    table = torch.tensor([[0, 1, 2, 3, 4], [0, 5, 6, 7, 8]], dtype=torch.int32, device=DEV)
    lens = [75, 80]
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    w = torch.rand((2, 2, 80), device=DEV)
    kept, kl = uq.select_tokens(w, lens_t, 80, 40, sinks=16, recent=8)
    c2, s2, w2 = codes.clone(), scales.clone(), w.clone()
    uq.compact_kv(desc, kept, kl, lens_t, codes, scales, table, weights=w)
    compact_plain(desc, kept, kl.tolist(), lens, c2, s2, table, w2)
    assert torch.equal(codes, c2) and torch.equal(scales, s2) and torch.equal(w, w2)


def test_compact_bad_pages_stay_in_the_pools(uq):
    """Page ids outside the pools: read as page 0, not written."""
    desc = uq.CacheDesc(num_kv_heads=1, num_pages=6)
    codes, scales = ref.fill_pools(desc, DEV, 3)
    table = torch.tensor([[1, 99, 2, -5]], dtype=torch.int32, device=DEV)
    kept = torch.arange(0, 64, 2, dtype=torch.int32, device=DEV).view(1, 1, 32)
    before = codes.clone()
    uq.compact_kv(desc, kept, torch.tensor([32], dtype=torch.int32, device=DEV),
                  torch.tensor([64], dtype=torch.int32, device=DEV), codes, scales, table)
    torch.cuda.synchronize()
    pages = codes.view(6, -1)
    same = [p for p in range(6) if torch.equal(pages[p], before.view(6, -1)[p])]
    assert same == [0, 2, 3, 4, 5]


def test_select_and_compact_from_a_graph(uq):
    """Both calls captured, replayed with eager work between."""
    lens = [500, 90, 300]
    table, pages = ref.tables(lens, DEV, 9)
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=pages)
    start = ref.fill_pools(desc, DEV, 9)
    codes, scales = (x.clone() for x in start)
    w0 = torch.rand((3, 2, 500), device=DEV)
    w = w0.clone()
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    freed, count = torch.zeros(table.numel(), dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)

    def both():
        kept, kl = uq.select_tokens(w, lens_t, 500, 100, sinks=2, recent=9)
        uq.compact_kv(desc, kept, kl, lens_t, codes, scales, table, weights=w, freed_pages=freed, freed_count=count)
        return kept, kl

    both()
    want = [x.clone() for x in (codes, scales, w, freed, count)]
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        both()
    for _ in range(3):
        codes.copy_(start[0])
        scales.copy_(start[1])
        w.copy_(w0)
        freed.zero_()
        torch.cuda.synchronize()
        gr.replay()
        torch.cuda.synchronize()
        for x, y in zip((codes, scales, w, freed, count), want):
            assert torch.equal(x, y)
