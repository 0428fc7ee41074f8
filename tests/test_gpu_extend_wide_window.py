"""uq_extend_attention under windows and first tokens as wide as int32 holds: the
same tokens are visible as without a window, also to sequences with more
queries than context, whose first positions are negative."""
import pytest
import torch

import serving_ref as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
MOST = 2147483647


@pytest.fixture(scope="module")
def uq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_20474_amd import uq as mod
    return mod


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("lens,news", [([3, 0, 20], [6, 4, 20]), ([3, 150, 700], [300, 400, 90]), ([0], [7]), ([1], [70])])
@pytest.mark.parametrize("window,sinks", [(MOST, 0), (MOST, MOST), (MOST - 1, 3), (MOST - 70, 1), (40, MOST), (1, MOST - 5)])
def test_everything_is_visible(uq, d, lens, news, window, sinks):
    print(f"d {d} lens {lens} news {news} window {window} sinks {sinks}", flush=True)
    table, pages = ref.tables(lens, DEV, 5)
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=pages, head_dim=d)
    codes, scales = ref.fill_pools(desc, DEV, 5)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    cu = [sum(news[:i]) for i in range(len(news) + 1)]
    q = torch.randn((cu[-1], 8, d), generator=torch.Generator(device=DEV).manual_seed(d), device=DEV)
    args = (desc, q, i32(cu), codes, scales, table, i32(lens), max(lens))
    got = uq.extend_attention(*args, window=window, sinks=sinks, out_dtype=torch.float32)
    plain = uq.extend_attention(*args, out_dtype=torch.float32)
    want = ref.attend(desc, ref.pool_values(desc, codes, scales), q, cu, table, lens)
    for x in (got, plain):
        assert float((x.double() - want).norm()) <= 1e-3 * float(want.norm())
    # position below 0: nothing is visible
    for b, (n, m) in enumerate(zip(lens, news)):
        assert torch.all(got[cu[b]:cu[b] + max(m - n, 0)] == 0)
        assert n == 0 or torch.all(got[cu[b] + max(m - n, 0):cu[b + 1]].abs().amax((1, 2)) > 0)


def test_long_windows_split_over_blocks(uq):
    lens, news = [9000, 2], [5, 9]
    table, pages = ref.tables(lens, DEV, 6)
    desc = uq.CacheDesc(num_kv_heads=1, num_pages=pages)
    codes, scales = ref.fill_pools(desc, DEV, 6)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    cu = [0, 5, 14]
    q = torch.randn((14, 8, 128), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV)
    want = ref.attend(desc, ref.pool_values(desc, codes, scales), q, cu, table, lens)
    for window, sinks in ((MOST, 0), (9000, MOST), (8999, MOST)):
        got = uq.extend_attention(desc, q, i32(cu), codes, scales, table, i32(lens), 9000, window=window, sinks=sinks,
                                  out_dtype=torch.float32)
        assert float((got.double() - want).norm()) <= 1e-3 * float(want.norm())
