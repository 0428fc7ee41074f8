"""uq_extend_attention where most of the weight is on one token whose value is
small, as on a first token that every query attends to: the output is then the
sum of many weights far below the largest one.

The tail's scores are Gaussian, about `gap` powers of two below the peak's.
Queries are FP8 of 4 significant bits and keys multiples of 2^-4, so that every
score is exact and only the weights' precision is left.  A weight keeps 11 bits
(cut, the mean loss given back): at most 6.3e-4 of it either way.  Below 2^-5 of
the largest of its 32 tokens it may be off by 2^-15 of that one, half of it on
average: of 31 tokens at that border, each 2^-16 of a sum that is 2 times the largest,
2.4e-4.  Values have random signs, so that the errors of a sum are to the sum at
most as those of its terms to the terms: 6.3e-4 + 2.4e-4 < 1e-3, the library's
bar, here for every token's row.
"""
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


def batch(uq, d, n, gap, seqs, new, group, hkv, peaks, seed, window=0, sinks=0, v_down=10, sharp=0):
    """`seqs` sequences of `new` queries over the same n tokens; `peaks`: the tokens with the weight, but for
    the last `sharp` heads of a group, whose scores are spread over many powers of two."""
    print(f"d {d} n {n} gap {gap} sequences {seqs} x {new} heads {group * hkv}/{hkv} peaks {peaks} window {window} "
          f"sinks {sinks} v_down {v_down}", flush=True)
    table, pages = ref.tables([n], DEV, seed)
    desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=pages, rotate_v=False, head_dim=d)
    codes, scales = ref.fill_pools(desc, DEV, seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    sign = torch.randint(0, 2, (hkv, d), generator=g, device=DEV)
    c = codes.view(pages, hkv, 2, 8 * d)
    s = scales.view(pages, hkv, 2, d // 32, 16)
    s[:, :, 0] = 127 - 3
    nib = (6 + 8 * sign).to(torch.uint8)                       # 4 with the query's sign
    pair = nib[:, 0::2] | (nib[:, 1::2] << 4)
    for t in peaks:
        page, off = int(table[0, t // 16]), t % 16
        c[page, :, 0].view(hkv, d // 32, 16, 16)[:, :, off] = pair.view(hkv, d // 32, 16)
        s[page, :, 0, :, off] = 127 - 2
        s[page, :, 1, :, off] -= v_down
    T = seqs * new
    mag = 1 + torch.randint(0, 4, (T, hkv, group, d), generator=g, device=DEV) / 8
    q = mag * (1 - 2 * sign[:, None, :])
    if sharp:
        q[:, :, group - sharp:] = 8 * mag[:, :, group - sharp:] * (
            1 - 2 * torch.randint(0, 2, (hkv, sharp, d), generator=g, device=DEV))
    q = q.reshape(T, hkv * group, d)
    q8 = q.to(torch.float8_e4m3fn)
    assert torch.equal(q8.float(), q)
    # the peak's score is the sum of the magnitudes, about 1.1875 d: `gap` powers of two
    scale = gap * 0.6931471805599453 / (1.1875 * d)
    tables = table.expand(seqs, -1).contiguous()
    lens, cu = [n] * seqs, list(range(0, T + 1, new))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    out = uq.extend_attention(desc, q8.view(torch.uint8), i32(cu), codes, scales, tables, i32(lens), n, window=window,
                              sinks=sinks, softmax_scale=scale, out_dtype=torch.float32)
    torch.cuda.synchronize()
    kv = ref.pool_values(desc, codes, scales)
    want = ref.attend(desc, kv, q8.view(torch.uint8), cu, tables, lens, window, sinks, scale=scale, prepared=True)
    rel = (out.double() - want).norm(dim=-1) / want.norm(dim=-1)
    print(f"  rel mean {float(rel.mean()):.2e} worst {float(rel.max()):.2e}", flush=True)
    assert float((out.double() - want).norm() / want.norm()) <= REL
    assert float(((out.double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)).max()) <= REL
    return desc, codes, scales, tables, i32(lens), q8, scale, out


# few rows split over blocks, more rows split, shares of one length, whole walks of few and of more rows
LAYOUTS = {"few": (1, 5, 8, 1), "rows": (1, 40, 8, 1), "shares": (3, 2, 8, 1), "whole-few": (64, 1, 8, 8),
           "whole-rows": (64, 9, 8, 8)}


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("window,sinks", [(0, 0), (12000, 4)])
def test_peak_first(uq, d, layout, window, sinks):
    batch(uq, d, 16384, 23.0, *LAYOUTS[layout], [0], seed=d, window=window, sinks=sinks)


@pytest.mark.parametrize("layout", ["few", "whole-rows"])
@pytest.mark.parametrize("n,gap", [(8192, 16), (32768, 16), (32768, 18), (131072, 20), (131072, 28), (16384, 17.3),
                                   (16384, 20.2), (65536, 30)])
def test_how_far_below(uq, layout, n, gap):
    batch(uq, 128, n, float(gap), *LAYOUTS[layout], [0], seed=n)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("layout", ["few", "rows", "whole-rows"])
@pytest.mark.parametrize("peaks", [[8000], [16000], [0, 5, 7000, 7001, 16383 - 41]])
def test_peaks_along_the_context(uq, d, layout, peaks):
    batch(uq, d, 16384, 22.0, *LAYOUTS[layout], peaks, seed=d + 1)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_wide_scores(uq, d):
    """Scores over many powers of two, so that the weights of one 32 tokens and of the next lie far apart."""
    batch(uq, d, 8192, 150.0, 1, 40, 8, 1, [0, 4000], seed=d + 2, v_down=0)
    batch(uq, d, 8192, 60.0, 1, 5, 8, 1, [4000], seed=d + 3, v_down=0)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("layout", ["few", "rows", "whole-rows"])
@pytest.mark.parametrize("peaks", [[0], [0, 7000]])
def test_heads_of_two_kinds(uq, d, layout, peaks):
    """Heads whose weight is on a peak with small values next to sharp ones, in the rows of one wave."""
    batch(uq, d, 16384, 22.0, *LAYOUTS[layout], peaks, seed=d + 4, sharp=4)


def test_prompt_and_decode_agree(uq):
    """The same token as one query of a step and as decode attention."""
    for seed, gap in ((5, 20.0), (6, 26.0)):
        desc, codes, scales, table, lens, q8, scale, out = batch(uq, 128, 32768, gap, 64, 1, 8, 8, [0], seed=seed)
        one = uq.decode_attention(desc, q8.view(torch.uint8), codes, scales, table, lens, 32768, softmax_scale=scale)
        assert float(((one - out).norm(dim=-1) / one.norm(dim=-1)).max()) <= REL
