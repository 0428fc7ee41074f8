"""uq_token_weights against the softmax weights summed in 64 bits over the same
cache bytes and FP8 queries.

Tolerance, elementwise and relative.  A score is off by the QK instruction's error,
at most eta = scale 2^-12.5 max|q| max|k| on operands like these
(tests/test_gpu_instruction_precision.py), which moves a weight by eta in its
exponential and by as much in the row's sum.  In fp32: the argument of the
exponential is rounded to half a step, |x| 2^-24 ln 2, and weights below 2^-60 of the
row's largest are not looked at, so 2^-18; the exponential and the two products behind it 4
steps of 2^-23; the sums, added one after another, (n / 4 + rows / 4 + 16) half steps of
2^-24.
"""
import math

import pytest
import torch

import serving_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def uq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_20474_amd import uq as mod
    return mod


def log(msg):
    print(msg, flush=True)


DEV = "cuda:0"


def expected(k_all, q8, cu, table, lens, hkv, last, causal, scale):
    """Weights [B][Hkv] -> tensors of n values, in 64 bits."""
    out, g = [], q8.shape[1] // hkv
    for b, n in enumerate(lens):
        m = max(0, cu[b + 1] - cu[b])
        use = min(m, last) if last else m
        t = torch.arange(n, device=DEV)
        slot = table[b].long()[t // 16] * 16 + t % 16
        q = q8[cu[b + 1] - use:cu[b + 1]] if use else q8[:0]
        pos = torch.arange(n - use, n, device=DEV)[:, None]
        rows = []
        for h in range(hkv):
            s = (q[:, h * g:(h + 1) * g].transpose(0, 1).reshape(-1, q.shape[2]) @ k_all[slot, h].t().contiguous()) * scale
            s = s.reshape(g, use, n)
            if causal:
                s = s.masked_fill(t > pos, -math.inf)
            e = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-1e300)) if n else s
            rows.append((e / e.sum(-1, keepdim=True).clamp(min=1e-300)).sum((0, 1)))
        out.append(rows)
    return out


class Case:
    def __init__(self, uq, lens, news, hq, hkv, d, seed, last=0, causal=True, pad=0, bound=0, width_pad=0, gain=1.5,
                 scale=None, table_width=None, poison=True):
        log(f"lens {lens} news {news} heads {hq}/{hkv} d {d} last {last} causal {causal} seed {seed}")
        self.uq, self.lens, self.hkv, self.last, self.causal = uq, lens, hkv, last, causal
        self.scale = d ** -0.5 if scale is None else scale
        self.bound = max(bound, *lens, 0)
        self.table, pages = ref.tables(lens, DEV, seed, width=max(1, -(-self.bound // 16), table_width or 0))
        self.desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=pages, head_dim=d)
        self.codes, self.scales = ref.fill_pools(self.desc, DEV, seed)
        self.k = ref.pool_values(self.desc, self.codes, self.scales)[0]
        if poison:   # slots behind a context: scale bytes that stand for NaN
            sc = self.scales.view(pages, hkv, 2, d // 32, 16)
            for b, n in enumerate(lens):
                if n > 0 and n % 16:
                    sc[self.table[b, n // 16].long(), :, :, :, n % 16:] = 255
        self.cu = [0]
        for m in news:
            self.cu.append(self.cu[-1] + m)
        g = torch.Generator(device=DEV).manual_seed(seed + 1)
        rows = torch.randn((self.cu[-1] + pad, hq, d), generator=g, device=DEV) * gain
        self.q = rows.clamp(-448, 448).to(torch.float8_e4m3fn)
        self.rows = max([1] + [min(m, last) if last else m for m in news]) * (hq // hkv)
        self.before = torch.rand((len(lens), hkv, self.bound + width_pad), generator=g, device=DEV) * 0.01
        self.cu_t = torch.tensor(self.cu, dtype=torch.int32, device=DEV)
        self.lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)

    def call(self, q=None, weights=None, **kw):
        w = self.before.clone() if weights is None else weights
        return self.uq.token_weights(self.desc, self.q if q is None else q, self.cu_t, self.codes, self.scales, self.table,
                                     self.lens_t, self.bound, w, last=self.last, causal=self.causal,
                                     softmax_scale=self.scale, **kw)

    def check(self, got=None):
        got = self.call() if got is None else got
        torch.cuda.synchronize()
        q8 = self.q.double()
        want = expected(self.k, q8, self.cu, self.table, self.lens, self.hkv, self.last, self.causal, self.scale)
        eta = self.scale * 2 ** -12.5 * float(q8.abs().max() if q8.numel() else 0) * float(self.k.abs().max())
        tol = 2 * eta + 2 ** -18 + 4 * 2 ** -23 + (max(self.lens) / 4 + self.rows / 4 + 16) * 2 ** -24
        worst = 0.0
        for b, n in enumerate(self.lens):
            assert torch.equal(got[b, :, n:], self.before[b, :, n:]), f"sequence {b}: entries behind the context changed"
            for h in range(self.hkv):
                w = self.before[b, h, :n].double() + want[b][h]
                err = ((got[b, h, :n].double() - w).abs() / w.clamp(min=2 ** -60)).max().item() if n else 0.0
                worst = max(worst, err)
        log(f"worst relative error {worst:.2e}, bound {tol:.2e}")
        assert worst <= tol
        return got


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(8, 8), (10, 2), (16, 1), (24, 2)])
def test_single_queries(uq, d, hq, hkv):
    Case(uq, [1, 15, 16, 17, 33, 500, 1300, 2], [1] * 8, hq, hkv, d, seed=d + hq).check()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (10, 2), (16, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_several_queries(uq, d, hq, hkv, causal):
    Case(uq, [40, 17, 300, 1, 700], [40, 5, 130, 1, 33], hq, hkv, d, seed=3 * d + hq, causal=causal).check()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("last", [1, 7, 50])
def test_last_queries(uq, d, last):
    # sequences with fewer queries than `last`, as many and more; rows by sequence and by token row
    Case(uq, [400, 60, 90], [300, 7, 50], 12, 2, d, seed=d + last, last=last).check()
    Case(uq, [64, 60], [30, 3], 12, 2, d, seed=d + last, last=last).check()


def test_prompt_alone(uq):
    Case(uq, [1500], [1500], 12, 2, 128, seed=4).check()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_long_context_few_heads(uq, d):
    # contexts in chunks, rows in splits
    Case(uq, [9000, 4100], [60, 3], 8, 1, d, seed=d).check()


def test_chunks_of_many_rows(uq):
    Case(uq, [6000], [700], 16, 1, 128, seed=5).check()


def test_many_sequences(uq):
    lens = [(37 * i) % 150 for i in range(150)]
    news = [min(n, i % 4) for i, n in enumerate(lens)]
    Case(uq, lens, news, 6, 2, 128, seed=6, pad=9, bound=400, width_pad=13).check()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_single_tokens_beside_a_prompt(uq, d):
    Case(uq, [700, 3000, 45, 16, 900], [700, 1, 1, 1, 2], 8, 2, d, seed=20 + d).check()


def test_empty_sequences_and_rows_that_see_nothing(uq):
    # no context, no queries, more queries than context: the ones before its start see nothing
    Case(uq, [0, 30, 5, 0, 20], [3, 0, 12, 0, 2], 8, 2, 128, seed=7, pad=4, bound=64).check()
    Case(uq, [0, 30, 5, 0, 20], [3, 0, 12, 0, 2], 8, 2, 128, seed=7, pad=4, causal=False, bound=64).check()


def test_no_tokens_at_all(uq):
    c = Case(uq, [0, 0], [1, 2], 8, 2, 128, seed=7, bound=16)
    assert torch.equal(c.call(), c.before)


def test_sums_to_the_rows(uq):
    """Every row gives 1 in all: G queries per KV head and query."""
    c = Case(uq, [700, 90], [33, 90], 16, 4, 128, seed=8)
    got = c.call(weights=torch.zeros_like(c.before)).double().sum(-1)
    want = torch.tensor([33 * 4, 90 * 4], dtype=torch.float64, device=DEV)[:, None]
    # rows add up to 1 within the rounding of their weights and of the row's sum
    assert ((got - want).abs() / want).max().item() <= 2 ** -18 + 8 * 2 ** -23 + (700 / 4 + 90) * 2 ** -24


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_rows_are_prepared_as_the_writer_does(uq, d, dtype):
    """Rows in any type, with a token stride: the bits of the call with prepared queries."""
    c = Case(uq, [90, 300], [9, 21], 8, 2, d, seed=d)
    g = torch.Generator(device=DEV).manual_seed(9)
    rows = torch.randn((c.cu[-1], 11, d), generator=g, device=DEV).to(dtype)[:, :8]
    pools = c.desc.alloc_pools(DEV, fill=0)
    kv = torch.zeros((c.cu[-1], 2, d), dtype=dtype, device=DEV)
    prepared = uq.norm_rope_write(c.desc, uq.NormRope(), rows, kv, kv,
                                  torch.full((c.cu[-1],), -1, dtype=torch.int64, device=DEV), *pools)
    assert torch.equal(c.call(q=rows), c.call(q=prepared))


def test_strided_prepared_rows(uq):
    c = Case(uq, [90, 300], [9, 21], 8, 2, 128, seed=2)
    wide = torch.full((c.cu[-1], 10, 128), 0x7F, dtype=torch.uint8, device=DEV)
    wide[:, :8] = c.q.view(torch.uint8)
    assert torch.equal(c.call(q=wide[:, :8]), c.check())


@pytest.mark.parametrize("d", [64, 128, 256])
def test_large_scores(uq, d):
    """Scores beyond 2^20: one token of each row has all the weight."""
    c = Case(uq, [50, 333, 7], [4, 20, 1], 8, 2, d, seed=11, scale=1e16)
    got = c.call(weights=torch.zeros_like(c.before))
    want = expected(c.k, c.q.double(), c.cu, c.table, c.lens, 2, 0, True, 1e16)
    for b, n in enumerate(c.lens):
        for h in range(2):
            assert torch.equal(got[b, h, :n].double(), want[b][h])


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("m", [1, 60])
def test_scores_that_climb(uq, d, m):
    """Later tokens' scores are up to hundreds of powers of two above the first ones', in fp32's
    range: products and sums are exact, so the weights are those of the formula to the rounding of
    the exponential and the sums."""
    n = 900
    c = Case(uq, [n], [m], 16, 2, d, seed=19, scale=1.0, poison=False)
    c.codes.fill_(0x22)                                   # every channel 1
    exps = torch.sort(torch.randint(-12, 1, (n,), generator=torch.Generator().manual_seed(d)))[0]
    exps[100:140] = -12                                    # (and back once)
    page, off = c.table[0].long().cpu()[torch.arange(n) // 16], torch.arange(n) % 16
    c.scales.view(c.desc.num_pages, 2, 2, d // 32, 16)[page.to(DEV), :, :, :, off.to(DEV)] = (
        (exps + 127).to(torch.uint8).to(DEV)[:, None, None, None])
    c.q = torch.ones_like(c.q.float()).to(torch.float8_e4m3fn)
    s = d * torch.exp2(exps.double()).to(DEV)
    want = torch.zeros(n, dtype=torch.float64, device=DEV)
    for i in range(m):
        want[:n - m + i + 1] += 8 * torch.softmax(s[:n - m + i + 1], 0)
    got = c.call(weights=torch.zeros_like(c.before))[0].double()
    # |c s| <= 2^9: the product with c = fp32(log2 e) and the exponential's argument are off by 2^-15 each
    tol = 2 ** -13 + (n / 4 + 8 * m / 4 + 16) * 2 ** -24
    for h in range(2):
        assert ((got[h, :n] - want).abs() <= tol * want + 2 ** -60).all()


def test_equal_scores(uq):
    """Queries of 0 spread their weight evenly over what they see."""
    c = Case(uq, [200], [70], 8, 2, 128, seed=12)
    c.q.zero_()
    c.check()


def test_order_does_not_change_bits(uq):
    """The same call twice, into a used workspace, on another stream and replayed
    from a graph."""
    c = Case(uq, [3000, 70, 900], [90, 70, 1], 8, 2, 128, seed=13)
    want = c.check()
    n = uq.token_weights_workspace_bytes(c.desc, c.q.shape[0], 3, 8, c.bound)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
    assert torch.equal(c.call(workspace=ws), want)
    side = torch.cuda.Stream()
    w = c.before.clone()
    side.wait_stream(torch.cuda.current_stream())
    c.call(weights=w, stream=side)
    side.synchronize()
    assert torch.equal(w, want)
    # two graphs that share the workspace, one replayed after the other
    other = Case(uq, [100, 40], [3, 40], 8, 2, 128, seed=14)
    other_want = other.check()
    graphs = []
    for case in (c, other):
        w = case.before.clone()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            case.call(weights=w, workspace=ws)
        graphs.append((gr, w, case.before))
    for _ in range(3):
        for (gr, w, before), expect in zip(graphs, (want, other_want)):
            w.copy_(before)
            gr.replay()
            torch.cuda.synchronize()
            assert torch.equal(w, expect)


def test_accumulates(uq):
    c = Case(uq, [90, 40], [9, 4], 8, 2, 128, seed=15)
    one = c.call(weights=torch.zeros_like(c.before))
    w = torch.zeros_like(c.before)
    for _ in range(2):
        c.call(weights=w)
    # a call adds the sums of at most two blocks of rows one after another, so a weight has been
    # rounded to half a step, 2^-24, at most four times, `one` twice
    assert ((w - (one + one)).abs() <= 6 * 2 ** -24 * (one + one)).all()


def test_tables_wider_than_the_bound(uq):
    Case(uq, [90, 300], [9, 21], 8, 2, 64, seed=16, table_width=50).check()


def test_bound_far_above_the_contexts(uq):
    Case(uq, [90, 300], [1, 1], 8, 2, 128, seed=17, bound=70000).check()


def test_pools_beyond_32_bits(uq):
    """A pool of more than 2^32 bytes of codes, the sequence's pages at its end."""
    h, d = 8, 256
    pages = (1 << 32) // (h * 16 * d) + 40
    desc = uq.CacheDesc(num_kv_heads=h, num_pages=pages, head_dim=d)
    codes = torch.empty(desc.codes_bytes(), dtype=torch.uint8, device=DEV)
    scales = torch.empty(desc.scales_bytes(), dtype=torch.uint8, device=DEV)
    c = Case(uq, [500], [3], 16, h, d, seed=18)
    tail = c.desc.num_pages
    codes[-c.desc.codes_bytes():] = c.codes
    scales[-c.desc.scales_bytes():] = c.scales
    table = torch.where(c.table >= 0, c.table + (pages - tail), c.table)
    w = uq.token_weights(desc, c.q, c.cu_t, codes, scales, table, c.lens_t, c.bound, c.before.clone())
    assert torch.equal(w, c.check())
