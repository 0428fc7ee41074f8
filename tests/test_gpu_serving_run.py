"""The calls around the cache as a serving engine uses them: several steps of
a ragged batch through plan_tokens, norm_rope_write, extend_attention,
decode_window and read_kv, eagerly, captured in a graph, and two at a time on
two streams; batches that mix long and short sequences; pools beyond 2^32
bytes.

Attention is compared with the 64-bit form on the bytes the step itself left
in the cache and on the prepared queries, with the tolerances of
test_gpu_extend.py (1e-3) and of decode attention (1e-3).  What one call
computes twice, eagerly and in a replay or on two streams, has to be equal bit
for bit: no call uses atomics on floats, and its grid does not depend on the
device's state.
"""
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


def i32(x, dev):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def close(got, want, tol, what):
    rel = float((got.double() - want).norm() / want.norm().clamp(min=1e-300))
    log(f"  {what}: rel {rel:.2e}")
    assert rel <= tol, what


class Engine:
    """A toy model step: one layer, everything a step needs allocated once."""

    def __init__(self, uq, dev, B, T, hq, hkv, d, mpps, pages, free, window, sinks, seed):
        self.uq, self.dev, self.B, self.T, self.window, self.sinks = uq, dev, B, T, window, sinks
        self.bound = mpps * 16
        self.desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=pages, rotate_v=True, head_dim=d)
        self.codes, self.scales = self.desc.alloc_pools(dev, fill=0xA5)
        self.table = torch.full((B, mpps), -1, dtype=torch.int32, device=dev)
        self.free = i32(free, dev)
        self.plan = uq.TokenPlan.alloc(B, T, dev)
        self.cached, self.new = i32([0] * B, dev), i32([0] * B, dev)
        g = torch.Generator(device=dev).manual_seed(seed)
        self.g = g
        half = d // 4
        ang = torch.arange(self.bound, device=dev)[:, None] * 10000.0 ** (-torch.arange(half, device=dev) / half)
        self.spec = uq.NormRope(positions=self.plan.positions,
                                cos_sin=torch.cat([ang.cos(), ang.sin()], 1).float().contiguous(),
                                q_weight=torch.rand(d, generator=g, device=dev) + 0.5,
                                k_weight=torch.rand(d, generator=g, device=dev) + 0.5)
        self.qkv = torch.empty((T, hq + 2 * hkv, d), dtype=torch.bfloat16, device=dev)
        self.q, self.k, self.v = self.qkv[:, :hq], self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:]
        self.q8 = torch.zeros((T, hq, d), dtype=torch.uint8, device=dev)
        self.out = torch.full((T, hq, d), 7.0, dtype=torch.float32, device=dev)
        self.back = torch.full((2, T, hkv, d), 7.0, dtype=torch.float32, device=dev)
        n = uq.extend_workspace_bytes(self.desc, T, B, hq, self.bound, window, sinks)
        self.work = torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device=dev)

    def feed(self, cached, new, free):
        self.cached.copy_(i32(cached, self.dev))
        self.new.copy_(i32(new, self.dev))
        self.free.copy_(i32(free, self.dev))
        self.qkv.copy_(torch.randn(self.qkv.shape, generator=self.g, device=self.dev))

    def step(self):
        uq = self.uq
        uq.plan_tokens(self.cached, self.new, self.free, self.table, self.plan)
        uq.norm_rope_write(self.desc, self.spec, self.q, self.k, self.v, self.plan.slots, self.codes, self.scales,
                           q_out=self.q8)
        uq.extend_attention(self.desc, self.q8, self.plan.cu_seqlens, self.codes, self.scales, self.table,
                            self.plan.context_lens, self.bound, window=self.window, sinks=self.sinks,
                            workspace=self.work, out=self.out)
        uq.read_kv(self.desc, self.plan.slots, self.codes, self.scales, k_out=self.back[0], v_out=self.back[1])

    def state(self):
        return [t.clone() for t in (self.table, self.plan.context_lens, self.plan.cu_seqlens, self.plan.positions,
                                    self.plan.slots, self.plan.result, self.codes, self.scales, self.q8, self.out,
                                    self.back)]


STEPS = [[37, 0, 250, 5, 64], [1, 16, 1, 1, 1], [3, 3, 3, 3, 3], [0, 80, 1, 1, 0], [1, 1, 1, 400, 1], [1, 1, 1, 1, 1]]


def replay_lengths(steps, free, mpps, T):
    """The lengths an engine would feed, from the plain plan: (cached, new, free list) per step."""
    B = len(steps[0])
    cached, table = [0] * B, [[-1] * mpps for _ in range(B)]
    free = list(free)
    for new in steps:
        yield list(cached), list(new), list(free), table
        got = ref.plan(cached, new, free, table, T)
        cached = [c + n if got["context"][b] or c + n == 0 else c for b, (c, n) in enumerate(zip(cached, new))]
        free = free[got["result"][1]:]


@pytest.mark.parametrize("d,hq,hkv", [(64, 8, 2), (128, 8, 1), (128, 16, 4), (256, 4, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (48, 4)])
def test_steps_of_a_batch(uq, d, hq, hkv, window, sinks):
    dev = torch.device("cuda:0")
    mpps, T, pages = 24, 400, 80
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(d + hq)).tolist()
    e = Engine(uq, dev, 5, T, hq, hkv, d, mpps, pages, perm, window, sinks, seed=d)
    other = e.desc.alloc_pools(dev, fill=0xA5)
    for i, (cached, new, free, table) in enumerate(replay_lengths(STEPS, perm, mpps, T)):
        log(f"step {i}: cached {cached} new {new} free {len(free)} d {d} heads {hq}/{hkv} window {window}")
        e.free = i32(free, dev)
        e.feed(cached, new, free)
        e.out.fill_(7.0)
        e.back.fill_(7.0)
        e.step()
        torch.cuda.synchronize()
        host = [row[:] for row in table]
        want = ref.plan(cached, new, free, host, T)
        p = e.plan
        for got, key in ((p.context_lens, "context"), (p.cu_seqlens, "cu"), (p.positions, "pos"), (p.slots, "slots"),
                         (p.seq_ids, "seq"), (p.result, "result")):
            assert got.tolist() == want[key], key
        assert e.table.tolist() == host

        # the cache: the rows, then the write call on the same slots
        q32, k32 = uq.norm_rope(e.spec, e.q, e.k, out_dtype=torch.float32)
        uq.quantize_kv(e.desc, k32, e.v.float().contiguous(), p.slots, *other)
        assert torch.equal(e.codes, other[0]) and torch.equal(e.scales, other[1])
        rows = ref.norm_rope(e.q, e.spec.q_weight, e.spec.eps, p.positions, e.spec.cos_sin, False)
        # FP8 borders may round the other way: a step of 2^-3 of few elements, far below half a step of all
        close(e.q8.view(torch.float8_e4m3fn).double(), ref.e4m3(ref.walsh(rows)), 5e-3, "queries")

        kv = ref.pool_values(e.desc, e.codes, e.scales)
        live = p.slots >= 0
        close(e.back[0][live], ref.walsh(kv[0][p.slots[live]]), 2e-6, "K back")
        close(e.back[1][live], ref.walsh(kv[1][p.slots[live]]), 2e-6, "V back")
        assert torch.all(e.back[:, ~live] == 7.0)

        n = want["cu"][-1]
        exp = ref.attend(e.desc, kv, e.q8, want["cu"], e.table, want["context"], window, sinks, prepared=True)
        close(e.out[:n], exp[:n], REL, "attention")
        assert torch.all(e.out[n:] == 7.0)
        ends = i32([c - 1 for c in want["cu"][1:]], dev).long()
        last = [b for b in range(5) if want["context"][b] > 0 and new[b] > 0]
        if window and last:
            q1 = (e.q8 if d == 128 else q32)[ends].contiguous()   # decode takes prepared queries at head size 128
            one = uq.decode_window(e.desc, q1, e.codes, e.scales, e.table, p.context_lens, e.bound, window, sinks)
            close(one[last], exp[ends[last]], REL, "last tokens by decode_window")


def test_a_step_in_a_graph(uq):
    """Every replay against the eager step on a second engine in the same state."""
    dev = torch.device("cuda:0")
    mpps, T, pages = 30, 300, 120
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).tolist()
    steps = [[37, 0, 200, 5, 58], [1, 16, 1, 1, 1], [3, 3, 3, 3, 3], [1, 1, 1, 1, 1], [0, 250, 0, 40, 1], [1] * 5]
    a, b = (Engine(uq, dev, 5, T, 8, 2, 128, mpps, pages, perm, 0, 0, seed=2) for _ in range(2))
    # warm up and capture with nothing to do: no new token, nothing written
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for i, (cached, new, free, _) in enumerate(replay_lengths(steps, perm, mpps, T)):
        log(f"replay {i}: cached {cached} new {new}")
        free = free + [free[-1]] * (pages - len(free))   # one array of one length; its tail is never reached
        for e in (a, b):
            e.feed(cached, new, free)
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x, y), i
        # eager work on the workspace and outputs the graph uses
        a.work.fill_(0xFF)
        a.uq.extend_attention(a.desc, a.q8, a.plan.cu_seqlens, a.codes, a.scales, a.table, a.plan.context_lens,
                              a.bound, workspace=a.work, out=a.out)
        torch.cuda.synchronize()
        assert torch.equal(a.out, b.out)


def test_window_decode_and_rows_in_a_graph(uq):
    dev = torch.device("cuda:0")
    lens = [5000, 17, 1, 900]
    table, pages = ref.tables(lens, dev, 3)
    desc = uq.CacheDesc(num_kv_heads=1, num_pages=pages, rotate_v=True, head_dim=128)
    codes, scales = ref.fill_pools(desc, dev, 3)
    ctx = i32(lens, dev)
    q = torch.zeros((4, 8, 128), device=dev)
    w = torch.ones(128, device=dev)
    spec = uq.NormRope(q_weight=w)
    rows, out = torch.empty_like(q), torch.empty_like(q)
    work = torch.empty(uq.decode_window_workspace_bytes(desc, 4, 8, 5000, 2000, 4), dtype=torch.uint8, device=dev)

    def run(rows, out):
        uq.norm_rope(spec, q, q_out=rows)
        uq.decode_window(desc, rows, codes, scales, table, ctx, 5000, 2000, 4, workspace=work, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(rows, out)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(rows, out)
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator(device=dev).manual_seed(i), device=dev))
        ctx.copy_(i32([5000 - i, 17, 1 + i, 900], dev))
        work.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        rows2, out2 = torch.empty_like(q), torch.empty_like(q)
        run(rows2, out2)
        torch.cuda.synchronize()
        assert torch.equal(rows, rows2) and torch.equal(out, out2), i


def test_two_streams_at_once(uq):
    """Two engines on two streams, their steps interleaved by the host without a wait between."""
    dev = torch.device("cuda:0")
    mpps, T, pages = 60, 700, 200
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(4)).tolist()
    steps = [[300, 1, 250, 5, 64], [1, 16, 1, 1, 1], [3, 3, 3, 3, 3], [80, 80, 80, 80, 80]]
    engines = [Engine(uq, dev, 5, T, 8, 2, 128, mpps, pages, perm, w, 0, seed=5 + w) for w in (0, 100, 0, 100)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for cached, new, free, _ in replay_lengths(steps, perm, mpps, T):
        log(f"cached {cached} new {new}")
        free = free + [free[-1]] * (pages - len(free))
        for e in engines:
            e.feed(cached, new, free)
        torch.cuda.synchronize()
        for e, s in zip(engines[:2], streams):
            with torch.cuda.stream(s):
                e.step()
        torch.cuda.synchronize()
        for e in engines[2:]:
            e.step()
            torch.cuda.synchronize()
        for x, y in ((engines[0], engines[2]), (engines[1], engines[3])):
            for s, t in zip(x.state(), y.state()):
                assert torch.equal(s, t)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 5)])
@pytest.mark.parametrize("few", [1, 7])
def test_long_and_short_sequences_together(uq, d, window, sinks, few):
    """Few rows a sequence on average, so waves split the tokens of the short ones and share the long one's."""
    dev = torch.device("cuda:0")
    lens = [40 + 37 * i for i in range(60)] + [900, 16]
    news = [few] * 60 + [200, 9]
    table, pages = ref.tables(lens, dev, 11)
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=pages, rotate_v=False, head_dim=d)
    codes, scales = ref.fill_pools(desc, dev, 11)
    cu = [0]
    for m in news:
        cu.append(cu[-1] + m)
    for order in (1, -1):
        perm = list(range(62))[::order]
        t2, l2 = table[i32(perm, dev).long()].contiguous(), [lens[b] for b in perm]
        c2 = [0]
        for b in perm:
            c2.append(c2[-1] + news[b])
        q = torch.randn((cu[-1], 6, d), generator=torch.Generator(device=dev).manual_seed(few), device=dev)
        out = uq.extend_attention(desc, q, i32(c2, dev), codes, scales, t2, i32(l2, dev), max(lens), window=window,
                                  sinks=sinks, out_dtype=torch.float32)
        want = ref.attend(desc, ref.pool_values(desc, codes, scales), q, c2, t2, l2, window, sinks)
        close(out, want, REL, f"d {d} few {few} window {window} order {order}")
        worst = ((out - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)).max()
        assert worst <= 20 * REL


@pytest.mark.parametrize("d", [64, 128, 256])
def test_pools_beyond_32_bits(uq, d):
    """The same pages at the end of a pool of more than 2^32 bytes of codes give the same bits."""
    dev = torch.device("cuda:0")
    hkv, lens, news = 2, [400, 33, 1], [60, 33, 1]
    table, pages = ref.tables(lens, dev, 12)
    small = uq.CacheDesc(num_kv_heads=hkv, num_pages=pages, rotate_v=True, head_dim=d)
    far = 2 ** 32 // (small.codes_bytes() // pages) + 5
    big = uq.CacheDesc(num_kv_heads=hkv, num_pages=far + pages, rotate_v=True, head_dim=d)
    assert far * (small.codes_bytes() // pages) > 2 ** 32
    codes, scales = ref.fill_pools(small, dev, 12)
    codes2 = torch.empty(big.codes_bytes(), dtype=torch.uint8, device=dev)
    scales2 = torch.empty(big.scales_bytes(), dtype=torch.uint8, device=dev)
    ctx, cu, table2 = i32(lens, dev), i32([0, 60, 93, 94], dev), torch.where(table >= 0, table + far, table)
    g = torch.Generator(device=dev).manual_seed(d)
    q, k, v = (torch.randn((94, h, d), generator=g, device=dev) for h in (8, hkv, hkv))
    slots = torch.randperm(pages * 16, generator=torch.Generator().manual_seed(d))[:94].to(dev)
    c0, s0 = codes2[-small.codes_bytes():], scales2[-small.scales_bytes():]
    c0.copy_(codes)
    s0.copy_(scales)
    results = []
    for desc, c, s, t, off in ((small, codes, scales, table, 0), (big, codes2, scales2, table2, far * 16)):
        log(f"d {d} pages {desc.num_pages}")
        q8 = uq.norm_rope_write(desc, uq.NormRope(), q, k, v, slots + off, c, s)
        out = uq.extend_attention(desc, q8, cu, c, s, t, ctx, 400, out_dtype=torch.float32)
        one = uq.decode_window(desc, q[:3].contiguous(), c, s, t, ctx, 400, 100, 2)
        back = uq.read_kv(desc, slots + off, c, s, out_dtype=torch.float32)
        results.append([q8, out, one, *back])
    torch.cuda.synchronize()
    for x, y in zip(*results):
        assert torch.equal(x, y)
    assert torch.equal(c0, codes) and torch.equal(s0, scales)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hkv", [1, 3, 8])
def test_few_queries_over_contexts_of_all_lengths(uq, d, hkv):
    """Contexts split into shares of one length: one far above the others, empty ones, no rows, more queries
    than context."""
    dev = torch.device("cuda:0")
    lens = [9000, 0, 30, 3, 700, 2500, 1, 4000]
    news = [3, 1, 0, 5, 8, 2, 1, 4]
    table, pages = ref.tables(lens, dev, 13)
    desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=pages, rotate_v=True, head_dim=d)
    codes, scales = ref.fill_pools(desc, dev, 13)
    kv = ref.pool_values(desc, codes, scales)
    for step in range(2):
        cu = [0]
        for m in news:
            cu.append(cu[-1] + m)
        q = torch.randn((cu[-1] + 2, 4 * hkv, d), generator=torch.Generator(device=dev).manual_seed(d), device=dev)
        out = torch.full(q.shape, 7.0, device=dev)
        uq.extend_attention(desc, q, i32(cu, dev), codes, scales, table, i32(lens, dev), 9000, out=out)
        want = ref.attend(desc, kv, q, cu, table, lens)[:cu[-1]]
        assert torch.all(out[cu[-1]:] == 7.0)
        got = out[:cu[-1]]
        close(got, want, REL, f"d {d} heads {hkv}")
        norm = want.flatten(1).norm(dim=1)
        worst = ((got - want).flatten(1).norm(dim=1)[norm > 0] / norm[norm > 0]).max()
        assert worst <= 20 * REL
        assert torch.all(got[norm == 0] == 0)
        news = news[::-1]
