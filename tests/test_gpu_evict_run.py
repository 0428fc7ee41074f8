"""Positions with several axes, cross attention and eviction as a serving engine uses
them, together with the calls around the cache: several steps of a batch whose cache
may not grow beyond a budget, eagerly and captured in a graph.

Each step's attention is compared with its 64-bit form on the bytes that the step left in
the cache and on the prepared queries (1e-3, as in test_gpu_extend.py); the weights with the
softmax weights summed in 64 bits (tolerance of test_gpu_token_weights.py); the kept tokens and
the compacted cache with plain indexing (equal).  What a replay computes again has to be
equal bit for bit.
"""
import math

import pytest
import torch

import serving_ref as ref
from test_gpu_evict import chosen, compact_plain
from test_gpu_rope_axes import rotated
from test_gpu_token_weights import expected

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def uq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_20474_amd import uq as mod
    return mod


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Engine:
    """One layer of a model with positions on three axes and a cache of at most `budget` tokens a
    sequence after each step."""

    def __init__(self, uq, B, T, hq, hkv, d, mpps, budget, sinks, recent, seed):
        self.uq, self.B, self.T, self.hq, self.hkv, self.d = uq, B, T, hq, hkv, d
        self.budget, self.sinks, self.recent, self.bound = budget, sinks, recent, mpps * 16
        pages = B * mpps
        self.desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=pages, head_dim=d)
        self.codes, self.scales = self.desc.alloc_pools(DEV, fill=0xA5)
        self.table = torch.full((B, mpps), -1, dtype=torch.int32, device=DEV)
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        self.free = torch.randperm(pages, generator=self.g, device=DEV).int()
        self.plan = uq.TokenPlan.alloc(B, T, DEV)
        self.cached, self.new = i32([0] * B), i32([0] * B)
        half = d // 2
        self.axes = uq.pair_axes_of((half - 2 * (half // 3), half // 3, half // 3), in_turns=True)
        angle = torch.outer(torch.arange(5000, dtype=torch.float64), 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half))
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().to(DEV)
        self.pos = torch.zeros((3, T), dtype=torch.int32, device=DEV)
        self.w = [torch.rand(d, generator=self.g, device=DEV) + 0.5 for _ in range(2)]
        self.rows = torch.empty((T, hq + 2 * hkv, d), dtype=torch.bfloat16, device=DEV)
        self.q8 = torch.empty((T, hq, d), dtype=torch.uint8, device=DEV)
        self.out = torch.empty((T, hq, d), dtype=torch.float32, device=DEV)
        self.weights = torch.zeros((B, hkv, self.bound), device=DEV)
        self.kept = torch.empty((B, hkv, budget), dtype=torch.int32, device=DEV)
        self.kept_lens = torch.empty(B, dtype=torch.int32, device=DEV)
        self.freed = torch.empty(B * mpps, dtype=torch.int32, device=DEV)
        self.count = torch.empty(1, dtype=torch.int32, device=DEV)
        # one workspace for all calls of a stream
        self.ws = torch.empty(max(uq.extend_workspace_bytes(self.desc, T, B, hq, self.bound),
                                  uq.token_weights_workspace_bytes(self.desc, T, B, hq, self.bound),
                                  uq.select_workspace_bytes(B, hkv, self.bound, budget),
                                  uq.compact_workspace_bytes(self.desc, B, budget)), dtype=torch.uint8, device=DEV)

    def inputs(self, new, places):
        self.new.copy_(i32(new))
        self.rows.normal_(generator=self.g)
        self.pos.copy_(places)

    def attend(self):
        """Everything up to the weights."""
        uq, p = self.uq, self.plan
        uq.plan_tokens(self.cached, self.new, self.free, self.table, p)
        q, k, v = self.rows[:, :self.hq], self.rows[:, self.hq:self.hq + self.hkv], self.rows[:, self.hq + self.hkv:]
        spec = uq.NormRope(self.pos, self.cos_sin, self.w[0], self.w[1], pair_axes=self.axes)
        uq.norm_rope_write(self.desc, spec, q, k, v, p.slots, self.codes, self.scales, q_out=self.q8)
        uq.extend_attention(self.desc, self.q8, p.cu_seqlens, self.codes, self.scales, self.table, p.context_lens, self.bound,
                            workspace=self.ws, out=self.out)
        uq.token_weights(self.desc, self.q8, p.cu_seqlens, self.codes, self.scales, self.table, p.context_lens, self.bound,
                         self.weights, workspace=self.ws)

    def evict(self):
        uq, p = self.uq, self.plan
        uq.select_tokens(self.weights, p.context_lens, self.bound, self.budget, sinks=self.sinks, recent=self.recent,
                         kept=self.kept, kept_lens=self.kept_lens, workspace=self.ws)
        uq.compact_kv(self.desc, self.kept, self.kept_lens, p.context_lens, self.codes, self.scales, self.table,
                      weights=self.weights, freed_pages=self.freed, freed_count=self.count, workspace=self.ws)

    def state(self):
        return [self.codes, self.scales, self.table, self.weights, self.out, self.q8, self.kept, self.kept_lens, self.freed,
                self.count]


@pytest.mark.parametrize("d,hq,hkv", [(128, 8, 2), (64, 4, 4), (256, 6, 1)])
def test_steps_within_a_budget(uq, d, hq, hkv):
    B, T, mpps, budget, sinks, recent = 3, 200, 16, 100, 4, 20
    e = Engine(uq, B, T, hq, hkv, d, mpps, budget, sinks, recent, seed=d)
    total = [0] * B        # tokens of each sequence so far: positions go on when its cache does not grow
    for step, new in enumerate([[90, 7, 60], [1, 1, 1], [40, 0, 100], [1, 150, 1], [1, 1, 1]]):
        places = torch.randint(0, 3, (3, T), generator=e.g, device=DEV, dtype=torch.int32)
        at = 0
        for b, m in enumerate(new):
            places[:, at:at + m] += torch.arange(total[b], total[b] + m, dtype=torch.int32, device=DEV)
            at += m
            total[b] += m
        e.inputs(new, places)
        cached, before = e.cached.tolist(), e.weights.clone()
        e.attend()
        lens, cu = e.plan.context_lens.tolist(), e.plan.cu_seqlens.tolist()
        assert lens == [c + m for c, m in zip(cached, new)] and e.plan.result.tolist()[2] == 0
        taken = e.plan.result[1].item()
        kv = ref.pool_values(e.desc, e.codes, e.scales)
        want = ref.attend(e.desc, kv, e.q8, cu, e.table, lens, prepared=True)[:cu[-1]]
        assert float((e.out[:cu[-1]].double() - want).norm() / want.norm()) <= 1e-3
        # the queries are those of the rotation: FP8 rounds to half a step, 2^-4
        q = ref.walsh(rotated(e.rows[:cu[-1], :hq], e.w[0], e.pos[:, :cu[-1]], e.axes, e.cos_sin, False))
        q8 = e.q8[:cu[-1]].view(torch.float8_e4m3fn).double()
        assert ((q8 - q).abs() <= 2 ** -4 * q.abs() * (1 + 2 ** -10) + 2 ** -10 * (1 + 2 ** -10)).all()
        sums = expected(kv[0], e.q8.view(torch.float8_e4m3fn).double(), cu, e.table, lens, hkv, 0, True, d ** -0.5)
        eta = d ** -0.5 * 2 ** -12.5 * float(q8.abs().max()) * float(kv[0].abs().max())
        tol = 2 * eta + 2 ** -18 + 4 * 2 ** -23 + (max(lens) / 4 + max(new) * hq // hkv / 4 + 16) * 2 ** -24
        for b, n in enumerate(lens):
            assert torch.equal(e.weights[b, :, n:], before[b, :, n:])
            for h in range(hkv):
                w = before[b, h, :n].double() + sums[b][h]
                if n:
                    assert ((e.weights[b, h, :n].double() - w).abs() / w.clamp(min=2 ** -60)).max() <= tol
        c2, s2, w2 = e.codes.clone(), e.scales.clone(), e.weights.clone()
        e.evict()
        kl = e.kept_lens.tolist()
        for b, n in enumerate(lens):
            assert kl[b] == min(n, budget)
            for h in range(hkv):
                assert e.kept[b, h, :kl[b]].tolist() == chosen(w2[b, h].tolist(), n, budget, sinks, recent)
        freed = compact_plain(e.desc, e.kept, kl, lens, c2, s2, e.table, w2)
        assert torch.equal(e.codes, c2) and torch.equal(e.scales, s2) and torch.equal(e.weights, w2)
        assert e.count.item() == len(freed) and e.freed[:len(freed)].tolist() == freed
        # the engine's own bookkeeping
        e.free = torch.cat([e.free[taken:], e.freed[:e.count.item()]]).contiguous()
        e.cached = e.kept_lens.clone()
        assert len(set(e.free.tolist())) + sum(-(-n // 16) for n in kl) == B * mpps
        # single tokens read the compacted cache as any other
        q1 = torch.randn((B, hq, d), generator=e.g, device=DEV)
        kv = ref.pool_values(e.desc, e.codes, e.scales)
        got = uq.decode_attention(e.desc, q1, e.codes, e.scales, e.table, e.cached, e.bound)
        want = ref.attend(e.desc, kv, q1, list(range(B + 1)), e.table, kl)
        assert float((got.double() - want).norm() / want.norm()) <= 1e-3


def test_a_step_from_a_graph(uq):
    """Attention, weights, selection and compaction captured as one, with the workspace they
    share; replayed after other work, from the same state."""
    e = Engine(uq, 3, 200, 8, 2, 128, 16, 100, 4, 20, seed=5)
    g = torch.Generator(device=DEV).manual_seed(1)
    e.inputs([150, 40, 3], torch.randint(0, 4000, (3, 200), generator=g, device=DEV, dtype=torch.int32))
    start = [x.clone() for x in (e.codes, e.scales, e.table, e.weights)]

    def reset():
        for x, y in zip((e.codes, e.scales, e.table, e.weights), start):
            x.copy_(y)
        for x in (e.out, e.q8, e.kept, e.freed, e.count):
            x.zero_()

    reset()
    e.attend()
    e.evict()
    want = [x.clone() for x in e.state()]
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        e.attend()
        e.evict()
    for _ in range(3):
        reset()
        e.ws.fill_(0xFF)
        torch.cuda.synchronize()
        gr.replay()
        torch.cuda.synchronize()
        for x, y in zip(e.state(), want):
            assert torch.equal(x, y)


def test_two_streams_at_once(uq):
    """Two engines on two streams: each as alone."""
    alone, together = [], []
    for both in (False, True):
        engines = [Engine(uq, 3, 200, 8, 2, 128, 16, 100, 4, 20, seed=s) for s in (6, 7)]
        for s, e in enumerate(engines):
            g = torch.Generator(device=DEV).manual_seed(s)
            e.inputs([120 + s, 60, 9], torch.randint(0, 4000, (3, 200), generator=g, device=DEV, dtype=torch.int32))
            for x in (e.out, e.q8, e.freed):
                x.zero_()
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in engines] if both else [torch.cuda.current_stream()] * 2
        for e, s in zip(engines, streams):
            with torch.cuda.stream(s):
                e.attend()
                e.evict()
        torch.cuda.synchronize()
        (together if both else alone).extend(x for e in engines for x in e.state())
    assert all(torch.equal(x, y) for x, y in zip(alone, together))


def test_encoder_states_and_their_eviction(uq):
    """A decoder's queries over encoder states in the cache: cross attention, the weights it
    gives them without order, and cross attention over the states that stay."""
    lens, news, hq, hkv, d = [300, 47, 150], [9, 30, 1], 8, 2, 128
    table, pages = ref.tables(lens, DEV, 3, width=20)
    desc = uq.CacheDesc(num_kv_heads=hkv, num_pages=pages, head_dim=d)
    codes, scales = desc.alloc_pools(DEV, fill=0)
    g = torch.Generator(device=DEV).manual_seed(3)
    for b, n in enumerate(lens):
        k, v = (torch.randn((n, hkv, d), generator=g, device=DEV) for _ in range(2))
        slots = torch.arange(n, device=DEV) + b * 20 * 16
        uq.quantize_kv(desc, k, v, slots, codes, scales, page_table=table)
    cu, lens_t = i32([0, 9, 39, 40]), i32(lens)
    q = torch.randn((40, hq, d), generator=g, device=DEV)
    q8 = uq.prepare_query(desc, q)

    def plain(lens):
        kv, out = ref.pool_values(desc, codes, scales), torch.zeros((40, hq, d), dtype=torch.float64, device=DEV)
        weights = []
        for b, n in enumerate(lens):
            t = torch.arange(n, device=DEV)
            slot = table[b].long()[t // 16] * 16 + t % 16
            weights.append([])
            for h in range(hkv):
                rows = q8[cu[b]:cu[b + 1], 4 * h:4 * h + 4].view(torch.float8_e4m3fn).double().reshape(-1, d)
                p = torch.softmax(rows @ kv[0][slot, h].t().contiguous() / math.sqrt(d), -1)
                out[cu[b]:cu[b + 1], 4 * h:4 * h + 4] = (p @ kv[1][slot, h]).reshape(-1, 4, d)
                weights[b].append(p.sum(0))
        return ref.walsh(out), weights

    want, sums = plain(lens)
    out = uq.cross_attention(desc, q8, cu, codes, scales, table, lens_t, 320, out_dtype=torch.float32)
    assert float((out.double() - want).norm() / want.norm()) <= 1e-3
    w = uq.token_weights(desc, q8, cu, codes, scales, table, lens_t, 320, torch.zeros((3, hkv, 320), device=DEV), causal=False)
    for b, n in enumerate(lens):
        for h in range(hkv):
            assert ((w[b, h, :n].double() - sums[b][h]).abs() / sums[b][h]).max() <= 1e-3
    kept, kl = uq.select_tokens(w, lens_t, 320, 64)
    uq.compact_kv(desc, kept, kl, lens_t, codes, scales, table, weights=w)
    want, _ = plain(kl.tolist())
    out = uq.cross_attention(desc, q8, cu, codes, scales, table, kl, 64, out_dtype=torch.float32)
    assert float((out.double() - want).norm() / want.norm()) <= 1e-3
