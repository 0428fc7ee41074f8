"""Token plans (uq_plan_tokens) against the rule on Python lists: every output
equal, page-table entries that are not new left as they were."""
import random

import pytest
import torch

import serving_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def uq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_20474_amd import uq as mod
    return mod


def run(uq, cached, new, free, width, cap, seed=0):
    dev = torch.device("cuda:0")
    print(f"batch {len(cached)} cached {cached[:8]} new {new[:8]} free {len(free)} width {width} rows {cap}", flush=True)
    rng = random.Random(seed)
    table = [[rng.randrange(1 << 20) for _ in range(width)] for _ in cached]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    t = i32(table).reshape(len(cached), width)
    plan = uq.TokenPlan.alloc(len(cached), cap, dev)
    for x in (plan.context_lens, plan.cu_seqlens, plan.seq_ids, plan.positions, plan.slots, plan.result):
        x.fill_(-77)
    uq.plan_tokens(i32(cached), i32(new), i32(free), t, plan)
    torch.cuda.synchronize()
    want = ref.plan(cached, new, free, table, cap)
    assert plan.result.tolist() == want["result"]
    assert plan.context_lens.tolist() == want["context"]
    assert plan.cu_seqlens.tolist() == want["cu"]
    assert plan.seq_ids.tolist() == want["seq"]
    pos = plan.positions.tolist()
    assert all(p == w for p, w, s in zip(pos, want["pos"], want["slots"]) if s >= 0 or w < 1 << 31)
    assert plan.slots.tolist() == want["slots"]
    assert t.tolist() == table
    return want


FREE = [7, 3, 900, 12, 44, 5, 6, 8, 1, 0]


@pytest.mark.parametrize("cached,new,width,cap", [
    ([0], [1], 4, 1), ([15], [1], 4, 1), ([16], [1], 4, 3), ([0], [0], 1, 0), ([0], [0], 1, 5),
    ([0, 5, 16, 31, 32], [16, 1, 17, 1, 0], 4, 40),
    ([-3, 4], [2, -9], 4, 8),                       # negative lengths count as 0
    ([0, 0, 0], [17, 33, 1], 3, 64),
    ([0, 60, 3], [5, 5, 5], 4, 20),                 # the second does not fit its row
    ([0, 0, 0], [10, 10, 10], 4, 25),               # the third's rows do not fit
    ([0, 0, 0, 9, 0], [40, 1000, 5, 2, 0], 4, 30),  # nor the first's and those behind
    ([0, 2147483647, 0], [4, 2147483647, 4], 4, 50),
])
def test_small(uq, cached, new, width, cap):
    run(uq, cached, new, FREE, width, cap)


@pytest.mark.parametrize("free", [0, 1, 2, 3, 4])
def test_free_list_runs_out(uq, free):
    want = run(uq, [0, 16, 5, 30, 0], [17, 16, 3, 10, 1], FREE[:free], 4, 64)
    assert want["context"][2] == 8    # needs no page: admitted whatever the list holds
    assert want["result"][2] >= 1


@pytest.mark.parametrize("batch", [1, 2, 63, 64, 65, 255, 256, 257, 1000, 4096])
def test_random(uq, batch):
    rng = random.Random(batch)
    cached = [rng.choice([0, rng.randrange(200), rng.randrange(16) * 16]) for _ in range(batch)]
    new = [rng.choice([0, 1, 1, rng.randrange(40)]) for _ in range(batch)]
    need = sum(-(-(h + n) // 16) - -(-h // 16) for h, n in zip(cached, new))
    free = rng.sample(range(1 << 20), need + 2)
    run(uq, cached, new, free, 16, sum(new) + 7, batch)
    run(uq, cached, new, free[:need // 2], 12, sum(new) * 3 // 4, batch)


def test_one_long_prompt(uq):
    run(uq, [0, 3], [65536, 1], list(range(5000, 9200)), 4200, 65600)


def test_no_sequences(uq):
    dev = torch.device("cuda:0")
    empty = torch.empty(0, dtype=torch.int32, device=dev)
    plan = uq.TokenPlan.alloc(0, 5, dev)
    uq.plan_tokens(empty, empty, empty, torch.empty((0, 4), dtype=torch.int32, device=dev), plan)
    assert plan.cu_seqlens.tolist() == [0] and plan.result.tolist() == [0, 0, 0]
    assert plan.slots.tolist() == [-1] * 5


def test_steps_in_a_graph(uq):
    """Captured once, replayed with other lengths and pages."""
    dev = torch.device("cuda:0")
    rng = random.Random(5)
    B, width, cap = 9, 8, 64
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    cached, new = i32([0] * B), i32([1] * B)
    free, table = i32(list(range(100, 150))), torch.zeros((B, width), dtype=torch.int32, device=dev)
    plan = uq.TokenPlan.alloc(B, cap, dev)
    uq.plan_tokens(cached, new, free, table, plan)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        uq.plan_tokens(cached, new, free, table, plan)
    for _ in range(4):
        c, n, f = ([rng.randrange(60) for _ in range(B)], [rng.randrange(9) for _ in range(B)],
                   rng.sample(range(1 << 16), 50))
        cached.copy_(i32(c))
        new.copy_(i32(n))
        free.copy_(i32(f))
        t0 = [[rng.randrange(99) for _ in range(width)] for _ in range(B)]
        table.copy_(i32(t0))
        graph.replay()
        torch.cuda.synchronize()
        want = ref.plan(c, n, f, t0, cap)
        assert plan.slots.tolist() == want["slots"] and table.tolist() == t0
        assert plan.result.tolist() == want["result"]
