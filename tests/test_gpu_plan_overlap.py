"""plan_tokens through views of one buffer, next to each other and overlapping."""
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


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_the_lengths_of_a_step_are_not_the_lengths_before_it(uq):
    plan = uq.TokenPlan.alloc(2, 8, DEV)
    plan.context_lens.fill_(0)
    table = torch.zeros((2, 4), dtype=torch.int32, device=DEV)
    new, free = i32([3, 2]), i32([5, 6, 7, 8])
    with pytest.raises(uq.UQError):
        uq.plan_tokens(plan.context_lens, new, free, table, plan)
    with pytest.raises(uq.UQError):
        uq.plan_tokens(i32([0, 0]), new, table.view(-1)[:4], table, plan)
    assert plan.context_lens.tolist() == [0, 0] and not table.any()


def test_neighbours_and_two_plans_in_turn(uq):
    """Arrays side by side in one buffer, the lengths handed from one plan to the other."""
    B, T, width = 3, 20, 4
    free = list(range(40, 52))
    buf = torch.full((2, 4 * B + 1 + 2 * T + 3), -77, dtype=torch.int32, device=DEV)
    slots = torch.empty((2, T), dtype=torch.int64, device=DEV)
    plans, news = [], []
    for r in range(2):
        parts = buf[r].split([B, B, B + 1, B, T, T, 3])
        news.append(parts[1])
        plans.append(uq.TokenPlan(parts[0], parts[2], parts[4], parts[5], slots[r], parts[6]))
    table = torch.zeros((B, width), dtype=torch.int32, device=DEV)
    host = [[0] * width for _ in range(B)]
    plans[1].context_lens.zero_()
    cached = [0] * B
    for i, new in enumerate([[5, 0, 13], [1, 16, 2], [0, 1, 1], [11, 3, 3]]):
        print(f"step {i}: cached {cached} new {new}", flush=True)
        news[i % 2].copy_(i32(new))
        plan = uq.plan_tokens(plans[(i + 1) % 2].context_lens, news[i % 2], i32(free), table, plans[i % 2])
        torch.cuda.synchronize()
        want = ref.plan(cached, new, free, host, T)
        assert plan.context_lens.tolist() == want["context"] and plan.slots.tolist() == want["slots"]
        assert plan.result.tolist() == want["result"] and table.tolist() == host
        cached, free = want["context"], free[want["result"][1]:]
