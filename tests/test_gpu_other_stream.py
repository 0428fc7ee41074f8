"""Calls on another stream than the current one, with the tensors that they make
themselves: zeroes come before the kernels, and the memory belongs to that
stream, whatever the current one still has to do."""
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


@pytest.fixture(scope="module")
def calls(uq):
    """name -> call(stream) of every call that makes tensors, on inputs that are ready."""
    lens, news = [3000, 40, 7], [5, 17, 2]
    table, pages = ref.tables(lens, DEV, 3)
    desc = uq.CacheDesc(num_kv_heads=2, num_pages=pages)
    codes, scales = ref.fill_pools(desc, DEV, 3)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    ctx, cu = i32(lens), i32([0, 5, 22, 24])
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k, v = (torch.randn((24, h, 128), generator=g, device=DEV) for h in (8, 2, 2))
    slots = torch.arange(24, device=DEV) * 3
    spec = uq.NormRope(q_weight=torch.ones(128, device=DEV))
    pools = [x.clone() for x in (codes, scales)]
    cs = torch.tensor([0.15, 0.16], device=DEV)
    q3 = q[:3].contiguous()
    out = {
        "extend": lambda s: uq.extend_attention(desc, q, cu, codes, scales, table, ctx, 3000, stream=s),
        "read": lambda s: uq.read_kv(desc, slots, codes, scales, stream=s),
        "rows": lambda s: uq.norm_rope(spec, q, k, stream=s),
        "write": lambda s: uq.norm_rope_write(desc, spec, q, k, v, slots, *pools, stream=s),
        "window": lambda s: uq.decode_window(desc, q3, codes, scales, table, ctx, 3000, 100, 2, stream=s),
        "decode": lambda s: uq.decode_attention(desc, q3, codes, scales, table, ctx, 3000, stream=s),
        "query": lambda s: uq.prepare_query(desc, q, stream=s),
        "error": lambda s: uq.quantize_error(k, cs, stream=s),
    }
    torch.cuda.synchronize()
    return out


NAMES = ["extend", "read", "rows", "write", "window", "decode", "query", "error"]


def parts(x):
    return [t.clone() for t in (x if isinstance(x, tuple) else (x,))]


@pytest.mark.parametrize("name", NAMES)
def test_while_the_current_stream_is_busy(calls, name):
    call = calls[name]
    want = parts(call(None))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda._sleep(20_000_000)     # the current stream's own work, some milliseconds
        got = call(side)
        side.synchronize()
        torch.cuda.synchronize()
        for a, b in zip(parts(got), want):
            assert torch.equal(a, b)
        got = None


@pytest.mark.parametrize("name", NAMES)
def test_the_tensors_are_made_on_the_call_s_stream(calls, name, monkeypatch):
    side = torch.cuda.Stream()
    seen = []

    def wrap(make):
        def made(*args, **kw):
            seen.append(torch.cuda.current_stream().cuda_stream)
            return make(*args, **kw)
        return made
    before = torch.cuda.current_stream().cuda_stream
    with monkeypatch.context() as m:
        m.setattr(torch, "empty", wrap(torch.empty))
        m.setattr(torch, "zeros", wrap(torch.zeros))
        calls[name](side)
    torch.cuda.synchronize()
    assert seen and all(s == side.cuda_stream for s in seen)
    assert torch.cuda.current_stream().cuda_stream == before
