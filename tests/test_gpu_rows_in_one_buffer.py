"""norm_rope and norm_rope_write with inputs and outputs in one buffer, next to each
other, between the rows of a strided input, and in place: the same rows as from
memory of their own.  Overlapping ones are refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
T, HQ, HKV, D = 21, 4, 2, 128


@pytest.fixture(scope="module")
def uq():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2606_20474_amd import uq as mod
    return mod


def rows(seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    q, k, v = (torch.randn((T, h, D), generator=g, device=DEV).bfloat16() for h in (HQ, HKV, HKV))
    w = torch.rand(D, generator=g, device=DEV) + 0.5
    return q, k, v, w


def test_side_by_side_and_in_place(uq):
    q, k, v, w = rows()
    spec = uq.NormRope(q_weight=w, k_weight=w)
    want = uq.norm_rope(spec, q, k)
    nq, nk = q.numel(), k.numel()
    buf = torch.zeros(2 * (nq + nk), dtype=torch.bfloat16, device=DEV)
    bq, bqo, bk, bko = (x.view(T, -1, D) for x in buf.split([nq, nq, nk, nk]))
    bq.copy_(q)
    bk.copy_(k)
    uq.norm_rope(spec, bq, bk, q_out=bqo, k_out=bko)
    assert torch.equal(bqo, want[0]) and torch.equal(bko, want[1])
    assert torch.equal(bq, q) and torch.equal(bk, k)
    with pytest.raises(uq.UQError):
        uq.norm_rope(spec, bq, bk, q_out=buf[D:D + nq].view(T, HQ, D), k_out=bko)
    with pytest.raises(uq.UQError):
        uq.norm_rope(spec, bq, bk, q_out=buf.view(torch.float32)[:nq].view(T, HQ, D), k_out=bko.float())
    assert torch.equal(bq, q) and torch.equal(bk, k)
    uq.norm_rope(spec, bq, bk, q_out=bq, k_out=bk)
    assert torch.equal(bq, want[0]) and torch.equal(bk, want[1])


def test_outputs_between_the_rows(uq):
    """Token rows far enough apart that the outputs fit between two of them."""
    q, k, v, w = rows()
    spec = uq.NormRope(q_weight=w, k_weight=w)
    want = uq.norm_rope(spec, q[:2], k[:2])
    buf = torch.zeros((2, 64, D), dtype=torch.bfloat16, device=DEV)
    buf[:, :HQ], buf[:, HQ:HQ + HKV] = q[:2], k[:2]
    at = HQ + HKV
    qo, ko = buf[0, at:at + 2 * HQ].view(2, HQ, D), buf[0, at + 2 * HQ:at + 2 * (HQ + HKV)].view(2, HKV, D)
    uq.norm_rope(spec, buf[:, :HQ], buf[:, HQ:at], q_out=qo, k_out=ko)
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    one = uq.norm_rope(spec, buf[:1, :HQ], q_out=buf[:1, :HQ])[0]     # one token: any stride
    assert torch.equal(one, want[0][:1])


def test_write_side_by_side_and_in_place(uq):
    q, k, v, w = rows()
    spec = uq.NormRope(q_weight=w, k_weight=w)
    desc = uq.CacheDesc(num_kv_heads=HKV, num_pages=3)
    slots = torch.arange(T, device=DEV)
    a, b = desc.alloc_pools(DEV, fill=9), desc.alloc_pools(DEV, fill=9)
    for dt in (torch.uint8, torch.bfloat16):
        want = uq.norm_rope_write(desc, spec, q, k, v, slots, *a, q_out_dtype=dt)
        fused = torch.cat([q, k, v], 1)
        n = fused.numel() * 2
        buf = torch.zeros(2 * n, dtype=torch.uint8, device=DEV)
        rows_ = buf[:n].view(torch.bfloat16).view(T, HQ + 2 * HKV, D)
        rows_.copy_(fused)
        out = buf[n:n + want.numel() * want.element_size()].view(dt).view(T, HQ, D)
        uq.norm_rope_write(desc, spec, rows_[:, :HQ], rows_[:, HQ:HQ + HKV], rows_[:, HQ + HKV:], slots, *b, q_out=out)
        assert torch.equal(out, want) and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    with pytest.raises(uq.UQError):
        uq.norm_rope_write(desc, spec, q, k, v, slots, *b, q_out=q.view(-1).view(torch.uint8)[:q.numel()].view(T, HQ, D))
    want = uq.norm_rope(spec, q)[0]
    assert torch.equal(uq.norm_rope_write(desc, spec, q, k, v, slots, *b, q_out=q), want) and torch.equal(q, want)
