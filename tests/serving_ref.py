"""Plain 64-bit forms of the calls around the cache (token plans, norm and
rotation, reading back, windowed and multi-query attention), written from
their formulas in torch; shared by their tests."""
import math

import torch

PAGE = 16


def walsh(x):
    """H_d x / sqrt(d) over the last dimension."""
    d, shape = x.shape[-1], x.shape
    x = x.double()
    h = 1
    while h < d:
        y = x.reshape(-1, d // (2 * h), 2, h)
        x = torch.stack([y[:, :, 0] + y[:, :, 1], y[:, :, 0] - y[:, :, 1]], 2)
        h *= 2
    return x.reshape(shape) / math.sqrt(d)


def e4m3(x):
    return x.clamp(-448, 448).float().to(torch.float8_e4m3fn).double()


def pool_values(desc, codes, scales):
    """K and V [num_pages * 16, Hkv, d] as stored (rotated), in 64 bits."""
    P, H, d = desc.num_pages, desc.num_kv_heads, desc.head_dim
    c = codes[:desc.codes_bytes()].view(P, H, 2, 8 * d).long()
    nib = torch.stack([c & 15, c >> 4], -1).flatten(-2)
    level = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64,
                         device=codes.device)
    val = level[nib]
    sc = torch.exp2(scales[:desc.scales_bytes()].view(P, H, 2, d // 32, PAGE).double() - 127)
    k = val[:, :, 0].reshape(P, H, d // 32, PAGE, 32) * sc[:, :, 0, :, :, None]
    v = val[:, :, 1].reshape(P, H, 4, d // 8, 4, 8).permute(0, 1, 2, 4, 3, 5).reshape(P, H, PAGE, d // 32, 32)
    v = v * sc[:, :, 1].transpose(-1, -2)[..., None]
    return (k.permute(0, 3, 1, 2, 4).reshape(P * PAGE, H, d), v.permute(0, 2, 1, 3, 4).reshape(P * PAGE, H, d))


def visible(n, p, window, sinks):
    """Tokens of a context of n that a query at position p sees."""
    return [t for t in range(min(n, p + 1)) if not window or t > p - window or t < sinks]


def attend(desc, kv, q, cu, page_table, lens, window=0, sinks=0, scale=None, prepared=False):
    """Rows q [T, Hq, d] (64-bit out, NaN where no sequence has the row)."""
    k_all, v_all = kv
    d, hkv = desc.head_dim, desc.num_kv_heads
    scale = d ** -0.5 if scale is None else scale
    q8 = q.view(torch.float8_e4m3fn).double() if prepared else e4m3(walsh(q.double()))
    out = torch.full(q.shape, math.nan, dtype=torch.float64, device=q.device)
    g = q.shape[1] // hkv
    for b, n in enumerate(lens):
        m = cu[b + 1] - cu[b]
        if m <= 0:
            continue
        t = torch.arange(max(n, 0), device=q.device)
        p = torch.arange(n - m, n, device=q.device)[:, None]
        seen = t <= p
        if window:
            seen &= (t > p - window) | (t < sinks)
        slot = page_table[b].long()[t // PAGE] * PAGE + t % PAGE
        k, v = k_all[slot], v_all[slot]
        anyone = seen.any(0)     # tokens no query sees may hold anything
        k = torch.where(anyone[:, None, None], k, 0.0)
        v = torch.where(anyone[:, None, None], v, 0.0)
        for h in range(hkv):
            qh = q8[cu[b]:cu[b + 1], h * g:(h + 1) * g].transpose(0, 1)      # [G, m, d]
            s = (qh @ k[:, h].t().contiguous()) * scale
            s = s.masked_fill(~seen, -math.inf)
            e = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-1e300)) if n > 0 else s
            o = (e @ v[:, h]) / e.sum(-1, keepdim=True).clamp(min=1e-300)
            out[cu[b]:cu[b + 1], h * g:(h + 1) * g] = o.transpose(0, 1)
    return walsh(out) if desc.rotate_v else out


def fill_pools(desc, device, seed, v_scale=1.0):
    """Pools of Gaussian-like codes, every token written, scale bytes around 1/4."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    codes = torch.randint(0, 256, (desc.codes_bytes(),), generator=g, dtype=torch.int32).to(torch.uint8)
    scales = torch.randint(123, 127, (desc.scales_bytes(),), generator=g, dtype=torch.int32)
    sc = scales.view(desc.num_pages, desc.num_kv_heads, 2, -1)
    sc[:, :, 1] += round(math.log2(v_scale))
    return codes.to(device), scales.to(torch.uint8).to(device)


def tables(lens, device, seed, width=None, spare=3):
    """(page table int32 [B, width], pages in the pool): a random permutation."""
    g = torch.Generator().manual_seed(seed)
    pages = [-(-max(n, 0) // PAGE) for n in lens]
    total = sum(pages) + spare
    perm = torch.randperm(total, generator=g).int()
    t = torch.full((len(lens), width or max(1, *pages)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        t[b, :n] = perm[at:at + n]
        at += n
    return t.to(device), total


def norm_rope(x, w, eps, pos, cos_sin, interleaved):
    """[T, H, d] in 64 bits."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w.double()
    if cos_sin is None:
        return x
    r = cos_sin.shape[1]
    cs = cos_sin.double()[pos.long().clamp(0, cos_sin.shape[0] - 1)][:, None]
    c, s = cs[..., :r // 2], cs[..., r // 2:]
    x = x.clone()
    a, b = (x[..., 0:r:2].clone(), x[..., 1:r:2].clone()) if interleaved else (x[..., :r // 2].clone(),
                                                                              x[..., r // 2:r].clone())
    ya, yb = a * c - b * s, b * c + a * s
    if interleaved:
        x[..., 0:r:2], x[..., 1:r:2] = ya, yb
    else:
        x[..., :r // 2], x[..., r // 2:r] = ya, yb
    return x


def plan(cached, new, free, table, cap):
    """uq_plan_tokens on Python lists; returns a dict of lists, `table` changed in place."""
    B, width = len(cached), len(table[0]) if table else 0
    out = dict(context=[], cu=[0], seq=[-1] * cap, pos=[0] * cap, slots=[-1] * cap)
    row, used, taken, refused = 0, 0, 0, 0
    for b in range(B):
        h, n = max(cached[b], 0), max(new[b], 0)
        total, held = -(-(h + n) // PAGE), -(-h // PAGE)
        fits = total <= width and row + n <= cap
        need = total - held if fits else 0
        ok = fits and (need == 0 or used + need <= len(free))
        if ok:
            for i in range(need):
                table[b][held + i] = free[used + i]
            taken += need
        used += need
        refused += not ok
        out["context"].append(h + n if ok else 0)
        for i in range(n):
            if row + i < cap:
                p = h + i
                out["seq"][row + i], out["pos"][row + i] = b, p
                if ok:
                    out["slots"][row + i] = table[b][p // PAGE] * PAGE + p % PAGE
        row = min(row + n, cap + 1)
        out["cu"].append(min(row, cap))
    out["result"] = [min(row, cap), taken, refused]
    return out
