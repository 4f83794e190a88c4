"""The KV-path operators' definitions in 64 bits, on the CPU, and what their
results may be off by."""
import math

import torch

TOP = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
# largest relative error of rounding to a type, and half its smallest step
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}


def turned(x, pos, table, interleaved=False, inverse=False):
    """(x turned, a bound of the error of computing it in 32 bits), from the
    fp32 table, x in 64 bits."""
    part = table.shape[1]
    half = part // 2
    cos = table[pos].double()[:, None, :half]
    sin = table[pos].double()[:, None, half:] * (-1.0 if inverse else 1.0)
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    y, e = x.clone(), torch.zeros_like(x)
    u, v = x[..., a], x[..., b]
    y[..., a], y[..., b] = u * cos - v * sin, v * cos + u * sin
    # two products and a sum, each rounded once
    e[..., a] = 2.0 ** -23 * ((u * cos).abs() + (v * sin).abs())
    e[..., b] = 2.0 ** -23 * ((v * cos).abs() + (u * sin).abs())
    return y, e


def codes(x, kind):
    """(codes as fp32, scales) of fp32 rows by the operator's own arithmetic:
    fp32 throughout, 1 / t rounded, times the largest code rounded, times x
    rounded, to the nearest code with ties to even."""
    t = x.abs().amax(-1)
    ok = t >= 2.0 ** -100
    one = torch.ones_like(t)
    by = torch.where(ok, (one / torch.where(ok, t, one)) * TOP[kind], torch.zeros_like(t))
    y = (x * by[..., None]).clamp(-TOP[kind], TOP[kind])
    scale = torch.where(ok, t / torch.full_like(t, TOP[kind]), torch.zeros_like(t))
    return (y.round() if kind == torch.int8 else y.to(kind).float()), scale


def rows_of(cache, name, slots):
    """Rows of slots (all of them valid), in 64 bits."""
    x = getattr(cache, name).cpu()
    at, off = slots // cache.page_size, slots % cache.page_size
    y = x.float()[at, :, off].double() if x.dtype != torch.float8_e4m3fn else \
        x.view(torch.uint8)[at, :, off].view(x.dtype).float().double()
    s = getattr(cache, name + "_scale")
    return y if s is None else y * s.cpu()[at, :, off].double()[..., None]


def attend(q, cache, pages, starts, lens, scale=None, causal=True, window=0):
    """(out, lse, bound of out, bound of lse) in 64 bits.  The bounds:

    scores are sums of D exact products in fp32 with a few roundings after (and,
    of a bf16 query against codes, of a query rounded 2^-25 below its largest
    element): off by z; a weight is off by 2 z and its own rounding to 16 bits
    (the cache's type, fp16 for codes; these lose what lies below their
    smallest step); sums of n terms are off by n 2^-24; the result is rounded
    once.
    """
    q, pages = q.cpu(), pages.cpu().long()
    starts, lens = starts.cpu().tolist(), lens.cpu().tolist()
    T, H, D = q.shape
    G = H // cache.kv_heads
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    wt = torch.float16 if cache.k_scale is not None else cache.dtype
    out = torch.zeros(T, H, D, dtype=torch.float64)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for b, m in enumerate(lens):
        a, n = starts[b], starts[b + 1] - starts[b]
        j = torch.arange(min(m, pages.shape[1] * cache.page_size))
        page = pages[b][j // cache.page_size]
        there = (page >= 0) & (page < cache.pages)
        slots = torch.where(there, page, torch.zeros_like(page)) * cache.page_size \
            + j % cache.page_size
        k, v = rows_of(cache, "k", slots), rows_of(cache, "v", slots)
        for i in range(n):
            p = m - n + i
            see = there.clone()
            if causal:
                see &= j <= p
            if window:
                see &= j > p - window
            if not bool(see.any()):
                continue
            kk, vv = k[see], v[see]
            for h in range(H):
                qq = q[a + i, h].double()
                kh, vh = kk[:, h // G], vv[:, h // G]
                z = kh @ qq * scale
                L = torch.logsumexp(z, 0)
                w = (z - L).exp()
                o = w @ vh
                out[a + i, h], lse[a + i, h] = o, L
                zerr = ((D + 8) * 2.0 ** -24 * (kh.abs() @ qq.abs())
                        + 2.0 ** -25 * qq.abs().max() * kh.abs().sum(-1)) * scale
                zerr = float(zerr.max()) + 2.0 ** -22 * float(z.abs().max())
                size = w @ vh.abs()
                lost = LEAST[wt] * 4 * kh.shape[0] * float((w[:, None] * vh.abs()).max())
                if cache.k_scale is not None:
                    lost *= 512
                tol[a + i, h] = (size * (ROUND[wt] + 2 * zerr + (kh.shape[0] + 64) * 2.0 ** -24)
                                 + lost) * 1.01 + o.abs() * ROUND[q.dtype] + LEAST[q.dtype]
                ltol[a + i, h] = zerr + (kh.shape[0] + 64) * 2.0 ** -24 \
                    + 2.0 ** -22 * (1 + abs(float(L)))
    return out, lse, tol, ltol


def within(got, want, tol, what):
    got = got.detach().cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), f"{what}: not finite elsewhere"
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{what}: other infinities"
    off = (got - want).abs()[fine] - tol[fine]
    assert off.numel() == 0 or float(off.max()) <= 0.0, \
        f"{what}: over its bound by {float(off.max()):.3g}, of {float(tol[fine].max()):.3g}"
