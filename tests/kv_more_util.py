"""Definitions in 64 bits, on the CPU, of the operators that bound a cache: norms
with the rotation, accumulated attention weights, eviction; and what the results
may be off by."""
import math

import torch

from kv_util import LEAST, ROUND, rows_of

ULP = 2.0 ** -24   # half a step of fp32, relative


def normed(x, w, eps):
    """(x over its root mean square times w, bound of the error in 32 bits).

    The sum of D squares is off by (D + 1) 2^-24 of itself, its mean, eps and the
    inverse root (two units, so four halves) by 6 more, of which the root takes
    half; two products round once each."""
    x = x.double()
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    if w is not None:
        y = y * w.double()
    return y, y.abs() * ((x.shape[-1] + 7) / 2 + 6) * ULP


def turned_normed(x, w, eps, pos, table, interleaved, norm=True):
    """(vectors normed where `norm` says so, then turned, bound in 32 bits)."""
    y, e = normed(x, w, eps) if norm else (x.double(), torch.zeros_like(x, dtype=torch.float64))
    if table is None:
        return y, e
    part = table.shape[1]
    half = part // 2
    row = table.double()[pos][:, None]
    cos, sin = row[..., :half], row[..., half:]
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    z, f = y.clone(), e.clone()
    z[..., a], z[..., b] = y[..., a] * cos - y[..., b] * sin, y[..., b] * cos + y[..., a] * sin
    for p, q in ((a, b), (b, a)):
        # what came in off, and two products and a sum, each rounded once
        f[..., p] = e[..., p] * cos.abs() + e[..., q] * sin.abs() \
            + 2 * ULP * ((y[..., p] * cos).abs() + (y[..., q] * sin).abs())
    return z, f


def rounded(y, e, dtype):
    """The bound of y, off by e, behind its rounding to a type."""
    return e * 1.01 + (y.abs() + e) * ROUND[dtype] + LEAST[dtype]


def weighed(q, lse, cache, pages, starts, lens, weights, scale=None, causal=True, window=0,
            accumulate=True):
    """(weights behind the call, bound of the error), on the CPU.

    A score is a sum of D exact products in fp32, off by (D + 8) 2^-24 of the sum
    of their magnitudes; factors, log-sum and their difference round a few times,
    2^-22 of score and log-sum together; 2^x is off by a unit; a sum of n terms by
    (n + 64) 2^-24 of itself."""
    q, pages, lse = q.cpu().double(), pages.cpu().long(), lse.cpu().double()
    starts, lens = starts.cpu().tolist(), lens.cpu().tolist()
    H, D = q.shape[1:]
    KH = cache.kv_heads
    G = H // KH
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out = weights.cpu().double()
    tol = torch.zeros_like(out)
    for b, m in enumerate(lens):
        a, n = starts[b], starts[b + 1] - starts[b]
        j = torch.arange(min(m, pages.shape[1] * cache.page_size))
        page = pages[b][j // cache.page_size]
        there = (page >= 0) & (page < cache.pages)
        j, page = j[there], page[there]
        off = j % cache.page_size
        k = rows_of(cache, "k", page * cache.page_size + off)       # [keys, KH, D]
        p = m - n + torch.arange(n)[:, None]
        see = torch.ones(n, j.numel(), dtype=torch.bool)
        if causal:
            see &= j <= p
        if window:
            see &= j > p.clamp(min=0) - window
        new = torch.zeros(j.numel(), KH, dtype=torch.float64)
        err = torch.zeros_like(new)
        for h in range(H):
            kh, qq, L = k[:, h // G], q[a:a + n, h], lse[a:a + n, h][:, None]
            z = qq @ kh.T * scale
            w = torch.where(see & (L > -math.inf), (z - L).exp(), torch.zeros_like(z))
            off_by = (D + 8) * ULP * (qq.abs() @ kh.abs().T) * scale \
                + 4 * ULP * (z.abs() + torch.where(torch.isfinite(L), L.abs(), 0.0)) + 2 * ULP
            new[:, h // G] += w.sum(0)
            err[:, h // G] += (w * torch.where(w > 0, off_by, 0.0)).sum(0)
        stays = (j < m - n) & accumulate
        old = torch.where(stays[:, None], out[page, :, off], 0.0)
        out[page, :, off] = old + new
        tol[page, :, off] = err * 1.01 + (n * G + 64) * ULP * new + 2 * ULP * (old + new).abs() + 2.0 ** -140
    return out, tol


def order(w):
    """Weights as numbers to be compared: NaN above infinity."""
    w = w.double()
    return torch.where(torch.isnan(w), torch.full_like(w, 1e300),
                       torch.nan_to_num(w, nan=0.0, posinf=1e299, neginf=-1e299))


def kept_keys(w, keep, recent):
    """Indices of the kept keys of one request and head, from their weights."""
    m = w.numel()
    if m <= keep:
        return list(range(m))
    x = order(w[:m - recent]).tolist()
    first = sorted(range(m - recent), key=lambda j: (-x[j], j))[:keep - recent]
    return sorted(first) + list(range(m - recent, m))


def evicted(cache, pages, lens, weights, keep, recent, to=None):
    """(kept, new lengths, the tensors behind the call by name), on the CPU, by
    copies of bits."""
    names = [n for n in ("k", "v", "k_scale", "v_scale") if getattr(cache, n) is not None]
    old = {n: getattr(cache, n).cpu() for n in names}
    for n in ("k", "v"):
        old[n] = old[n].view(torch.uint8 if old[n].element_size() == 1 else torch.int16)
    old["weights"] = weights.cpu()
    new = {n: x.clone() for n, x in old.items()}
    pages, P = pages.cpu().long(), cache.page_size
    to = pages if to is None else to.cpu().long()
    lens = lens.cpu().tolist()
    kept = torch.full((len(lens), cache.kv_heads, keep), -1, dtype=torch.int32)
    for b, m in enumerate(lens):
        j = torch.arange(m)
        for h in range(cache.kv_heads):
            w = old["weights"][pages[b][j // P], h, j % P]
            idx = torch.tensor(kept_keys(w, keep, recent), dtype=torch.int64)
            d = torch.arange(idx.numel())
            kept[b, h, :idx.numel()] = idx.int()
            for n in new:
                new[n][to[b][d // P], h, d % P] = old[n][pages[b][idx // P], h, idx % P]
    return kept, torch.tensor([min(m, keep) for m in lens], dtype=torch.int32), new
