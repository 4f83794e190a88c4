"""Attention over an 8-bit cache that `append` filled, in 64 bits, with bounds
that a wrong result over thousands of keys does not pass."""
import math

import torch

from kv_util import LEAST, ROUND, rows_of


def attend_codes(q, cache, pages, starts, lens, causal=True, window=0):
    """(out, bound of out), every page there.

    The reference of a weight is at most the largest z_j + log2 t_j, t_j the scale
    of row j, so that 2^(z_j - reference) t_j is at most 1 and rounding it to fp16
    loses 2^-11 of itself, or 2^-25 where it is subnormal.  A stored row has a code
    of the largest magnitude M, so some key reaches M in these units with weight
    times value, and the 2^-25 M lost at most for each of n keys are n 2^-25 of the
    largest weight times value.  Scores are off by zerr, which counts twice (in the
    weight and in the denominator); a sum of n terms by (n + 64) 2^-24 of the sum of
    their magnitudes; the result is rounded once.
    """
    q, pages = q.cpu(), pages.cpu().long()
    starts, lens = starts.cpu().tolist(), lens.cpu().tolist()
    T, H, D = q.shape
    G = H // cache.kv_heads
    scale = 1.0 / math.sqrt(D)
    out = torch.zeros(T, H, D, dtype=torch.float64)
    tol = torch.zeros_like(out)
    for b, m in enumerate(lens):
        a, n = starts[b], starts[b + 1] - starts[b]
        j = torch.arange(m)
        slots = pages[b][j // cache.page_size] * cache.page_size + j % cache.page_size
        k, v = rows_of(cache, "k", slots), rows_of(cache, "v", slots)
        p = m - n + torch.arange(n)[:, None]
        see = torch.ones(n, m, dtype=torch.bool)
        if causal:
            see &= j <= p
        if window:
            see &= j > p - window
        count = see.sum(-1, keepdim=True)
        for h in range(H):
            kh, vh, qq = k[:, h // G], v[:, h // G], q[a:a + n, h].double()
            z = (qq @ kh.T * scale).masked_fill(~see, -math.inf)
            w = (z - torch.logsumexp(z, -1, keepdim=True)).exp()
            o = w @ vh
            zerr = (D + 8) * 2.0 ** -24 * (qq.abs() @ kh.abs().T) \
                + 2.0 ** -25 * qq.abs().amax(-1, keepdim=True) * kh.abs().sum(-1)
            zerr = (zerr * scale * see).amax(-1, keepdim=True) \
                + 2.0 ** -22 * z.masked_fill(~see, 0.0).abs().amax(-1, keepdim=True)
            lost = count * 2.0 ** -25 * (w * vh.abs().amax(-1)).amax(-1, keepdim=True)
            e = (w @ vh.abs()) * (2.0 ** -11 + 2 * zerr + (count + 64) * 2.0 ** -24) + lost
            out[a:a + n, h] = o
            tol[a:a + n, h] = e * 1.01 + o.abs() * ROUND[q.dtype] + LEAST[q.dtype]
    return out, tol


def says_something(out, tol):
    """Whether a result of zeros, or one negated, would be refused: four fifths
    of the elements are larger than their bounds."""
    return float((out.abs() > tol).double().mean()) >= 0.8
