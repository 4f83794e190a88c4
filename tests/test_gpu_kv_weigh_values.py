"""Accumulated weights where keys, queries or log-sums are not finite, against
their definition in 64 bits."""
import math

import pytest
import torch

from kv_more_util import weighed
from kv_util import attend, within
from paper_2504_11320_amd import kv
from test_gpu_kv_weigh import batch, fill

pytestmark = pytest.mark.gpu


def weigh(q, lse, c, pages, starts, lens, w, **kw):
    got = w.cuda()
    kv.weigh(q.cuda(), lse.cuda(), c, pages.cuda(), starts.cuda(), lens.cuda(), got, **kw)
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads", [1, 4, 7, 16, 32])
def test_an_infinite_key_that_nobody_attends_to(dtype, dim, heads):
    """Where every row's score of a key is -infinity, the key's weight is what it
    was: rows by themselves, a few together, many."""
    ql, kl = [1, 3, 1, 40], [70, 50, 16, 130]
    q, pages, starts, lens, n = batch(ql, kl, 16, heads, dim, dtype, 31)
    q[..., 3] = q[..., 3].abs() + 0.25
    c = fill(n, 16, 1, dim, dtype, 32)
    for b, j in ((0, 0), (0, 33), (0, 69), (1, 5), (1, 49), (2, 15), (3, 64), (3, 100), (3, 129)):
        c.k[int(pages[b, j // 16]), 0, j % 16, 3] = -math.inf
    out, lse = kv.attention(q.cuda(), c, pages.cuda(), starts.cuda(), lens.cuda(), return_lse=True)
    assert bool(torch.isfinite(out).all())
    # the last key of a request of one token is never all that it sees
    assert bool(torch.isfinite(lse).all())
    w = torch.rand(n, 1, 16, generator=torch.Generator().manual_seed(33))
    want, tol = weighed(q, lse, c, pages, starts, lens, w)
    assert bool(torch.isfinite(want).all())
    within(weigh(q, lse, c, pages, starts, lens, w), want, tol, "beside an infinity")


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("heads", [1, 4, 16, 32])
def test_an_infinite_scale_that_nobody_attends_to(dtype, heads):
    """The same of 8-bit keys: an infinite scale takes products below zero to
    -infinity."""
    ql, kl = [1, 3, 40], [70, 50, 130]
    q, pages, starts, lens, n = batch(ql, kl, 16, heads, 64, torch.float16, 34)
    q = q.abs() + 0.25
    c = fill(n, 16, 1, 64, dtype, 35)
    lse = attend(q, c, pages, starts, lens)[1].float()
    w = torch.rand(n, 1, 16, generator=torch.Generator().manual_seed(36))
    want, tol = weighed(q, lse, c, pages, starts, lens, w)
    for b, j in ((0, 33), (1, 5), (2, 64), (2, 100)):
        at = int(pages[b, j // 16]), 0, j % 16
        c.k[at] = torch.full((64,), -1.0).to(dtype).cuda()
        c.k_scale[at] = math.inf
        old = j < kl[b] - ql[b]
        want[at], tol[at] = float(w[at]) if old else 0.0, 0.0
    within(weigh(q, lse, c, pages, starts, lens, w), want, tol, "beside an infinite scale")


def idle_rows(ql, kl, heads, dim, dtype, cache_dtype, seed, **kw):
    """Rows under a log-sum of -infinity, among them all of a request's last
    token and of a whole request: whatever their queries hold, and the keys that
    only they see, they count nothing."""
    q, pages, starts, lens, n = batch(ql, kl, 16, heads, dim, dtype, seed)
    c = fill(n, 16, 1, dim, cache_dtype, seed + 1)
    lse = attend(q, c, pages, starts, lens, **kw)[1].float()
    g = torch.Generator().manual_seed(seed + 2)
    idle = torch.rand(lse.shape, generator=g) < 0.1
    for b in range(len(ql)):
        idle[int(starts[b + 1]) - 1] = True
    idle[int(starts[-2]):] = True
    lse[idle] = -math.inf
    w = torch.rand(n, 1, 16, generator=g)
    want, tol = weighed(q, lse, c, pages, starts, lens, w, **kw)
    # what must not count: queries that are not finite, and where causal each
    # request's last key, which its last token alone sees
    bad = torch.tensor([math.nan, math.inf, -math.inf])
    at = idle.nonzero()
    q[at[:, 0], at[:, 1], torch.arange(len(at)) % dim] = bad[torch.arange(len(at)) % 3].to(dtype)
    if kw.get("causal", True):
        for b, m in enumerate(kl):
            row = int(pages[b, (m - 1) // 16]), 0, (m - 1) % 16
            if c.k_scale is None:
                c.k[row] = float(bad[b % 3])
            else:
                c.k_scale[row] = float(bad[b % 3])
    got = weigh(q, lse, c, pages, starts, lens, w, **kw)
    within(got, want, tol, f"idle rows of {ql}")


@pytest.mark.parametrize("cache_dtype", [torch.bfloat16, torch.float16, torch.float8_e4m3fn,
                                         torch.int8])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads", [1, 7, 16])
def test_rows_that_saw_nothing_count_nothing(cache_dtype, dim, heads):
    dtype = cache_dtype if cache_dtype.itemsize == 2 else torch.float16
    idle_rows([1, 3, 1, 2], [70, 50, 16, 33], heads, dim, dtype, cache_dtype, 41)
    idle_rows([1, 150, 3, 40], [70, 200, 16, 133], heads, dim, dtype, cache_dtype, 51)
    idle_rows([150, 40], [200, 133], heads, dim, dtype, cache_dtype, 61, causal=False)
    idle_rows([150, 40], [200, 133], heads, dim, dtype, cache_dtype, 71, window=60)


def test_rows_that_saw_nothing_in_parts():
    """Rows split over workgroups, more blocks of rows than one turn of the ring."""
    idle_rows([900, 70], [900, 90], 4, 128, torch.bfloat16, torch.bfloat16, 81)
    idle_rows([500, 70], [900, 90], 16, 64, torch.float16, torch.int8, 91, causal=False)
