"""Accumulated attention weights of cached keys against their definition in 64
bits."""
import math

import pytest
import torch

from kv_more_util import weighed
from kv_util import attend, within
from paper_2504_11320_amd import kv

pytestmark = pytest.mark.gpu

CACHES = (torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8)


def fill(pages, page, kv_heads, dim, dtype, seed):
    """A cache on the card with rows in every slot."""
    g = torch.Generator().manual_seed(seed)
    c = kv.Cache.empty(pages, page, kv_heads, dim, dtype)
    k = torch.randn(pages * page, kv_heads, dim, generator=g)
    v = torch.randn(pages * page, kv_heads, dim, generator=g)
    t = dtype if dtype in (torch.bfloat16, torch.float16) else torch.bfloat16
    kv.append(c, k.to(t).cuda(), v.to(t).cuda(), torch.arange(pages * page).cuda())
    return c


def batch(ql, kl, page, heads, dim, dtype, seed, spare=2, by=1.5):
    """(q, pages, starts, lens, number of pages): pages in no order."""
    g = torch.Generator().manual_seed(seed)
    need = [max(0, -(-m // page)) for m in kl]
    n = sum(need) + spare
    at = torch.randperm(n, generator=g).int()
    table = torch.full((len(kl), max(need + [1])), -1, dtype=torch.int32)
    a = 0
    for b, c in enumerate(need):
        table[b, :c] = at[a:a + c]
        a += c
    starts = torch.tensor([0] + torch.tensor(ql).cumsum(0).tolist(), dtype=torch.int32)
    q = (by * torch.randn(sum(ql), heads, dim, generator=g)).to(dtype)
    return q, table, starts, torch.tensor(kl, dtype=torch.int32), n


def run(ql, kl, page, heads, kv_heads, dim, cache_dtype, dtype=None, seed=1, accumulate=True,
        causal=True, window=0, scale=None, change=None, **bounds):
    """One call on log-sums of the definition, every weight checked."""
    dtype = dtype or (cache_dtype if cache_dtype in (torch.bfloat16, torch.float16)
                      else torch.bfloat16)
    q, pages, starts, lens, n = batch(ql, kl, page, heads, dim, dtype, seed)
    if change:
        change(pages)
    c = fill(n, page, kv_heads, dim, cache_dtype, seed + 1)
    kw = dict(scale=scale, causal=causal, window=window)
    lse = attend(q, c, pages, starts, lens, **kw)[1].float()
    w = torch.rand(n, kv_heads, page, generator=torch.Generator().manual_seed(seed + 2))
    want, tol = weighed(q, lse, c, pages, starts, lens, w, accumulate=accumulate, **kw)
    got = w.cuda()
    kv.weigh(q.cuda(), lse.cuda(), c, pages.cuda(), starts.cuda(), lens.cuda(), got,
             accumulate=accumulate, **kw, **bounds)
    within(got, want, tol, f"weights of {ql} over {kl}")
    return got


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (8, 2), (7, 1), (16, 1)])
def test_single_tokens(cache_dtype, dim, heads, kv_heads):
    kl = [1, 2, 15, 16, 17, 63, 64, 65, 257, 300]
    run([1] * len(kl), kl, 16, heads, kv_heads, dim, cache_dtype, max_q_len=1, max_kv_len=300)


@pytest.mark.parametrize("cache_dtype", CACHES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (6, 2)])
@pytest.mark.parametrize("accumulate", [True, False])
def test_prompts_and_tokens(cache_dtype, dim, heads, kv_heads, accumulate):
    """Whole prompts, a chunk behind cached keys, single tokens, requests without
    tokens, in one batch."""
    ql = [70, 1, 33, 0, 1, 150, 5, 0]
    kl = [70, 90, 200, 40, 1, 150, 261, 0]
    run(ql, kl, 16, heads, kv_heads, dim, cache_dtype, accumulate=accumulate, max_q_len=150,
        max_kv_len=261)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cache_dtype", [torch.float8_e4m3fn, torch.int8])
def test_codes_against_queries_of_both_types(dtype, cache_dtype):
    run([40, 1, 300], [100, 77, 300], 8, 8, 2, 128, cache_dtype, dtype)


@pytest.mark.parametrize("window", [1, 7, 64, 100, 1 << 30, (1 << 31) - 1])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("accumulate", [True, False])
def test_windows(window, causal, accumulate):
    run([1, 90, 300, 20], [130, 200, 300, 20], 16, 4, 2, 64, torch.bfloat16, window=window,
        causal=causal, accumulate=accumulate)


@pytest.mark.parametrize("page", [1, 2, 64, 1024])
@pytest.mark.parametrize("causal", [True, False])
def test_pages(page, causal):
    run([1, 65, 130], [1100, 65, 700], page, 4, 2, 64, torch.bfloat16, causal=causal)


def test_bounds_below_the_lengths():
    """Requests longer than the bounds are computed all the same."""
    for q, m in ((1, 1), (1, 300), (300, 1), (3, 70)):
        run([1, 90, 300, 5], [1300, 900, 300, 700], 16, 4, 2, 64, torch.bfloat16, max_q_len=q,
            max_kv_len=m)


@pytest.mark.parametrize("accumulate", [True, False])
def test_more_tokens_than_keys(accumulate):
    """Tokens before the first key see nothing, where causal; their log-sums are
    -infinity."""
    run([30, 200], [10, 130], 16, 4, 2, 64, torch.bfloat16, accumulate=accumulate)
    run([30, 200], [10, 130], 16, 4, 2, 64, torch.float16, accumulate=accumulate, causal=False,
        window=20)


def test_keys_that_are_not_there():
    """Holes have no weight and take nothing from others; a row that sees only
    holes counts nothing."""
    def holes(pages):
        pages[0, 0], pages[1, 2], pages[2, 0], pages[2, 1] = -1, 1 << 20, -5, 1 << 30

    for cache_dtype in (torch.bfloat16, torch.int8):
        run([1, 60, 100], [100, 100, 100], 16, 4, 2, 64, cache_dtype, change=holes)
        run([1, 60, 20], [100, 100, 20], 16, 4, 2, 64, cache_dtype, change=holes, accumulate=False)


@pytest.mark.parametrize("scale", [1e-3, 0.5])
def test_scales(scale):
    run([1, 100], [70, 100], 16, 4, 4, 64, torch.bfloat16, scale=scale)


def test_a_key_that_is_not_finite():
    """It spoils its own weight, and no other, whoever does not see it."""
    q, pages, starts, lens, n = batch([100, 1], [100, 90], 16, 4, 64, torch.bfloat16, 5)
    c = fill(n, 16, 2, 64, torch.bfloat16, 6)
    lse = attend(q, c, pages, starts, lens)[1].float()
    want, tol = weighed(q, lse, c, pages, starts, lens, torch.zeros(n, 2, 16))
    for j, h in ((50, 0), (99, 1)):
        c.k[int(pages[0, j // 16]), h, j % 16, 3] = float("nan")
        want[int(pages[0, j // 16]), h, j % 16] = float("nan")
    got = torch.zeros(n, 2, 16).cuda()
    kv.weigh(q.cuda(), lse.cuda(), c, pages.cuda(), starts.cuda(), lens.cuda(), got)
    within(got, want, tol, "beside a NaN")


def test_special_log_sums():
    """+infinity takes a row's weights to zero, -infinity counts nothing, NaN is
    the keys' that the row sees and no others'."""
    q, pages, starts, lens, n = batch([5, 1], [40, 90], 16, 2, 64, torch.float16, 7)
    c = fill(n, 16, 2, 64, torch.float16, 8)
    lse = attend(q, c, pages, starts, lens)[1].float()
    lse[1, 0], lse[2, 1], lse[3, 0] = math.inf, -math.inf, math.nan
    finite = lse.clone()
    finite[1, 0] = finite[2, 1] = finite[3, 0] = -math.inf
    w = torch.rand(n, 2, 16, generator=torch.Generator().manual_seed(9))
    want, tol = weighed(q, finite, c, pages, starts, lens, w)
    j = torch.arange(39)   # what the fourth token sees: position 38
    want[pages[0].long()[j // 16], 0, j % 16] = math.nan
    got = w.cuda()
    kv.weigh(q.cuda(), lse.cuda(), c, pages.cuda(), starts.cuda(), lens.cuda(), got)
    within(got, want, tol, "special log-sums")


def test_rows_that_are_not_the_batchs_stay():
    """Weights of free pages, of other requests, behind a request's end; stale
    weights of new keys do not count, whatever they are."""
    q, pages, starts, lens, n = batch([3, 1], [19, 40], 16, 2, 64, torch.bfloat16, 10, spare=7)
    c = fill(n, 16, 2, 64, torch.bfloat16, 11)
    lse = attend(q, c, pages, starts, lens)[1].float()
    w = torch.rand(n, 2, 16, generator=torch.Generator().manual_seed(12))
    clean = w.clone()
    for b, j in ((0, 16), (0, 17), (0, 18), (1, 39)):
        w[int(pages[b, j // 16]), :, j % 16] = math.nan
        clean[int(pages[b, j // 16]), :, j % 16] = 0.0
    for b, m in ((0, 19), (1, 40)):
        for j in range(m, -(-m // 16) * 16):
            w[int(pages[b, j // 16]), :, j % 16] = -7.0
            clean[int(pages[b, j // 16]), :, j % 16] = -7.0
    want, tol = weighed(q, lse, c, pages, starts, lens, clean)
    got = w.cuda()
    kv.weigh(q.cuda(), lse.cuda(), c, pages.cuda(), starts.cuda(), lens.cuda(), got)
    within(got, want, tol, "rows of others")


def test_strided_queries_and_a_table_with_a_stride():
    q, pages, starts, lens, n = batch([90, 1], [120, 300], 16, 4, 128, torch.bfloat16, 13)
    c = fill(n, 16, 2, 128, torch.bfloat16, 14)
    lse = attend(q, c, pages, starts, lens)[1].float()
    w = torch.zeros(n, 2, 16)
    want, tol = weighed(q, lse, c, pages, starts, lens, w)
    wide = torch.full((2, pages.shape[1] + 3), 1 << 30, dtype=torch.int32)
    wide[:, :pages.shape[1]] = pages
    for first, heads_first in ((0, False), (1, False), (8, True), (3, True)):
        base = torch.zeros((4, 91, 140) if heads_first else (91, 4, 140), dtype=torch.bfloat16).cuda()
        x = base[..., first:first + 128]
        x = x.transpose(0, 1) if heads_first else x
        x.copy_(q)
        got = w.cuda()
        kv.weigh(x, lse.cuda(), c, wide.cuda()[:, :pages.shape[1]], starts.cuda(), lens.cuda(), got)
        within(got, want, tol, f"from {first}")


def test_the_same_bits_and_what_weights_add_up_to():
    """Two calls agree bit for bit; the weights of a request add up to its tokens
    and heads; log-sums are attention's."""
    ql, kl = [1, 700, 40], [1500, 700, 900]
    q, pages, starts, lens, n = batch(ql, kl, 16, 8, 128, torch.bfloat16, 15)
    c = fill(n, 16, 2, 128, torch.bfloat16, 16)
    dev = [t.cuda() for t in (q, pages, starts, lens)]
    _, lse = kv.attention(dev[0], c, *dev[1:], return_lse=True)
    got = []
    for _ in range(3):
        w = torch.zeros(n, 2, 16).cuda()
        kv.weigh(dev[0], lse, c, *dev[1:], w)
        got.append(w)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
    for b, m in enumerate(kl):
        j = torch.arange(m)
        total = got[0].cpu().double()[pages[b].long()[j // 16], :, j % 16].sum(0)
        # a row's weights add up to one, off by a score's error
        assert float((total / (4 * ql[b]) - 1).abs().max()) < 1e-4


def test_a_workspace_of_ones_own():
    ql, kl = [300], [300]
    q, pages, starts, lens, n = batch(ql, kl, 16, 8, 64, torch.bfloat16, 17)
    c = fill(n, 16, 1, 64, torch.bfloat16, 18)
    lse = attend(q, c, pages, starts, lens)[1].float()
    dev = [t.cuda() for t in (q, lse, pages, starts, lens)]
    a, b = (torch.zeros(n, 1, 16).cuda() for _ in range(2))
    size = kv.weigh_workspace_bytes(dev[0], c, *dev[2:])
    ws = torch.full((size + 64,), 0xff, dtype=torch.uint8).cuda()
    kv.weigh(dev[0], dev[1], c, *dev[2:], a, workspace=ws[:size])
    kv.weigh(dev[0], dev[1], c, *dev[2:], b)
    assert torch.equal(a, b) and bool((ws[size:] == 0xff).all())
    if size:
        with pytest.raises(Exception, match="workspace"):
            kv.weigh(dev[0], dev[1], c, *dev[2:], b, workspace=ws[:size - 16])


def test_long_contexts():
    """Keys in many workgroups, tokens in many blocks."""
    run([1, 32], [9000, 5000], 64, 8, 1, 64, torch.int8, max_q_len=32, max_kv_len=9000)
    run([1100], [1100], 16, 4, 1, 64, torch.bfloat16)


@pytest.mark.parametrize("cache_dtype", [torch.bfloat16, torch.int8])
@pytest.mark.parametrize("dim,heads", [(64, 7), (128, 3), (128, 16), (256, 5), (64, 96)])
def test_rows_in_parts(cache_dtype, dim, heads):
    """Few keys for many rows, which several workgroups share; groups that do not
    fill blocks of rows, and larger ones."""
    n = 900 if heads < 16 else 260
    for ql, kl, kw in (([n], [n], {}), ([n // 2], [n // 2 + 300], dict(window=70)),
                       ([n, 3], [100, 500], dict(causal=False)), ([n], [n], dict(accumulate=False))):
        run(ql, kl, 16, heads, 1, dim, cache_dtype, **kw)


def test_no_tokens():
    """A batch without tokens leaves weights as they are, or takes its requests' to
    zero where nothing counts."""
    c = fill(4, 16, 2, 64, torch.bfloat16, 20)
    q, lse = torch.zeros(0, 4, 64).bfloat16().cuda(), torch.zeros(0, 4).cuda()
    pages = torch.tensor([[2, 0]], dtype=torch.int32).cuda()
    starts, lens = torch.zeros(2, dtype=torch.int32).cuda(), torch.tensor([20], dtype=torch.int32).cuda()
    w = torch.ones(4, 2, 16).cuda()
    kv.weigh(q, lse, c, pages, starts, lens, w)
    assert bool((w == 1).all())
    kv.weigh(q, lse, c, pages, starts, lens, w, accumulate=False)
    want = torch.ones(4, 2, 16)
    want[2], want[0, :, :4] = 0, 0
    assert torch.equal(w.cpu(), want)
    none = torch.zeros(0, dtype=torch.int32).cuda()
    kv.weigh(q, lse, c, pages[:0], starts[:1], none, w)
    assert torch.equal(w.cpu(), want)


def test_written_weights_count_a_version():
    q, pages, starts, lens, n = batch([1], [20], 16, 2, 64, torch.float16, 21)
    c = fill(n, 16, 2, 64, torch.float16, 22)
    w = torch.zeros(n, 2, 16).cuda()
    before = w._version, c.k._version
    kv.weigh(q.cuda(), torch.zeros(1, 2).cuda(), c, pages.cuda(), starts.cuda(), lens.cuda(), w)
    assert (w._version, c.k._version) == (before[0] + 1, before[1])
