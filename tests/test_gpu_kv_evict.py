"""Eviction from a cache by accumulated weights: bit for bit what the definition
keeps and moves."""
import math

import pytest
import torch

from kv_more_util import evicted
from paper_2504_11320_amd import kv

pytestmark = pytest.mark.gpu

CACHES = (torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8)


def make(lens, page, kv_heads, dim, dtype, seed, keep=1, to=False, kind="heavy"):
    """(cache, pages, lens, weights, to): random bits in every row."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-m // page) for m in lens]
    width = -(-keep // page)
    n = sum(need) + 2 + (width * len(lens) if to else 0)
    at = torch.randperm(n, generator=g).int()
    table = torch.full((len(lens), max(need + [1])), -1, dtype=torch.int32)
    a = 0
    for b, c in enumerate(need):
        table[b, :c] = at[a:a + c]
        a += c
    c = kv.Cache.empty(n, page, kv_heads, dim, dtype)
    for x in (c.k, c.v):
        x.view(torch.uint8).copy_(torch.randint(0, 256, x.view(torch.uint8).shape, generator=g,
                                                dtype=torch.uint8))
    for x in (c.k_scale, c.v_scale):
        if x is not None:
            x.copy_(torch.randn(x.shape, generator=g))
    shape = (n, kv_heads, page)
    if kind == "heavy":
        w = torch.exp(2.0 * torch.randn(shape, generator=g))
    elif kind == "few":       # mostly equal ones, zeros of both signs
        w = torch.tensor([0.0, -0.0, 1.0, 2.0])[torch.randint(0, 4, shape, generator=g)]
    elif kind == "equal":
        w = torch.full(shape, 0.25)
    elif kind == "near":      # the last places decide
        w = (torch.randint(0, 50, shape, generator=g, dtype=torch.int32) + 0x3f800000).view(torch.float32)
    else:
        w = torch.randn(shape, generator=g)
        pick = torch.randint(0, 12, shape, generator=g)
        for i, x in enumerate((math.nan, math.inf, -math.inf, -math.nan, 1e-45, -1e-45)):
            w[pick == i] = x
    places = at[a:a + width * len(lens)].reshape(len(lens), width) if to else None
    return c, table, torch.tensor(lens, dtype=torch.int32), w, places


def bits(x):
    return x.view(torch.uint8 if x.element_size() == 1 else
                  torch.int16 if x.element_size() == 2 else torch.int32).cpu()


def check(lens, page, kv_heads, dim, dtype, keep, recent, to, seed=1, kind="heavy", change=None, **kw):
    c, pages, n, w, places = make(lens, page, kv_heads, dim, dtype, seed, keep, to, kind)
    if change:
        change(pages, w)
    kept, left, want = evicted(c, pages, n, w, keep, recent, places)
    got_w = w.cuda()
    got, got_n = kv.evict(c, pages.cuda(), n.cuda(), got_w, keep=keep, recent=recent,
                          to=None if places is None else places.cuda(), **kw)
    assert got.dtype == torch.int32 and torch.equal(got.cpu(), kept), "kept keys"
    assert torch.equal(got_n.cpu(), left), "lengths"
    for name, x in want.items():
        now = got_w if name == "weights" else getattr(c, name)
        assert torch.equal(bits(now), bits(x)), name


LENS = [0, 1, 19, 20, 21, 22, 64, 65, 100, 300]


@pytest.mark.parametrize("dtype", CACHES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("to", [False, True])
def test_types_and_dims(dtype, dim, to):
    check(LENS, 16, 3, dim, dtype, keep=20, recent=5, to=to)


@pytest.mark.parametrize("keep,recent", [(1, 0), (1, 1), (2, 1), (20, 0), (20, 20), (64, 3), (256, 64),
                                         (299, 0), (299, 298), (300, 7), (5000, 0)])
@pytest.mark.parametrize("kind", ["heavy", "few", "equal", "near", "special"])
@pytest.mark.parametrize("to", [False, True])
def test_what_is_kept(keep, recent, kind, to):
    check(LENS, 16, 2, 64, torch.bfloat16, keep, recent, to, seed=keep + 3, kind=kind)


@pytest.mark.parametrize("page", [1, 2, 128, 1024])
@pytest.mark.parametrize("to", [False, True])
def test_pages(page, to):
    check([700, 3, 1025], page, 2, 64, torch.int8, keep=130, recent=30, to=to)


@pytest.mark.parametrize("bound", [None, 1, 300, 5000])
@pytest.mark.parametrize("to", [False, True])
def test_long_requests(bound, to):
    """More keys than shared memory holds the weights of; bounds below and above
    the lengths."""
    check([4096, 4097, 40000, 5], 64, 1, 64, torch.float16, keep=3000, recent=100, to=to,
          max_kv_len=bound)


@pytest.mark.parametrize("to", [False, True])
def test_very_long(to):
    check([131072, 33000], 64, 2, 64, torch.int8, keep=16384, recent=4096, to=to, kind="few")
    check([131072], 64, 1, 64, torch.bfloat16, keep=20000, recent=0, to=to)


def test_many_requests():
    check([33 + i % 7 for i in range(200)], 8, 4, 64, torch.float8_e4m3fn, keep=30, recent=8, to=False)


def test_a_table_of_fewer_columns():
    """Keys behind the table do not count."""
    c, pages, n, w, _ = make([100], 16, 1, 64, torch.bfloat16, 5)
    n[0] = 1000
    cut = torch.tensor([pages.shape[1] * 16], dtype=torch.int32)
    kept, left, want = evicted(c, pages, cut, w, 20, 5)
    got, got_n = kv.evict(c, pages.cuda(), n.cuda(), w.cuda(), keep=20, recent=5)
    assert torch.equal(got.cpu(), kept) and torch.equal(got_n.cpu(), left)
    assert torch.equal(bits(c.k), bits(want["k"]))
    n[0] = -4
    got, got_n = kv.evict(c, pages.cuda(), n.cuda(), w.cuda(), keep=20)
    assert bool((got == -1).all()) and got_n.tolist() == [0]


@pytest.mark.parametrize("to", [False, True])
def test_pages_that_are_not_there(to):
    """Their keys go first, and nothing is written in the place of one that stays
    or into a page that is not there."""
    c, pages, n, w, places = make([64, 64], 16, 2, 64, torch.int8, 6, 40, to)
    pages[0, 1] = -1                       # 16 of 64 keys; 40 of the others stay
    dst = (places if to else pages).clone()
    if to:
        places[1, 2] = 1 << 20             # places 32 .. 39 of the second request
    before = {x: getattr(c, x).cpu().clone() for x in ("k", "v", "k_scale", "v_scale")}
    got, left = kv.evict(c, pages.cuda(), n.cuda(), w.cuda(), keep=40, recent=8,
                         to=places.cuda() if to else None)
    assert left.tolist() == [40, 40]
    ok = [i for i in range(64) if not 16 <= i < 32]
    for h in range(2):
        heavy = sorted(ok[:-8], key=lambda i: (-float(w[int(pages[0, i // 16]), h, i % 16]), i))
        want = sorted(heavy[:32]) + ok[-8:]
        assert got[0, h].tolist() == want
        for d, i in enumerate(want):
            if not to and 16 <= d < 32:    # no place to go to
                continue
            src, page = int(pages[0, i // 16]), int(dst[0, d // 16])
            assert torch.equal(c.k[page, h, d % 16].cpu(), before["k"][src, h, i % 16])
            assert float(c.v_scale[page, h, d % 16]) == float(before["v_scale"][src, h, i % 16])
        if to:
            page = int(dst[1, 2])
            assert torch.equal(c.k[page, h].cpu(), before["k"][page, h])


def test_written_tensors_count_a_version():
    c, pages, n, w, _ = make([50], 16, 1, 64, torch.int8, 7)
    w = w.cuda()
    before = [x._version for x in (c.k, c.v, c.k_scale, c.v_scale, w)]
    kv.evict(c, pages.cuda(), n.cuda(), w, keep=20)
    assert [x._version for x in (c.k, c.v, c.k_scale, c.v_scale, w)] == [x + 1 for x in before]


def test_no_requests():
    c = kv.Cache.empty(2, 16, 2, 64)
    none = torch.zeros(0, dtype=torch.int32).cuda()
    kept, left = kv.evict(c, none.reshape(0, 3), none, torch.zeros(2, 2, 16).cuda(), keep=4)
    assert kept.shape == (0, 2, 4) and left.shape == (0,)
