"""Attention over the pages of a cache, on the GPU, against its definition in 64
bits: lengths from none to thousands, shared heads, windows, holes, page ends
inside tiles, unbounded values in masked places, parts that are joined."""
import math

import pytest
import torch

from kv_util import attend, within

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16
E4, I8 = torch.float8_e4m3fn, torch.int8


@pytest.fixture(scope="module")
def kv():
    from paper_2504_11320_amd import kv
    return kv


def make(kv, q_lens, kv_lens, heads, kv_heads, dim, page, ctype, qtype, seed=0, tail=None,
         spread=1.5):
    """A batch over a cache whose rows behind a request's end hold `tail`."""
    g = torch.Generator()
    g.manual_seed(seed + 7 * sum(kv_lens) + sum(q_lens) + dim)
    need = [-(-m // page) for m in kv_lens]
    pages = sum(need) + 3
    cache = kv.Cache.empty(pages, page, kv_heads, dim, ctype)
    at = torch.randperm(pages, generator=g).int()
    table = torch.full((len(kv_lens), max(need + [1])), -1, dtype=torch.int32)
    a = 0
    for b, n in enumerate(need):
        table[b, :n] = at[a:a + n]
        a += n
    slots = []
    for b, m in enumerate(kv_lens):
        j = torch.arange(m)
        slots.append(table[b].long()[j // page] * page + j % page)
    slots = torch.cat(slots) if slots else torch.zeros(0, dtype=torch.int64)
    if tail is not None:  # what an earlier owner left behind
        if ctype in (E4, I8):
            cache.k.view(torch.uint8).fill_(0x7F)
            cache.v.view(torch.uint8).fill_(0x7F)
            cache.k_scale.fill_(tail)
            cache.v_scale.fill_(tail)
        else:
            cache.k.fill_(tail)
            cache.v.fill_(tail)
    n = slots.numel()
    k = torch.randn(n, kv_heads, dim, generator=g) * torch.exp2(0.7 * torch.randn(dim, generator=g))
    v = torch.randn(n, kv_heads, dim, generator=g)
    if n:
        kv.append(cache, k.cuda(), v.cuda(), slots.cuda())
    starts = [0]
    for n in q_lens:
        starts.append(starts[-1] + n)
    q = (spread * torch.randn(starts[-1], heads, dim, generator=g)).to(qtype)
    return dict(q=q.cuda(), cache=cache, pages=table.cuda(),
                starts=torch.tensor(starts, dtype=torch.int32, device="cuda"),
                kv_lens=torch.tensor(kv_lens, dtype=torch.int32, device="cuda"))


def check(kv, s, what, causal=True, window=0, scale=None, **hints):
    out, lse = kv.attention(s["q"], s["cache"], s["pages"], s["starts"], s["kv_lens"],
                            causal=causal, window=window, scale=scale, return_lse=True, **hints)
    o, L, tol, ltol = attend(s["q"], s["cache"], s["pages"], s["starts"], s["kv_lens"], scale,
                             causal, window)
    covered = int(s["starts"][-1])
    within(out[:covered], o[:covered], tol[:covered], what)
    within(lse[:covered], L[:covered], ltol[:covered], what + ", lse")
    return out


TYPES = [(BF, BF), (FP, FP), (E4, BF), (E4, FP), (I8, BF), (I8, FP)]


@pytest.mark.parametrize("ctype,qtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("group", [1, 4])
def test_single_tokens(kv, ctype, qtype, dim, group):
    """One token a request, key lengths around every tile boundary, a request
    without keys."""
    lens = [1, 0, 2, 15, 16, 17, 31, 32, 33, 63, 64, 127, 128, 129, 160, 161, 300]
    s = make(kv, [1] * len(lens), lens, 2 * group, 2, dim, 16, ctype, qtype, tail=math.nan)
    out = check(kv, s, f"single tokens {ctype} {dim}", max_q_len=1)
    assert bool((out[1] == 0).all())


@pytest.mark.parametrize("ctype,qtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts(kv, ctype, qtype, dim, causal):
    """Prompts of ragged lengths beside single tokens, with and without a
    context before them, empty requests in between, rows that see no key."""
    q = [5, 1, 33, 0, 64, 1, 130, 20, 17]
    m = [5, 40, 33, 9, 100, 0, 131, 8, 17]
    s = make(kv, q, m, 3, 1, dim, 32, ctype, qtype, tail=math.inf)
    check(kv, s, f"prompts {ctype} {dim}", causal)


@pytest.mark.parametrize("page", [1, 2, 8, 64, 1024])
@pytest.mark.parametrize("ctype", [BF, E4])
def test_page_sizes(kv, ctype, page):
    s = make(kv, [1, 40, 3], [77, 130, 259], 4, 2, 128, page, ctype, BF, tail=math.nan)
    check(kv, s, f"pages of {page}")


@pytest.mark.parametrize("group", [1, 2, 7, 16, 17, 33])
def test_shared_heads(kv, group):
    """Groups that fill a block of rows, and that do not fit one."""
    s = make(kv, [1, 2, 9], [50, 70, 100], 2 * group, 2, 64, 16, E4, BF)
    check(kv, s, f"{group} heads a KV head")
    check(kv, s, f"{group} heads a KV head", max_q_len=1)


@pytest.mark.parametrize("window", [1, 2, 31, 64, 100, 5000])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(kv, window, causal):
    s = make(kv, [1, 1, 200, 6], [500, 3, 333, 150], 2, 1, 64, 16, BF, BF, tail=math.nan)
    check(kv, s, f"window {window}", causal, window)


def test_holes(kv):
    """Pages that are not there: their keys are not either, and a request all of
    whose pages are missing has no keys."""
    for ctype in (BF, I8):
        s = make(kv, [1, 50, 1, 20], [100, 120, 60, 20], 2, 2, 64, 8, ctype, BF, tail=math.nan)
        p = s["pages"]
        p[0, 0] = -1
        p[0, 5] = s["cache"].pages
        p[1, 3:7] = -5
        p[1, 14] = 1 << 30
        p[2, :] = -1
        p[3, 0] = -1
        out = check(kv, s, "holes")
        assert bool((out[int(s["starts"][2])] == 0).all())
        assert bool((out[int(s["starts"][3])] == 0).all())   # sees the first page alone


def test_lengths_behind_the_table(kv):
    """Keys behind the table's columns are not there."""
    s = make(kv, [1, 30], [64, 90], 2, 1, 64, 16, BF, BF)
    s["pages"] = s["pages"][:, :3].contiguous()
    check(kv, s, "short table")


@pytest.mark.parametrize("ctype", [BF, I8])
@pytest.mark.parametrize("group", [1, 8])
def test_long_requests_are_split(kv, ctype, group):
    """One long request: parts over its keys are joined.  With the launch laid
    out for less than there is, and for more."""
    m = 5003
    s = make(kv, [1], [m], group, 1, 64, 16, ctype, BF, tail=math.nan)
    for bound in (m, 100, 1, 0, None):
        check(kv, s, f"split, laid out for {bound}", max_q_len=1, max_kv_len=bound)
    check(kv, s, "split, window", window=3000, max_q_len=1)
    s = make(kv, [40], [2500], group, 1, 64, 16, ctype, BF, tail=math.nan)
    for bound in (2500, 600, None):
        check(kv, s, f"split prompt, laid out for {bound}", max_kv_len=bound)
    check(kv, s, "prompt laid out for one token", max_q_len=1)
    check(kv, s, "prompt laid out for two tokens", max_q_len=17)


def test_split_request_beside_empty_ones(kv):
    s = make(kv, [1, 1, 0, 25, 1], [3000, 0, 10, 1800, 1], 2, 2, 64, 32, E4, FP, tail=math.nan)
    check(kv, s, "split beside empty")
    check(kv, s, "split beside empty, no causal", causal=False)


def _unbounded_case(kv, ctype, q_lens, kv_lens, where, value):
    """Values that are not finite at a key that only some queries see."""
    s = make(kv, q_lens, kv_lens, 2, 1, 64, 16, ctype, BF)
    c = s["cache"]
    for b, j in where:
        page = int(s["pages"][b, j // 16])
        if c.k_scale is None:
            c.v[page, 0, j % 16, 5] = value
            c.v[page, 0, j % 16, 40] = -value
        else:
            c.v_scale[page, 0, j % 16] = math.nan
    return s


@pytest.mark.parametrize("ctype", [BF, FP, E4, I8])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_unbounded_values_reach_only_those_who_see_them(kv, ctype, value):
    """A token's output does not depend on what lies behind its own position, or
    before its window."""
    for q, m, where in (([6], [40], [(0, 37)]), ([50], [120], [(0, 100), (0, 119)]),
                        ([1, 150], [9, 150], [(0, 8), (1, 70)])):
        s = _unbounded_case(kv, ctype, q, m, where, value)
        if ctype == FP:
            s["q"] = s["q"].half()
        for window in (0, 20):
            got = kv.attention(s["q"], s["cache"], s["pages"], s["starts"], s["kv_lens"],
                               window=window).cpu().float()
            for b, j in where:
                for i in range(q[b]):
                    p = m[b] - q[b] + i
                    see = any(bb == b and jj <= p and (not window or jj > p - window)
                              for bb, jj in where)
                    row = got[int(s["starts"][b]) + i]
                    if not see:
                        assert bool(torch.isfinite(row).all()), (ctype, b, i)
                    else:
                        assert not bool(torch.isfinite(row[:, 5]).any()), (ctype, b, i)
                        if ctype in (BF, FP):
                            rest = [d for d in range(64) if d not in (5, 40)]
                            assert bool(torch.isfinite(row[:, rest]).all())


def test_unbounded_keys_and_queries(kv):
    """A key that is NaN makes the rows that see it NaN and no others; so does a
    query its own row."""
    for ctype in (BF, E4):
        s = make(kv, [30, 1], [90, 50], 2, 1, 64, 16, ctype, BF)
        c = s["cache"]
        page = int(s["pages"][0, 70 // 16])
        if c.k_scale is None:
            c.k[page, 0, 70 % 16, 3] = math.nan
        else:
            c.k_scale[page, 0, 70 % 16] = math.nan
        s["q"][30, 1, 9] = math.nan
        out, lse = kv.attention(s["q"], c, s["pages"], s["starts"], s["kv_lens"], return_lse=True)
        for i in range(30):
            assert bool(torch.isnan(out[i]).all()) == (60 + i >= 70), i
            assert bool(torch.isfinite(out[i]).all()) == (60 + i < 70), i
        assert bool(torch.isfinite(out[30, 0]).all()) and bool(torch.isnan(out[30, 1]).all())
        assert bool(torch.isnan(lse[30, 1])) and bool(torch.isfinite(lse[30, 0]))


@pytest.mark.parametrize("ctype,qtype", TYPES)
def test_sharp_and_large_scores(kv, ctype, qtype):
    """Scores of hundreds: the running maximum moves, weights underflow."""
    s = make(kv, [1, 70], [700, 200], 2, 1, 128, 16, ctype, qtype, spread=60.0)
    check(kv, s, "sharp")
    check(kv, s, "given scale", scale=0.001)


def test_rows_of_zero_and_tiny_values(kv):
    """8-bit rows whose scales span the range, zeros among them."""
    for ctype in (E4, I8):
        s = make(kv, [1, 40], [90, 80], 2, 1, 64, 16, ctype, BF)
        c = s["cache"]
        g = torch.Generator().manual_seed(3)
        by = torch.exp2(torch.randint(-40, 20, c.v_scale.shape, generator=g).float()).cuda()
        c.v_scale *= by
        c.v_scale[:, :, ::5] = 0
        c.v.view(torch.uint8)[:, :, ::5] = 0
        check(kv, s, "scales far apart")
        c.v_scale.zero_()
        c.v.view(torch.uint8).zero_()
        out = check(kv, s, "all values zero")
        assert bool((out == 0).all())


def test_queries_bf16_of_any_size(kv):
    """bf16 queries far outside the 16-bit range that the codes' products use."""
    s = make(kv, [4, 40], [90, 80], 2, 1, 64, 16, I8, BF)
    for by in (2.0 ** 90, 2.0 ** -90):
        t = dict(s, q=(s["q"].float() * by).bfloat16())
        check(kv, t, f"queries times {by}", scale=0.125 / by)


def test_strides(kv):
    """Queries and outputs within larger tensors, a page table with more
    columns, unaligned bases."""
    s = make(kv, [1, 20, 3], [30, 60, 90], 4, 2, 64, 16, E4, BF)
    want = check(kv, s, "contiguous")
    T = s["q"].shape[0]
    for wide, shift in ((64 + 8, 8), (64 + 3, 1)):
        big = torch.zeros(T, 6, wide, dtype=BF, device="cuda")
        big[:, 1:5, shift:shift + 64] = s["q"]
        out = torch.full((T, 6, wide), 9.0, dtype=BF, device="cuda")
        kv.attention(big[:, 1:5, shift:shift + 64], s["cache"], s["pages"], s["starts"],
                     s["kv_lens"], out=out[:, 1:5, shift:shift + 64])
        assert torch.equal(out[:, 1:5, shift:shift + 64], want)
        out[:, 1:5, shift:shift + 64] = 9.0
        assert bool((out == 9.0).all())
    qt = s["q"].transpose(0, 1).contiguous().transpose(0, 1)
    pages = torch.full((3, 20), -1, dtype=torch.int32, device="cuda")
    pages[:, :s["pages"].shape[1]] = s["pages"]
    assert torch.equal(kv.attention(qt, s["cache"], pages[:, :s["pages"].shape[1]], s["starts"],
                                    s["kv_lens"]), want)


def test_rows_outside_requests_stay(kv):
    s = make(kv, [3, 30], [10, 40], 2, 1, 64, 16, BF, BF)
    q = torch.cat([s["q"], s["q"][:4]])
    out = torch.full_like(q, 5.0)
    kv.attention(q, s["cache"], s["pages"], s["starts"], s["kv_lens"], out=out)
    assert bool((out[33:] == 5.0).all()) and bool((out[:33] != 5.0).any())
    none = kv.attention(q[:0], s["cache"], s["pages"][:0], s["starts"][:1], s["kv_lens"][:0])
    assert none.shape == (0, 2, 64)


def test_long_cache(kv):
    """Pages whose byte and element offsets pass 32 bits."""
    heads, dim, page = 4, 256, 64
    pages = (5 << 30) // (heads * dim * page)
    k = torch.empty((pages, heads, page, dim), dtype=I8, device="cuda")
    cache = kv.Cache(k, torch.empty_like(k),
                     *(torch.zeros(pages, heads, page, device="cuda") for _ in range(2)))
    lens, q = [200, 130], [1, 40]
    table = torch.tensor([[pages - 1, pages - 2, pages // 2 + 1, pages - 7],
                          [pages - 4, pages - 5, pages - 6, -1]], dtype=torch.int32)
    g = torch.Generator().manual_seed(2)
    small = kv.Cache.empty(7, page, heads, dim, I8)
    stable = torch.tensor([[0, 1, 2, 3], [4, 5, 6, -1]], dtype=torch.int32)
    for b, m in enumerate(lens):
        j = torch.arange(m)
        x, y = (torch.randn(m, heads, dim, generator=g).cuda() for _ in range(2))
        for c, t in ((cache, table), (small, stable)):
            kv.append(c, x, y, (t[b].long()[j // page] * page + j % page).cuda())
    qq = torch.randn(41, 8, dim, generator=g).half().cuda()
    starts = torch.tensor([0, 1, 41], dtype=torch.int32, device="cuda")
    kl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    assert torch.equal(kv.attention(qq, cache, table.cuda(), starts, kl),
                       kv.attention(qq, small, stable.cuda(), starts, kl))


def test_same_bits_again(kv):
    """No order of atomics: the same call gives the same bits, whatever ran
    between."""
    s = make(kv, [1, 40], [4000, 900], 4, 2, 128, 16, E4, BF)
    first = kv.attention(s["q"], s["cache"], s["pages"], s["starts"], s["kv_lens"])
    for _ in range(3):
        kv.attention(-s["q"], s["cache"], s["pages"], s["starts"], s["kv_lens"])
        assert torch.equal(first, kv.attention(s["q"], s["cache"], s["pages"], s["starts"],
                                               s["kv_lens"]))


def test_streams_graph_and_workspace(kv):
    s = make(kv, [1, 1], [2000, 700], 4, 2, 128, 16, E4, BF)
    args = (s["q"], s["cache"], s["pages"], s["starts"], s["kv_lens"])
    want = kv.attention(*args)
    size = kv.attention_workspace_bytes(*args)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kv.attention(*args, out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv.attention(*args, out=out, workspace=ws)
    for i in range(3):
        # lengths change on the device between replays
        s["kv_lens"].copy_(torch.tensor([2000 - 300 * i, 700 - 100 * i], dtype=torch.int32))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, kv.attention(*args))


def test_steps_agree_with_the_whole_prompt(kv):
    """Decoding a prompt token by token gives what prefilling it gives, row by
    row, within the sum of the bounds."""
    n = 70
    s = make(kv, [n], [n], 4, 2, 64, 16, E4, FP)
    whole = kv.attention(s["q"], s["cache"], s["pages"], s["starts"], s["kv_lens"])
    o, _, tol, _ = attend(s["q"], s["cache"], s["pages"], s["starts"], s["kv_lens"])
    for i in (0, 1, 31, 32, 69):
        one = kv.attention(s["q"][i:i + 1], s["cache"], s["pages"],
                           torch.tensor([0, 1], dtype=torch.int32, device="cuda"),
                           torch.tensor([i + 1], dtype=torch.int32, device="cuda"))
        within(one, o[i:i + 1], tol[i:i + 1], f"step {i}")
        within(whole[i:i + 1], o[i:i + 1], tol[i:i + 1], f"row {i}")
