"""Entering, weighing and evicting in a cache whose offsets pass 32 bits: bit for bit
what a small cache with the same pages gives."""
import pytest
import torch

from paper_2504_11320_amd import kv

pytestmark = pytest.mark.gpu

PAGE, KH, D = 16, 32, 128


def gen(seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    return g


def bits(x):
    return x.view(torch.uint8)


def test_offsets_past_32_bits():
    big = kv.Cache.empty(36000, PAGE, KH, D)           # 4.7 GB each of keys and values
    kl, ql = [300, 90, 2500], [40, 1, 1]
    need = [-(-m // PAGE) for m in kl]
    n = sum(need)
    at = (35999 - torch.randperm(1500, generator=gen(1), device="cuda")[:n + 10]).int()
    assert int(at.min()) * KH * PAGE * D * 2 > 1 << 32
    small = kv.Cache.empty(n + 10, PAGE, KH, D)
    for c in ("k", "v"):
        getattr(small, c).normal_(generator=gen(2))
        getattr(big, c)[at.long()] = getattr(small, c)
    weights = torch.rand(n + 10, KH, PAGE, generator=gen(3), device="cuda")
    wide = torch.zeros(36000, KH, PAGE, device="cuda")
    wide[at.long()] = weights
    table = torch.full((3, max(need)), -1, dtype=torch.int32, device="cuda")
    a = 0
    for b, x in enumerate(need):
        table[b, :x] = torch.arange(a, a + x)
        a += x

    def moved(t):   # the table of the large cache
        return torch.where(t < 0, t, at[t.clamp(min=0).long()])

    starts = torch.tensor([0, 40, 41, 42], dtype=torch.int32, device="cuda")
    lens = torch.tensor(kl, dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(42, h, D, generator=gen(4 + h), device="cuda").bfloat16() for h in (64, KH, KH))
    position = torch.cat([torch.arange(m - x, m) for x, m in zip(ql, kl)]).cuda()
    request = torch.repeat_interleave(torch.arange(3), torch.tensor(ql)).cuda()
    turn = dict(positions=position, table=kv.rotary_table(4096, D), q_norm=torch.ones(D).cuda(),
                k_norm=torch.ones(D).cuda())
    to = torch.arange(n, n + 9, dtype=torch.int32, device="cuda").view(3, 3)
    got = []
    for c, t, w, dst in ((small, table, weights, to), (big, moved(table), wide, moved(to))):
        slots = t[request, position // PAGE].long() * PAGE + position % PAGE
        x = kv.enter(c, q, k, v, slots, **turn)
        out, lse = kv.attention(x, c, t, starts, lens, return_lse=True)
        kv.weigh(x, lse, c, t, starts, lens, w)
        lists = kv.evict(c, t, lens, w, keep=40, recent=8, to=dst)                         # to other pages
        lists += kv.evict(c, t, lens, w, keep=70, recent=8, max_kv_len=2048)               # in place
        got.append((x, out, lse) + lists)
    for a, b in zip(*got):
        assert torch.equal(a, b)
    for a, b in ((small.k, big.k), (small.v, big.v), (weights, wide)):
        assert torch.equal(bits(a), bits(b[at.long()]))
    rest = torch.ones(36000, dtype=torch.bool, device="cuda")
    rest[at.long()] = False
    for x in (big.k, big.v, wide):
        assert not bool(x[rest].any())
