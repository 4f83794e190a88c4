"""The operators as a server with a budget of cached tokens uses them: a batch
enters, attends, its keys are weighed, and requests go back to their budget."""
import math

import numpy as np
import pytest
import torch

from kv_more_util import kept_keys, weighed
from kv_util import attend, rows_of, within
from paper_2504_11320_amd import iteration as I
from paper_2504_11320_amd import kv

pytestmark = pytest.mark.gpu

H, KH, D, PAGE = 4, 2, 64, 16


def gen(seed):
    return torch.Generator().manual_seed(seed)


def vectors(n, heads, dtype, seed):
    return torch.randn(n, heads, D, generator=gen(seed)).to(dtype).cuda()


class Request:
    """One request on pages of its own, and what its keys are and have received,
    head by head, kept on the CPU."""

    def __init__(self, cache, pages):
        self.cache, self.pages, self.length, self.position = cache, pages, 0, 0
        self.keys = [[] for _ in range(KH)]     # (key, value) in 64 bits
        self.weights = torch.zeros(cache.pages, KH, PAGE).cuda()

    def step(self, n, seed, keep, recent, table, norms):
        """n tokens in; the outputs, checked; back to the budget."""
        c = self.cache
        dtype = c.dtype if c.k_scale is None else torch.bfloat16
        q, k, v = vectors(n, H, dtype, seed), vectors(n, KH, dtype, seed + 1), vectors(n, KH, dtype, seed + 2)
        j = torch.arange(self.length, self.length + n)
        slots = self.pages[0].cpu().long()[j // PAGE] * PAGE + j % PAGE
        pos = torch.arange(self.position, self.position + n).cuda()
        q = kv.enter(c, q, k, v, slots.cuda(), positions=pos, table=table, q_norm=norms[0],
                     k_norm=norms[1])
        new_k, new_v = rows_of(c, "k", slots), rows_of(c, "v", slots)
        for h in range(KH):
            self.keys[h] += [(new_k[i, h], new_v[i, h]) for i in range(n)]
        self.length += n
        self.position += n
        starts = torch.tensor([0, n], dtype=torch.int32).cuda()
        lens = torch.tensor([self.length], dtype=torch.int32).cuda()
        batch = (c, self.pages, starts, lens)
        out, lse = kv.attention(q, *batch, return_lse=True)
        # attention over what this request's books hold, not over the cache
        want, wlse, tol, ltol = attend(q, c, self.pages, starts, lens)
        for h in range(H):
            ks = torch.stack([x for x, _ in self.keys[h // (H // KH)]])
            vs = torch.stack([x for _, x in self.keys[h // (H // KH)]])
            for i in range(n):
                m = self.length - n + i + 1
                z = ks[:m] @ q[i, h].cpu().double() / math.sqrt(D)
                w = torch.softmax(z, 0)
                assert float((w @ vs[:m] - want[i, h]).abs().max()) < 1e-12
        within(out, want, tol, "attention")
        within(lse, wlse, ltol, "log-sums")
        before = self.weights.clone()
        kv.weigh(q, lse, *batch, self.weights)
        expect, wtol = weighed(q, lse, c, self.pages, starts, lens, before)
        within(self.weights, expect, wtol, "weights")
        held = self.weights.cpu()
        kept, left = kv.evict(c, self.pages, lens, self.weights, keep=keep, recent=recent)
        for h in range(KH):
            at = torch.arange(self.length)
            w = held[self.pages[0].cpu().long()[at // PAGE], h, at % PAGE]
            idx = kept_keys(w, keep, recent)
            assert kept[0, h, :len(idx)].tolist() == idx
            self.keys[h] = [self.keys[h][i] for i in idx]
        self.length = min(self.length, keep)
        assert left.tolist() == [self.length]
        at = torch.arange(self.length)
        slots = self.pages[0].cpu().long()[at // PAGE] * PAGE + at % PAGE
        for name, which in (("k", 0), ("v", 1)):
            rows = rows_of(c, name, slots)
            for h in range(KH):
                assert torch.equal(rows[:, h], torch.stack([x[which] for x in self.keys[h]]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8])
def test_a_request_on_a_budget(dtype):
    cache = kv.Cache.empty(12, PAGE, KH, D, dtype)
    pages = torch.randperm(12, generator=gen(1))[:8].int().reshape(1, 8).cuda()
    table = kv.rotary_table(400, D)
    norms = [torch.empty(D).normal_(1.0, 0.2, generator=gen(i)).cuda() for i in (2, 3)]
    r = Request(cache, pages)
    for i, n in enumerate((70, 1, 1, 20, 1, 3)):
        r.step(n, 10 + 3 * i, 40, 10, table, norms)


def test_captured_and_replayed():
    """The chain in a graph, with the kept rows going to other pages: every replay
    gives the eager results, with other work and other inputs between."""
    n, old = 3, 60
    cache = kv.Cache.empty(16, PAGE, KH, D)
    cache.k.normal_(generator=torch.Generator("cuda").manual_seed(4))
    cache.v.normal_(generator=torch.Generator("cuda").manual_seed(5))
    pages = torch.tensor([[3, 1, 7, 5]], dtype=torch.int32).cuda()
    to = torch.tensor([[8, 9]], dtype=torch.int32).cuda()
    x = [vectors(n, h, torch.bfloat16, 6 + h) for h in (H, KH, KH)]
    slots = torch.tensor([5 * 16 + 12 + i for i in range(n)]).cuda()
    pos = torch.arange(old, old + n).cuda()
    table = kv.rotary_table(100, D)
    norm = torch.ones(D).cuda()
    starts, lens = torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([old + n], dtype=torch.int32).cuda()
    weights = torch.zeros(16, KH, PAGE).cuda()

    def chain():
        q = kv.enter(cache, x[0], x[1], x[2], slots, positions=pos, table=table, q_norm=norm, k_norm=norm)
        out, lse = kv.attention(q, cache, pages, starts, lens, return_lse=True)
        kv.weigh(q, lse, cache, pages, starts, lens, weights, accumulate=False)
        kept, left = kv.evict(cache, pages, lens, weights, keep=32, recent=8, to=to)
        return out, lse, kept, left, weights, cache.k, cache.v

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = chain()
    def stale():   # what no call may take into account
        weights.fill_(7.0)
        cache.k[8:10].zero_()
        cache.v[8:10].zero_()

    for i in range(4):
        stale()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in got]
        stale()
        for a, b in zip(replayed, chain()):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        (x[0].float().flatten(1) @ x[0].float().flatten(1).T).sum().item()
        for t in x:
            t.mul_(-0.75)


def _server(cache=torch.bfloat16, layers=2, **kw):
    shape = I.Shape(layers=layers, heads=4, kv_heads=2, dim=64, ffn=320, cache=cache, **kw)
    return I.Server(shape, tokens=2048, page_size=16, positions=512)


def test_a_budget_that_nothing_exceeds_changes_nothing():
    x = torch.randn(133, 256, generator=gen(7)).bfloat16().cuda()
    batch = I.Batch([100, 33], [0, 0], 16)
    want = _server().iterate(x, batch)
    sv = _server(keep=100, recent=20)
    assert torch.equal(sv.iterate(x, batch), want)
    # every token's weights add up to one a head
    for w in sv.weights:
        total = w.double().sum((0, 2)).cpu()
        assert float((total / (2 * 133) - 1).abs().max()) < 1e-4


def test_norms_in_an_iteration():
    """An iteration with normed queries and keys is the one that norms, turns and
    appends in calls of their own, bit for bit with a 16-bit cache."""
    x = torch.randn(50, 256, generator=gen(8)).bfloat16().cuda()
    batch = I.Batch([49, 1], [0, 20], 16)
    sv, other = _server(qk_norm=True), _server(qk_norm=True)
    got = sv.iterate(x, batch)
    real = kv.enter

    def apart(cache, q, k, v, slots, positions, table, q_norm, k_norm, out):
        kv.append(cache, kv.norm_rotary(k, k_norm, positions, table), v, slots)
        return kv.norm_rotary(q, q_norm, positions, table)

    kv.enter = apart
    try:
        assert torch.equal(other.iterate(x, batch), got)
    finally:
        kv.enter = real
    plain = _server().iterate(x, batch)
    assert not torch.equal(plain, got)


def test_iterations_on_a_budget():
    """Requests go back to their budget in every layer; the next iteration runs on
    what is left, at the positions that the tokens have."""
    sv = _server(torch.float8_e4m3fn, qk_norm=True, keep=48, recent=16)
    x = torch.randn(200, 256, generator=gen(9)).bfloat16().cuda()
    first = I.Batch([150, 40], [0, 0], 16)
    out = sv.iterate(x[:190], first)
    assert bool(torch.isfinite(out.float()).all())
    then = I.Batch([1, 1], [48, 40], 16, at=[150, 40])
    assert then.positions.tolist() == [150, 40]
    # the second request's pages follow the ten of the first
    then.pages, then.slots = first.pages, torch.tensor([48, 10 * 16 + 40]).cuda()
    out = sv.iterate(x[190:192], then)
    assert bool(torch.isfinite(out.float()).all())
    for b in (dict(at=[1]), dict(at=[-1, 0])):
        with pytest.raises(ValueError):
            I.Batch([1, 1], [3, 4], 16, **b)
    for kw in (dict(keep=4, recent=5), dict(recent=1), dict(keep=-1), dict(keep=4, recent=-1)):
        with pytest.raises(ValueError):
            I.Shape(**kw)


def test_the_command(capsys):
    got = I.main(["--layers", "1", "--prompt", "64", "--out", "3", "--per-stage", "1", "2", "4",
                  "--qk-norm", "--keep", "40", "--recent", "8", "--cache", "int8"])
    assert got["keep"] == 40 and got["recent"] == 8 and len(got["points"]) == 3
    # at stage s a request holds at most 40 tokens and the new one
    assert [p[0] for p in got["points"]] == [n * (64 + 3 * 41) for n in (1, 2, 4)]
    assert np.isfinite(got["d0"]) and '"C"' in capsys.readouterr().out
