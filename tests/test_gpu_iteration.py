"""The KV path as a serving iteration uses it: a prompt prefilled whole, in
chunks and token by token gives the same hidden states, eagerly and from a
captured graph; the measured times give the simulator a workload that runs."""
import numpy as np
import pytest
import torch

import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def I():
    from paper_2504_11320_amd import iteration
    return iteration


def _server(I, cache, layers=2):
    shape = I.Shape(layers=layers, heads=4, kv_heads=2, dim=64, ffn=320, dtype=torch.bfloat16,
                    cache=cache)
    return I.Server(shape, tokens=2048, page_size=16, positions=512)


def _near(a, b):
    """Two orders of the same computation.  Each layer rounds about ten times to
    bf16 (2^-9 rms each) on both sides, and an 8-bit key or value that falls on
    the other side of a tie moves by 2^-4 of itself, one of D terms: 2 layers *
    2 sides give sqrt(40) * 2^-9 = 0.012, held to three times that."""
    return float((a.float() - b.float()).norm() / b.float().norm()) <= 0.04


@pytest.mark.parametrize("cache", [torch.bfloat16, torch.float8_e4m3fn, torch.int8])
def test_prefill_chunks_and_steps_agree(I, cache):
    n, other = 100, 37
    x = torch.randn(n, 256, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    y = torch.randn(other, 256, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    sv = _server(I, cache)

    def owner(b, n_new, n_old):
        # both requests keep their pages through the run
        batch = I.Batch([n_new, 0] if b == 0 else [0, n_new],
                        [n - n_new, other] if b == 0 else [n, other - n_new], 16)
        return batch

    whole = sv.iterate(torch.cat([x, y]), I.Batch([n, other], [0, 0], 16))
    assert bool(torch.isfinite(whole.float()).all())
    for cuts in ((0, 60, 61, 99, 100), (0, 1, 33, 100)):
        sv = _server(I, cache)
        sv.iterate(y, owner(1, other, 0))
        got = []
        for a, b in zip(cuts[:-1], cuts[1:]):
            batch = I.Batch([b - a, 0], [a, other], 16)
            # the second request's pages follow the whole of the first's
            full = I.Batch([n, other], [0, 0], 16)
            batch.pages = full.pages
            batch.slots = full.slots[a:b].contiguous()
            got.append(sv.iterate(x[a:b], batch))
        assert _near(torch.cat(got), whole[:n])
        # the last token of the other request, beside nothing
        full = I.Batch([n, other], [0, 0], 16)
        last = I.Batch([0, 1], [n, other - 1], 16)
        last.pages, last.slots = full.pages, full.slots[-1:].contiguous()
        assert _near(sv.iterate(y[-1:], last), whole[-1:])


def test_graph_replays(I):
    """An iteration captured into a graph gives the eager result at every
    replay, with the cache overwritten and other work between."""
    sv = _server(I, torch.float8_e4m3fn)
    batch = I.Batch([40, 1, 1], [0, 30, 200], 16)
    x = torch.randn(42, 256, device="cuda").bfloat16()
    for c in sv.caches:   # an old context that is there
        c.k.view(torch.uint8).random_(0, 120)
        c.v.view(torch.uint8).random_(0, 120)
        c.k_scale.uniform_(0.001, 0.01)
        c.v_scale.uniform_(0.001, 0.01)
    want = sv.iterate(x, batch)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sv.iterate(x, batch)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sv.iterate(x, batch)
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        x.mul_(-0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, sv.iterate(x, batch))
        x.mul_(-2.0)
        (x @ x.T).sum().item()


def test_measured_times_drive_the_simulator(I):
    """Iteration times measured on the card, fitted, as a workload that runs."""
    from paper_2504_11320_amd import binding as B
    from paper_2504_11320_amd import calibrate

    sv = _server(I, torch.float8_e4m3fn)
    points = I.measure(sv, [I.stage_batch(16, 4, n) for n in (1, 4, 12)], repeats=3)
    assert [p[0] for p in points] == [n * calibrate.stage_work(16, 4) for n in (1, 4, 12)]
    assert all(p[1] > 0 for p in points)
    got = I.fit(points)
    assert np.isfinite(got["d0"]) and np.isfinite(got["d1"])
    d0, d1, C = max(got["d0"], 1e-3), max(got["d1"], 1e-6), I.budget(sv.shape, 4e6)
    lam = 0.5 * calibrate.fluid_boundary(calibrate.stage_work(16, 4), d0, d1, C)
    wl = W.Workload(prompt_len=[16], lam=[lam], d0=d0, d1=d1, C=C, policy="wait", n=[2],
                    out_len=[4], hist_edges=W.default_edges(d0))
    res = B.run_batch([W.Job(wl, 0, W.ids(64))], horizon=500, device="cuda:0")
    assert bool((res["batches"] == 500).all()) and bool((res["completions"] > 0).all())
