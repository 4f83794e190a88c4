"""Iteration time and KV budget of a transformer on this card, for the
simulator (arXiv 2504.11320, Section 2.2 and the iteration-time calibration of
the appendix): tau(B) = d0 + d1 * (tokens of the batch).

A ``Server`` runs serving iterations of a decoder of a given ``Shape``, with
random weights and a paged KV cache: the KV path is the operators of ``kv``
(rotary positions, quantised writes, attention over the pages), the dense
products are library matrix products.  ``measure`` times iterations of given
batches, ``fit`` takes d0 and d1 from them by least squares, and ``budget`` is
the number of cached tokens that fit a byte budget.

    python -m paper_2504_11320_amd.iteration --cache fp8

measures the 32-layer shape with 32 heads of 128, prints d0, d1 and C, and the
fluid boundary that they give the simulator's prompts of 512 with 20 decode
tokens.
"""
from __future__ import annotations

import argparse
import dataclasses
import json
import math
from typing import List, Sequence, Tuple

import numpy as np
import torch

from . import calibrate, kv

CACHES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp8": torch.float8_e4m3fn,
          "int8": torch.int8}


@dataclasses.dataclass
class Shape:
    """A decoder: heads of ``dim``, a gated feed-forward block of ``ffn``."""

    layers: int = 32
    heads: int = 32
    kv_heads: int = 32
    dim: int = 128
    ffn: int = 11008
    dtype: torch.dtype = torch.bfloat16
    cache: torch.dtype = torch.bfloat16

    @property
    def hidden(self) -> int:
        return self.heads * self.dim

    def token_bytes(self) -> int:
        """KV cache bytes of a token, all layers."""
        return self.layers * kv.Cache.token_bytes(self.kv_heads, self.dim, self.cache)


def budget(shape: Shape, nbytes: float) -> int:
    """The KV budget C: cached tokens that fit ``nbytes``."""
    return int(nbytes // shape.token_bytes())


class Batch:
    """One iteration's work, on the device: per request, ``new`` tokens behind
    ``old`` cached ones.  Requests own consecutive pages of the cache."""

    def __init__(self, new: Sequence[int], old: Sequence[int], page_size: int, device="cuda"):
        if len(new) != len(old) or not len(new) or min(new) < 0 or min(old) < 0 or not sum(new):
            raise ValueError("a batch needs new >= 0 and old >= 0 tokens for each request")
        total = [a + b for a, b in zip(new, old)]
        need = [-(-n // page_size) for n in total]
        self.pages_needed = sum(need)
        table = np.full((len(new), max(need)), -1, dtype=np.int32)
        slots, positions, at = [], [], 0
        for b, n in enumerate(need):
            table[b, :n] = np.arange(at, at + n)
            j = np.arange(old[b], total[b])
            positions.append(j)
            slots.append(at * page_size + j)
            at += n
        self.tokens = sum(total)
        to = dict(device=device)
        self.pages = torch.tensor(table, **to)
        self.slots = torch.tensor(np.concatenate(slots), dtype=torch.int64, **to)
        self.positions = torch.tensor(np.concatenate(positions), dtype=torch.int64, **to)
        self.starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, **to)
        self.kv_lens = torch.tensor(total, dtype=torch.int32, **to)
        self.max_q, self.max_kv = max(new), max(total)


class Server:
    """Weights and caches of a shape.  ``iterate`` takes the new tokens' hidden
    states through every layer, writing their keys and values."""

    def __init__(self, shape: Shape, tokens: int, page_size: int = 16, positions: int = 4096,
                 seed: int = 0, device="cuda"):
        s = self.shape = shape
        self.page_size = page_size
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(rows, cols):
            w = torch.empty(rows, cols, dtype=s.dtype, device=device)
            return w.normal_(0.0, 1.0 / math.sqrt(rows), generator=g)

        wide = (s.heads + 2 * s.kv_heads) * s.dim
        self.qkv = [weight(s.hidden, wide) for _ in range(s.layers)]
        self.o = [weight(s.hidden, s.hidden) for _ in range(s.layers)]
        self.up = [weight(s.hidden, 2 * s.ffn) for _ in range(s.layers)]
        self.down = [weight(s.ffn, s.hidden) for _ in range(s.layers)]
        pages = -(-tokens // page_size)
        self.caches = [kv.Cache.empty(pages, page_size, s.kv_heads, s.dim, s.cache, device)
                       for _ in range(s.layers)]
        self.table = kv.rotary_table(positions, s.dim, device=device)

    @staticmethod
    def _norm(x):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-5)).to(x.dtype)

    def iterate(self, x: torch.Tensor, batch: Batch) -> torch.Tensor:
        """[new tokens, hidden] in, the same behind the last layer."""
        s = self.shape
        if batch.pages_needed > self.caches[0].pages:
            raise ValueError("the batch holds more tokens than the cache")
        split = [s.heads * s.dim, s.kv_heads * s.dim, s.kv_heads * s.dim]
        for i in range(s.layers):
            q, k, v = (t.unflatten(1, (-1, s.dim))
                       for t in (self._norm(x) @ self.qkv[i]).split(split, dim=1))
            kv.append(self.caches[i], k, v, batch.slots, positions=batch.positions,
                      table=self.table)
            q = kv.rotary(q, batch.positions, self.table, out=q)
            a = kv.attention(q, self.caches[i], batch.pages, batch.starts, batch.kv_lens,
                             max_q_len=batch.max_q, max_kv_len=batch.max_kv)
            x = x + a.flatten(1) @ self.o[i]
            gate, up = (self._norm(x) @ self.up[i]).chunk(2, dim=1)
            x = x + (torch.nn.functional.silu(gate) * up) @ self.down[i]
        return x

    def time(self, batch: Batch, repeats: int = 5) -> float:
        """Milliseconds of an iteration of this batch: the median of ``repeats``
        replays of a captured graph, so that launches do not count."""
        n = int(batch.slots.numel())
        x = torch.randn(n, self.shape.hidden, device=batch.pages.device).to(self.shape.dtype)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.iterate(x, batch)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.iterate(x, batch)
        graph.replay()
        times = []
        for _ in range(repeats):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            graph.replay()
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return float(np.median(times))


def stage_batch(prompt_len: int, out_len: int, per_stage: int) -> Tuple[List[int], List[int]]:
    """(new, old) of a batch with ``per_stage`` requests at every stage: prefills
    of the prompt, and one token at each of the ``out_len`` decode stages.  Stage
    s holds prompt + s tokens, s of them the batch's charge beside the prompt."""
    new = [prompt_len] * per_stage
    old = [0] * per_stage
    for s in range(1, out_len + 1):
        new += [1] * per_stage
        old += [prompt_len + s - 1] * per_stage
    return new, old


def measure(server: Server, batches: Sequence[Tuple[Sequence[int], Sequence[int]]],
            repeats: int = 5) -> List[Tuple[int, float]]:
    """(tokens, milliseconds) of an iteration of each batch."""
    out = []
    for new, old in batches:
        b = Batch(new, old, server.page_size, server.caches[0].device)
        out.append((b.tokens, server.time(b, repeats)))
    return out


def fit(points: Sequence[Tuple[float, float]]) -> dict:
    """d0, d1 of tau = d0 + d1 tokens by least squares, the mean absolute
    percentage error and R^2."""
    if len(points) < 2:
        raise ValueError("a fit needs two batches or more")
    x, y = np.array(points, dtype=np.float64).T
    if np.ptp(x) == 0:
        raise ValueError("a fit needs batches of different sizes")
    d1, d0 = np.polyfit(x, y, 1)
    r = y - (d0 + d1 * x)
    return {"d0": float(d0), "d1": float(d1), "mape": float(np.mean(np.abs(r) / y)),
            "r2": float(1.0 - np.sum(r ** 2) / np.sum((y - y.mean()) ** 2))}


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--cache", choices=sorted(CACHES), default="bf16")
    ap.add_argument("--layers", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=32)
    ap.add_argument("--prompt", type=int, default=512)
    ap.add_argument("--out", type=int, default=20)
    ap.add_argument("--per-stage", type=int, nargs="+", default=[1, 2, 3, 4, 6])
    ap.add_argument("--kv-bytes", type=float, default=200e9, help="bytes of KV cache")
    a = ap.parse_args(argv)
    shape = Shape(layers=a.layers, kv_heads=a.kv_heads, cache=CACHES[a.cache])
    batches = [stage_batch(a.prompt, a.out, n) for n in a.per_stage]
    most = max(sum(n) + sum(o) for n, o in batches) + 16 * max(len(n) for n, _ in batches)
    points = measure(Server(shape, most, positions=a.prompt + a.out + 1), batches)
    got = fit(points)
    got["C"] = budget(shape, a.kv_bytes)
    work = calibrate.stage_work(a.prompt, a.out)
    got["boundary_per_s"] = 1000.0 * calibrate.fluid_boundary(work, got["d0"], got["d1"], got["C"])
    got["points"] = points
    got["cache"] = a.cache
    print(json.dumps(got), flush=True)
    return got


if __name__ == "__main__":
    main()
