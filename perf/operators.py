"""Performance cases of the operators on the KV path of one serving iteration.

The simulator's iteration takes d0 + d1 * (tokens in the batch) and holds
C tokens of KV cache.  On a card those three numbers come from the work that
touches the cache: queries and keys are turned by their positions (rotary), new
keys and values are written into pages, in 16 bits or quantised to 8 (append),
rows are taken out again when a request moves between servers (read), and every
batched token attends over its request's pages (attention).  The shapes are the
32 heads of 128 that 524,288 bytes a token over 32 layers stand for, shared
heads beside them, and the lengths of the simulated workloads.

A case is a dict of plain values; `run` makes one pass, in elementary torch
operations in 32 bits, or, where `own` is true, by the calls of the framework.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32,
          "fp8": torch.float8_e4m3fn, "int8": torch.int8}
_SIZE = {"bf16": 2, "fp16": 2, "fp32": 4, "fp8": 1, "int8": 1}
_TOP = {"fp8": 448.0, "int8": 127.0}   # largest value of a code
_TINY = 2.0 ** -100                    # rows below this are stored as zeros


# ------------------------------------------------------------------ cases ----


def _rotary(**kw):
    c = dict(op="rotary", tokens=1, heads=32, dim=128, part=128, interleaved=False,
             inverse=False, scaling="none", positions=4096, dtype="bf16")
    return {**c, **kw}


def _append(**kw):
    c = dict(op="append", tokens=1, kv_heads=32, dim=128, page=16, cache="fp8", dtype="bf16",
             rotate=True, interleaved=False, positions=4096, skip=0)
    return {**c, **kw}


def _read(**kw):
    c = dict(op="read", tokens=1, kv_heads=32, dim=128, page=16, cache="fp8", dtype="bf16")
    return {**c, **kw}


def _attention(**kw):
    c = dict(op="attention", decodes=0, kv_min=1, kv_max=1, prompts=0, prompt_min=1,
             prompt_max=1, context_min=0, context_max=0, heads=32, kv_heads=32, dim=128,
             page=16, cache="bf16", dtype="bf16", causal=True, window=0, lse=False, mix=1)
    return {**c, **kw}


def listed():
    return [
        # one decoded token's queries: the smallest call, latency counts
        dict(_rotary(), name="rotary-token"),
        # the queries of a batch of long prompts, positions stretched over a
        # context of the whole KV budget
        dict(_rotary(tokens=8192, scaling="yarn", positions=131072), name="rotary-prompts"),
        # a gradient's way back: the inverse rotation of part of each head in
        # 32 bits, neighbouring elements paired, odd sizes
        dict(_rotary(tokens=1531, heads=13, dim=96, part=48, interleaved=True, inverse=True,
                     dtype="fp32"), name="rotary-part-gradient"),
        # one decode iteration of 128 requests: each writes one token, and the
        # rows as the cache now holds them come back
        dict(_append(tokens=128), name="append-decode"),
        # a prefill iteration: prompts of the heavy-tailed mix, some rows of
        # padding, 8-bit integers, shared heads
        dict(_append(tokens=8191, kv_heads=8, cache="int8", dtype="fp16", page=64, skip=100),
             name="append-prefill"),
        # a prefilled context of 630 tokens leaves for the decode server
        dict(_read(tokens=630), name="read-context"),
        # a quarter of the KV budget is moved
        dict(_read(tokens=32768, dtype="fp32"), name="read-budget"),
        # one request alone in the middle of its output
        dict(_attention(decodes=1, kv_min=777, kv_max=777), name="attention-one"),
        # a full decode batch of prompts of 512 with up to 1000 tokens out,
        # about the KV budget of 131,072 tokens, in 8 bits
        dict(_attention(decodes=128, kv_min=513, kv_max=1512, cache="fp8"),
             name="attention-decode"),
        # one request with the whole budget as its context, heads shared by 8
        dict(_attention(decodes=1, kv_min=131072, kv_max=131072, heads=64, kv_heads=8,
                        cache="int8", dtype="fp16", page=64, lse=True), name="attention-long"),
        # one chunk of 512 prompt tokens beside running decodes
        dict(_attention(decodes=31, kv_min=130, kv_max=1500, prompts=1, prompt_min=512,
                        prompt_max=512, context_min=1024, context_max=1024, kv_heads=8,
                        cache="fp8", page=32), name="attention-chunk"),
        # two long prompts prefilled at once
        dict(_attention(prompts=2, prompt_min=6011, prompt_max=8192, mix=3),
             name="attention-prefill"),
    ]


def _log(rng, lo, hi):
    """A whole number of lo..hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rotary", "append", "read", "attention", "attention", "attention"))
    if op == "rotary":
        dim = rng.choice((64, 80, 96, 128, 192, 256))
        part = rng.choice((dim, dim // 2, dim // 4))
        heads = rng.choice((1, 5, 8, 13, 32, 64))
        return _rotary(tokens=_log(rng, 1, min(16384, (1 << 25) // (heads * dim))), heads=heads,
                       dim=dim, part=part, interleaved=rng.random() < 0.5,
                       inverse=rng.random() < 0.3, dtype=rng.choice(("bf16", "fp16", "fp32")),
                       scaling=rng.choice(("none", "linear", "ntk", "yarn")),
                       positions=rng.choice((4096, 32768, 131072)))
    if op in ("append", "read"):
        kv_heads, dim = rng.choice((1, 2, 4, 8, 32)), rng.choice((64, 128, 256))
        kw = dict(tokens=_log(rng, 1, min(32768, (1 << 25) // (kv_heads * dim))),
                  kv_heads=kv_heads, dim=dim, page=rng.choice((1, 16, 32, 64, 128)),
                  cache=rng.choice(("fp8", "int8", "bf16", "fp16")))
        if op == "read":
            return _read(dtype=rng.choice(("bf16", "fp16", "fp32")), **kw)
        kw["dtype"] = kw["cache"] if kw["cache"].endswith("16") else rng.choice(("bf16", "fp16",
                                                                                  "fp32"))
        return _append(rotate=rng.random() < 0.7, interleaved=rng.random() < 0.3,
                       skip=rng.choice((0, 0, 3)) if kw["tokens"] > 8 else 0,
                       positions=rng.choice((4096, 32768)), **kw)
    kv_heads, group = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 1, 2, 4, 7, 8, 16))
    if kv_heads == 32:
        group = rng.choice((1, 2))
    dim = rng.choice((64, 128, 128, 256))
    cache = rng.choice(("bf16", "fp16", "fp8", "int8"))
    kw = dict(heads=kv_heads * group, kv_heads=kv_heads, dim=dim, cache=cache,
              page=rng.choice((8, 16, 32, 64, 128)), lse=rng.random() < 0.5,
              dtype=cache if cache.endswith("16") else rng.choice(("bf16", "fp16")),
              window=rng.choice((0, 0, 0, 257)), mix=rng.randrange(1, 1000))
    width = kv_heads * dim                        # elements of a token's keys
    kind = rng.choice(("decode", "decode", "prefill", "mixed"))
    if kind == "decode":
        seqs = _log(rng, 1, 192)
        top = _log(rng, 1, max(1, min(131072, (1 << 28) // width // seqs)))
        return _attention(decodes=seqs, kv_min=max(1, top // rng.choice((1, 2, 4))), kv_max=top,
                          **kw)
    more = rng.choice((0, _log(rng, 1, 4096)))
    most = 5e10 / (dim * kw["heads"])             # pairs of a prompt
    top = _log(rng, 2, min(8192, int(math.sqrt(most + 0.25 * more * more) - 0.5 * more)))
    kw["causal"] = rng.random() < 0.85
    if kind == "prefill":
        return _attention(prompts=rng.choice((1, 2, 3)), prompt_min=max(1, top * 2 // 3),
                          prompt_max=top, context_min=more // 2, context_max=more, **kw)
    return _attention(decodes=rng.choice((1, 3, 8)), kv_min=1, kv_max=_log(rng, 1, 2048),
                      prompts=1, prompt_min=min(top, 1024), prompt_max=min(top, 1024),
                      context_min=more, context_max=more, **kw)


def _lengths(c):
    """(query lengths, key lengths) of an attention case's requests."""
    r = random.Random(1000003 * c["mix"] + c["kv_max"] + c["prompt_max"])
    ql = [r.randint(c["prompt_min"], c["prompt_max"]) for _ in range(c["prompts"])]
    kl = [n + r.randint(c["context_min"], c["context_max"]) for n in ql]
    ql += [1] * c["decodes"]
    kl += [r.randint(c["kv_min"], c["kv_max"]) for _ in range(c["decodes"])]
    order = list(range(len(ql)))
    r.shuffle(order)
    return [ql[i] for i in order], [kl[i] for i in order]


def work(case):
    c = case
    if c["op"] == "rotary":
        n = c["tokens"] * c["heads"] * c["dim"]
        return {"bytes": 2 * n * _SIZE[c["dtype"]] + c["tokens"] * (8 + 4 * c["part"]),
                "flops": 3 * c["tokens"] * c["heads"] * c["part"]}
    if c["op"] in ("append", "read"):
        n = 2 * c["tokens"] * c["kv_heads"] * c["dim"]
        row = _SIZE[c["cache"]] * n + (8 * c["tokens"] * c["kv_heads"] if c["cache"] in _TOP
                                       else 0)
        if c["op"] == "read":
            return {"bytes": row + _SIZE[c["dtype"]] * n + 8 * c["tokens"], "flops": n}
        turn = c["tokens"] * (8 + 4 * c["dim"]) if c["rotate"] else 0
        # the new rows in, the cache's rows out, and as values out
        return {"bytes": 2 * row + 2 * _SIZE[c["dtype"]] * n + 16 * c["tokens"] + turn,
                "flops": (5 if c["rotate"] else 3) * n}
    ql, kl = _lengths(c)
    pairs = keys = 0
    for n, m in zip(ql, kl):
        w = c["window"] or m
        if c["causal"]:
            ends = [m - n + i + 1 for i in range(n)]          # keys up to the token's own
            pairs += sum(min(w, max(0, e)) for e in ends)
            keys += m - max(0, ends[0] - w)
        else:
            pairs += sum(max(0, m - max(0, m - n + i + 1 - w)) for i in range(n))
            keys += m - max(0, m - n + 1 - w)
    row = c["kv_heads"] * (2 * c["dim"] * _SIZE[c["cache"]] + (8 if c["cache"] in _TOP else 0))
    rows = sum(ql) * c["heads"]
    return {"bytes": keys * row + rows * (2 * c["dim"] * _SIZE[c["dtype"]]
                                          + (4 if c["lse"] else 0)),
            "flops": 4 * c["dim"] * c["heads"] * pairs}


# ----------------------------------------------------------------- inputs ----


def _frequencies(part, scaling):
    """(radians a position for each pair, what the result is multiplied by):
    plain; positions divided by 8; the base raised so that the slowest pair
    turns 8 times slower; and pairs blended by how often they turn within the
    original 4,096 positions."""
    i = torch.arange(part // 2, dtype=torch.float64)
    base, factor, original = 10000.0, 8.0, 4096
    if scaling == "ntk" and part > 2:
        base *= factor ** (part / (part - 2.0))
    f = base ** (-2.0 * i / part)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "yarn":
        turns = original * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _table(positions, part, scaling, device):
    """[positions, part] in 32 bits: the cosines, then the sines."""
    f, by = _frequencies(part, scaling)
    a = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * f.to(device)
    return torch.cat([a.cos() * by, a.sin() * by], dim=1).float()


def _randn(shape, g, device):
    return torch.randn(shape, generator=g, device=device, dtype=torch.float32)


def _keys(shape, g, device):
    """Values of keys: some channels are larger than the rest, the same in
    every token."""
    by = torch.exp2(0.7 * _randn(shape[-1:], g, device))
    return _randn(shape, g, device) * by


def _quantise(x, kind):
    """(codes, a scale a row) of the last axis: the scale takes the row's
    largest magnitude to the largest code, codes are rounded to the nearest
    (half to even)."""
    top = x.abs().amax(-1)
    ok = top >= _TINY
    scale = torch.where(ok, top / _TOP[kind], torch.zeros_like(top))
    by = torch.where(ok, _TOP[kind] / torch.where(ok, top, torch.ones_like(top)),
                     torch.zeros_like(top))
    y = (x * by[..., None]).clamp(-_TOP[kind], _TOP[kind])
    return (y.round() if kind == "int8" else y).to(_TYPES[kind]), scale


def _empty_cache(pages, c, device):
    shape = (pages, c["kv_heads"], c["page"], c["dim"])
    t = _TYPES[c["cache"]]
    s = {"k": torch.zeros(shape, device=device, dtype=t),
         "v": torch.zeros(shape, device=device, dtype=t), "k_scale": None, "v_scale": None}
    if c["cache"] in _TOP:
        s["k_scale"] = torch.zeros(shape[:3], device=device, dtype=torch.float32)
        s["v_scale"] = torch.zeros(shape[:3], device=device, dtype=torch.float32)
    return s


def _full_cache(pages, c, g, device):
    s = _empty_cache(pages, c, device)
    step = max(1, (1 << 27) // (c["kv_heads"] * c["page"] * c["dim"]))
    for a in range(0, pages, step):
        for n in ("k", "v"):
            part = s[n][a:a + step]
            x = (_keys if n == "k" else _randn)(tuple(part.shape), g, device)
            if c["cache"] in _TOP:
                part.view(torch.uint8)[:] = 0
                code, scale = _quantise(x, c["cache"])
                part.copy_(code)
                s[n + "_scale"][a:a + step] = scale
            else:
                part.copy_(x)
    return s


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    s = {"case": c}
    if c["op"] == "rotary":
        s["table"] = _table(c["positions"], c["part"], c["scaling"], dev)
        s["pos"] = torch.randint(0, c["positions"], (c["tokens"],), generator=g, device=dev)
        s["x"] = _randn((c["tokens"], c["heads"], c["dim"]), g, dev).to(_TYPES[c["dtype"]])
        return s
    if c["op"] in ("append", "read"):
        T = c["tokens"]
        pages = -(-T // c["page"]) + 3
        at = torch.randperm(pages, generator=g, device=dev)
        i = torch.arange(T, device=dev)
        s["slots"] = at[i // c["page"]] * c["page"] + i % c["page"]
        if c["op"] == "read":
            s.update(_full_cache(pages, c, g, dev))
            return s
        s.update(_empty_cache(pages, c, dev))
        if c["skip"]:  # rows of padding, which have no slot
            s["slots"][torch.randperm(T, generator=g, device=dev)[:c["skip"]]] = -1
        shape = (T, c["kv_heads"], c["dim"])
        s["new_k"] = _keys(shape, g, dev).to(_TYPES[c["dtype"]])
        s["new_v"] = _randn(shape, g, dev).to(_TYPES[c["dtype"]])
        if c["rotate"]:
            s["table"] = _table(c["positions"], c["dim"], "none", dev)
            s["pos"] = torch.randint(0, c["positions"], (T,), generator=g, device=dev)
        return s
    ql, kl = _lengths(c)
    need = [-(-n // c["page"]) for n in kl]
    pages = sum(need) + 5
    at = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    table = torch.full((len(kl), max(need)), -1, dtype=torch.int32, device=dev)
    a = 0
    for b, n in enumerate(need):
        table[b, :n] = at[a:a + n]
        a += n
    s.update(_full_cache(pages, c, g, dev))
    starts = [0]
    for n in ql:
        starts.append(starts[-1] + n)
    s.update(pages=table, starts=torch.tensor(starts, dtype=torch.int32, device=dev),
             lens=torch.tensor(kl, dtype=torch.int32, device=dev), max_q=max(ql), max_kv=max(kl))
    s["q"] = (1.5 * _randn((starts[-1], c["heads"], c["dim"]), g, dev)).to(_TYPES[c["dtype"]])
    return s


# ------------------------------------------------------------ plain forms ----


def _turn(x, pos, table, interleaved, inverse):
    """The pairs of the first `part` elements turned, in 32 bits."""
    part = table.shape[1]
    half = part // 2
    row = table[pos][:, None, :]
    cos, sin = row[..., :half], row[..., half:]
    if inverse:
        sin = -sin
    y = x.float().clone()
    a, b = (y[..., 0:part:2], y[..., 1:part:2]) if interleaved else (y[..., :half],
                                                                     y[..., half:part])
    u, v = a * cos - b * sin, b * cos + a * sin
    a.copy_(u)
    b.copy_(v)
    return y


def _rows(s, name, slots):
    """The rows of `slots` as the values that they stand for; zeros where a
    slot is negative."""
    c = s["case"]
    at = slots.clamp(min=0)
    page, off = at // c["page"], at % c["page"]
    x = s[name][page, :, off].float()
    if c["cache"] in _TOP:
        x = x * s[name + "_scale"][page, :, off][..., None]
    return torch.where((slots >= 0)[:, None, None], x, torch.zeros_like(x))


def _write(s, name, x):
    """Rows x (32 bits) into their slots."""
    c = s["case"]
    to = s["slots"] >= 0
    at = s["slots"][to]
    page, off = at // c["page"], at % c["page"]
    if c["cache"] in _TOP:
        code, scale = _quantise(x, c["cache"])
        s[name].view(torch.uint8)[page, :, off] = code.view(torch.uint8)[to]
        s[name + "_scale"][page, :, off] = scale[to]
    else:
        s[name][page, :, off] = x.to(s[name].dtype)[to]


def _attend(s):
    """Softmax of the scaled products over the keys that a token sees, times
    the values; requests are padded to the longest."""
    c, q = s["case"], s["q"]
    T, H, D = q.shape
    B, KH = s["lens"].numel(), c["kv_heads"]
    G = H // KH
    dev = q.device
    starts, lens = s["starts"].long(), s["lens"].long()
    n = starts[1:] - starts[:-1]
    i = torch.arange(s["max_q"], device=dev)
    at = (starts[:-1, None] + i).clamp(max=T - 1)
    x = q.float()[at].view(B, -1, KH, G, D).permute(0, 2, 3, 1, 4).reshape(B, KH, -1, D)
    table = s["pages"].long().clamp(min=0)

    def side(name):
        y = s[name][table].float()
        if c["cache"] in _TOP:
            y = y * s[name + "_scale"][table][..., None]
        return y.permute(0, 2, 1, 3, 4).reshape(B, KH, -1, D)

    z = torch.matmul(x, side("k").transpose(-1, -2)) * (1.0 / math.sqrt(D))
    key = torch.arange(z.shape[-1], device=dev)
    own_at = lens[:, None] - n[:, None] + i               # the token's own position
    see = (key < lens[:, None, None]).expand(B, i.numel(), -1)
    if c["causal"]:
        see = see & (key <= own_at[..., None])
    if c["window"]:
        see = see & (key > own_at[..., None] - c["window"])
    z = z.view(B, KH, G, i.numel(), -1).masked_fill_(~see[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    base = torch.where(top > -math.inf, top, torch.zeros_like(top))
    p = z.sub_(base).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, KH, -1, p.shape[-1]), side("v")).view(B, KH, G, -1, D)
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    lse = (base + total.log())[..., 0]
    row = torch.arange(T, device=dev)
    b = torch.searchsorted(starts[1:].contiguous(), row, right=True)
    j = row - starts[b]
    out = {"out": o[b, :, :, j].reshape(T, H, D).to(q.dtype)}
    if c["lse"]:
        out["lse"] = lse[b, :, :, j].reshape(T, H)
    return out


def _run_plain(s):
    c = s["case"]
    t = _TYPES[c["dtype"]]
    if c["op"] == "rotary":
        return _turn(s["x"], s["pos"], s["table"], c["interleaved"], c["inverse"]).to(t)
    if c["op"] == "read":
        return {n: _rows(s, n, s["slots"]).to(t) for n in ("k", "v")}
    if c["op"] == "append":
        k = s["new_k"].float()
        if c["rotate"]:
            k = _turn(k, s["pos"], s["table"], c["interleaved"], False)
        _write(s, "k", k)
        _write(s, "v", s["new_v"].float())
        out = {n: _rows(s, n, s["slots"]).to(t) for n in ("k", "v")}
        if c["cache"] in _TOP:
            out.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
        return out
    return _attend(s)


def _run_own(s):
    from paper_2504_11320_amd import kv

    c = s["case"]
    t = _TYPES[c["dtype"]]
    if c["op"] == "rotary":
        return kv.rotary(s["x"], s["pos"], s["table"], interleaved=c["interleaved"],
                         inverse=c["inverse"])
    cache = kv.Cache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    if c["op"] == "read":
        k, v = kv.read(cache, s["slots"], dtype=t)
        return {"k": k, "v": v}
    if c["op"] == "append":
        turn = dict(positions=s["pos"], table=s["table"],
                    interleaved=c["interleaved"]) if c["rotate"] else {}
        kv.append(cache, s["new_k"], s["new_v"], s["slots"], **turn)
        k, v = kv.read(cache, s["slots"], dtype=t)
        out = {"k": k, "v": v}
        if c["cache"] in _TOP:
            out.update(k_scale=s["k_scale"], v_scale=s["v_scale"])
        return out
    got = kv.attention(s["q"], cache, s["pages"], s["starts"], s["lens"], max_q_len=s["max_q"],
                       max_kv_len=s["max_kv"], causal=c["causal"], window=c["window"],
                       return_lse=c["lse"])
    return {"out": got[0], "lse": got[1]} if c["lse"] else {"out": got}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------- definition, 64 bits ----


def _exact_turn(x, pos, part, scaling, interleaved, inverse):
    f, by = _frequencies(part, scaling)
    a = pos.double()[:, None] * f.to(x.device) * (-1.0 if inverse else 1.0)
    z = torch.polar(torch.full_like(a, by), a)[:, None, :]
    y = x.double().clone()
    if interleaved:
        pair = torch.view_as_complex(y[..., :part].reshape(*y.shape[:2], -1, 2).contiguous()) * z
        y[..., :part] = torch.view_as_real(pair).reshape(*y.shape[:2], part)
    else:
        pair = torch.complex(y[..., :part // 2], y[..., part // 2:part]) * z
        y[..., :part // 2], y[..., part // 2:part] = pair.real, pair.imag
    return y


def _exact_codes(x, kind):
    """(values as stored, scales) of rows in 64 bits."""
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.where(top >= _TINY, top / _TOP[kind], torch.zeros_like(top))
    y = torch.where(scale > 0, x / scale, torch.zeros_like(x))
    if kind == "fp8":  # 3 bits behind the leading one, the smallest exponent -6
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        y = torch.round(y / step) * step
    else:
        y = torch.round(y)
    return y * scale, scale[..., 0]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "rotary":
        return _exact_turn(s["x"], s["pos"], c["part"], c["scaling"], c["interleaved"],
                           c["inverse"])
    if c["op"] == "read":
        return {n: _exact_rows(s, n, s["slots"]) for n in ("k", "v")}
    if c["op"] == "append":
        k, v = s["new_k"].double(), s["new_v"].double()
        if c["rotate"]:
            k = _exact_turn(k, s["pos"], c["dim"], "none", c["interleaved"], False)
        out, to = {}, s["slots"] >= 0
        at = s["slots"][to]
        for n, x in (("k", k), ("v", v)):
            if c["cache"] in _TOP:
                x, scale = _exact_codes(x, c["cache"])
                held = torch.zeros(s[n + "_scale"].shape, dtype=torch.float64, device=x.device)
                held[at // c["page"], :, at % c["page"]] = scale[to]
                out[n + "_scale"] = held
            x[~to] = 0.0
            out[n] = x
        return out
    return _exact_attention(s)


def _exact_rows(s, name, slots):
    c = s["case"]
    page, off = slots // c["page"], slots % c["page"]
    x = s[name][page, :, off].double()
    if c["cache"] in _TOP:
        x = x * s[name + "_scale"][page, :, off].double()[..., None]
    return x


def _exact_attention(s):
    """Request by request and head by head, over the rows that are there."""
    c, q = s["case"], s["q"]
    T, H, D = q.shape
    G = H // c["kv_heads"]
    ql, kl = _lengths(c)
    out = torch.zeros(T, H, D, dtype=torch.float64, device=q.device)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=q.device)
    a = 0
    for b, (n, m) in enumerate(zip(ql, kl)):
        i = torch.arange(m, device=q.device)
        slots = s["pages"][b].long()[i // c["page"]] * c["page"] + i % c["page"]
        k, v = _exact_rows(s, "k", slots), _exact_rows(s, "v", slots)
        own_at = m - n + torch.arange(n, device=q.device)[:, None]
        see = torch.ones(n, m, dtype=torch.bool, device=q.device)
        if c["causal"]:
            see &= i <= own_at
        if c["window"]:
            see &= i > own_at - c["window"]
        some = see.any(-1)
        for h in range(H):
            z = (q[a:a + n, h].double() @ k[:, h // G].T) / math.sqrt(D)
            z = z.masked_fill(~see, -math.inf)
            t = torch.logsumexp(z, -1)
            p = torch.where(some[:, None], (z - t[:, None]).exp(), torch.zeros_like(z))
            out[a:a + n, h] = p @ v[:, h // G]
            lse[a:a + n, h] = t
        a += n
    got = {"out": out}
    if c["lse"]:
        got["lse"] = lse
    return got
