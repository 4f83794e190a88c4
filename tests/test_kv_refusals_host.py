"""What the KV-path operators' Python calls refuse: gradients, memory that
overlaps, replaced tensors of a cache.  No GPU: the checks come first."""
import copy
import ctypes as C
import os
import pickle

import pytest
import torch

from paper_2504_11320_amd import binding as B
from paper_2504_11320_amd import build as Bd
from paper_2504_11320_amd import kv


def small(dtype=torch.bfloat16):
    return kv.Cache.empty(4, 16, 2, 64, dtype, device="cpu")


def tensors():
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    return dict(q=q, k=torch.zeros(3, 2, 64), v=torch.zeros(3, 2, 64),
                slots=torch.arange(3), pos=torch.arange(3), table=torch.zeros(10, 64),
                pages=torch.zeros(1, 2, dtype=torch.int32),
                starts=torch.tensor([0, 3], dtype=torch.int32),
                lens=torch.tensor([9], dtype=torch.int32))


CALLS = [("q", lambda t: kv.rotary(t["q"], t["pos"], t["table"])),
         ("table", lambda t: kv.rotary(t["q"], t["pos"], t["table"])),
         ("k", lambda t: kv.append(small(), t["k"], t["v"], t["slots"])),
         ("v", lambda t: kv.append(small(), t["k"], t["v"], t["slots"])),
         ("table", lambda t: kv.append(small(), t["k"], t["v"], t["slots"], positions=t["pos"],
                                       table=t["table"])),
         ("k", lambda t: kv.read(small(), t["slots"], out=(t["k"], t["v"]))),
         ("v", lambda t: kv.read(small(), t["slots"], out=(t["k"], t["v"]))),
         ("q", lambda t: kv.attention(t["q"], small(), t["pages"], t["starts"], t["lens"]))]


@pytest.mark.parametrize("which", range(len(CALLS)))
def test_gradients_are_refused(which):
    """No result without its gradient; under no_grad the call goes on to the
    next check, that the tensors are on the GPU."""
    name, call = CALLS[which]
    t = tensors()
    with pytest.raises(ValueError, match="on the GPU"):
        call(t)
    t[name].requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        call(t)
    with torch.no_grad(), pytest.raises(ValueError, match="on the GPU"):
        call(t)
    t[name] = t[name] * 1.0
    with pytest.raises(ValueError, match="gradient"):
        call(t)


def test_a_cache_of_parameters_is_refused():
    k, v = (torch.zeros(4, 2, 16, 64, dtype=torch.float16) for _ in range(2))
    kv.Cache(k, v)
    with torch.no_grad(), pytest.raises(ValueError, match="gradient"):
        kv.Cache(k, v.requires_grad_())
    c, s = torch.zeros(4, 2, 16, 64, dtype=torch.int8), torch.zeros(4, 2, 16)
    with pytest.raises(ValueError, match="gradient"):
        kv.Cache(c, c.clone(), s, s.clone().requires_grad_())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.int8])
def test_a_caches_tensors_stay(dtype):
    """The addresses of a cache's memory are kept beside its tensors, so these
    cannot be exchanged or taken away; operations in place can be written as
    assignments."""
    c = small(dtype)
    before = c.k, c.v, c.k_scale, c.v_scale
    for name in ("k", "v", "k_scale", "v_scale"):
        t = getattr(c, name)
        for other in (None if t is not None else torch.zeros(4, 2, 16), torch.zeros(4, 2, 16, 64),
                      None if t is None else t.clone()):
            if other is t:
                continue
            with pytest.raises(AttributeError):
                setattr(c, name, other)
        with pytest.raises(AttributeError):
            delattr(c, name)
    for name in ("pages", "kv_heads", "page_size", "dim", "dtype", "device"):
        with pytest.raises(AttributeError):
            setattr(c, name, 1)
    if dtype == torch.int8:
        c.v_scale += 1.0
        assert bool((c.v_scale == 1.0).all())
    assert all(a is b for a, b in zip(before, (c.k, c.v, c.k_scale, c.v_scale)))
    assert (c.pages, c.kv_heads, c.page_size, c.dim, c.dtype) == (4, 2, 16, 64, dtype)
    assert c.device == c.k.device
    # a copy has the addresses of its own tensors
    for other in (copy.copy(c), copy.deepcopy(c), pickle.loads(pickle.dumps(c))):
        assert other._c == kv.Cache(other.k, other.v, other.k_scale, other.v_scale)._c
        assert other.k.dtype == dtype and other.kv_heads == 2
    assert copy.copy(c).k is c.k and copy.deepcopy(c).k.data_ptr() != c.k.data_ptr()


FAKE = 1 << 40   # never dereferenced: the checks come first


def rows(data, token, head=64, type=kv.BF16):
    return kv.ROWS.pack(data, token, head, type)


# (x's address, token and head stride), (out's): 5 tokens of 2 heads of 64
OVERLAPS = [((0, 128, 64), (2, 128, 64)),            # one element on
            ((0, 128, 64), (256, 128, 64)),          # one token on
            ((256, 128, 64), (0, 128, 64)),
            ((0, 128, 64), (128, 128, 64)),          # one head on
            ((0, 384, 64), (128, 384, 64)),          # the same within wider rows
            ((0, 384, 64), (254, 384, 64)),          # one element of the second head
            ((0, 384, 64), (768 * 4, 384, 64)),      # the last token alone
            ((0, 64, 320), (128, 64, 320)),          # heads outside
            ((0, 384, 64), (0, 384, 128)),           # other heads' stride
            ((0, 384, 64), (-768 * 2, 384, 128)),
            ((0, 128, 64), (0, 64, 320)),            # one base, transposed
            ((0, 128, 64), (64, 256, 64)),
            ((1024, -128, 64), (0, 128, 64))]        # backwards


@pytest.mark.parametrize("x,out", OVERLAPS)
def test_overlapping_memory_is_refused(x, out):
    """An output that shares memory with the input, unless it is the input
    itself, or with the other output."""
    L = kv._lib()
    a, b = (rows(FAKE + at, token, head) for at, token, head in (x, out))
    turn = kv.TURN.pack(FAKE, FAKE, 0, 10, 32, 0)
    cache = kv.CACHE.pack(FAKE, FAKE, 0, 0, 4, 16, 2, 64, kv.BF16)
    batch = kv.BATCH.pack(FAKE, 8, 8, FAKE, FAKE, 1, 5, 2, 1.0, 1, 0, 5, 100)
    big = 1 << 30
    for p, q in ((a, b), (b, a)):
        assert L.wait_kv_rotary(p, q, 5, 2, 64, turn, 0, None) == B.WS_EINVAL
        assert b"overlap" in L.wait_sim_last_error() or b"in place" in L.wait_sim_last_error()
        assert L.wait_kv_read(cache, FAKE, 5, p, q, None) == B.WS_EINVAL
        assert b"overlap" in L.wait_sim_last_error()
        assert L.wait_kv_attention(cache, batch, p, q, None, FAKE, big, None) == B.WS_EINVAL
        assert b"overlap" in L.wait_sim_last_error()
    same = rows(FAKE, 128)
    assert L.wait_kv_read(cache, FAKE, 5, same, same, None) == B.WS_EINVAL


def test_nothing_is_promised_of_one_slot_twice():
    """Codes and scale of a row are separate stores of several lanes: the
    documents must not promise one of the rows."""
    src = open(os.path.join(Bd.INC, "wait_kv.h")).read()
    text = " ".join(src.replace("*", " ").split())
    assert "leave either" not in text
    assert "Slots within the cache must differ" in text
    assert "slots must differ" in " ".join(kv.append.__doc__.split())


def test_workspace_of_loose_bounds():
    """Rows that a batch cannot have take no room in the workspace: 128 single
    tokens of 32 heads over a table of 131,072 keys, where each may have 32 parts."""
    cache = kv.CACHE.pack(FAKE, FAKE, FAKE, FAKE, 8192, 16, 32, 128, kv.INT8)

    def size(max_q, heads=32, tokens=128, cols=8192):
        batch = kv.BATCH.pack(FAKE, cols, cols, FAKE, FAKE, 128, tokens, heads, 1.0, 1, 0, max_q,
                              cols * 16)
        n = C.c_size_t()
        assert kv._lib().wait_kv_attention_workspace_bytes(cache, batch, n) == B.WS_OK
        return n.value

    one = 32 * (128 + 2) * 4           # the parts of a row
    assert size(1) == 128 * 32 * one < 100e6
    assert size(1, cols=2048) == 128 * 32 * 8 * (128 + 2) * 4
    assert size(1, heads=64) == 128 * 64 * one
    assert size(5, heads=64, tokens=640) == 128 * 32 * 10 * one


def test_more_threads_than_a_launch_has():
    """Batches whose workgroups have 2^32 threads or more are refused as such,
    before anything is launched."""
    cache = kv.CACHE.pack(FAKE, FAKE, 0, 0, 4, 16, 1, 64, kv.BF16)
    for n_seq, tokens, max_q in ((1 << 24, 1 << 24, 1), (1 << 30, 1 << 30, 1),
                                 (1 << 23, 1 << 20, 100)):
        batch = kv.BATCH.pack(FAKE, 4, 4, FAKE, FAKE, n_seq, tokens, 1, 1.0, 1, 0, max_q, 64)
        r = rows(FAKE, 64)
        assert kv._lib().wait_kv_attention(cache, batch, r, r, None, None, 0, None) \
            == B.WS_EUNSUPPORTED
        assert b"workgroups" in kv._lib().wait_sim_last_error()


def test_workspace_without_bounds():
    """Where the lengths of the queries are not given, the parts of a batch's rows
    take no more room than the rows that there are."""
    cache = kv.CACHE.pack(FAKE, FAKE, FAKE, FAKE, 8192, 16, 32, 128, kv.INT8)
    one = 32 * (128 + 2) * 4           # the parts of a row
    for tokens, heads in ((128, 32), (128, 64), (140, 32)):
        batch = kv.BATCH.pack(FAKE, 8192, 8192, FAKE, FAKE, 128, tokens, heads, 1.0, 1, 0, tokens,
                              8192 * 16)
        n = C.c_size_t()
        assert kv._lib().wait_kv_attention_workspace_bytes(cache, batch, n) == B.WS_OK
        # beside the parts of many rows, of which there are 256 at most
        assert n.value <= tokens * heads * (one + 256 * (128 + 2) * 4)
        batch = kv.BATCH.pack(FAKE, 8192, 8192, FAKE, FAKE, 128, tokens, heads, 1.0, 1, 0, 2,
                              8192 * 16)
        assert kv._lib().wait_kv_attention_workspace_bytes(cache, batch, n) == B.WS_OK
        assert n.value == tokens * heads * one
