"""What the KV-path operators' Python calls refuse: gradients, memory that
overlaps, replaced tensors of a cache.  No GPU: the checks come first."""
import pytest
import torch

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


