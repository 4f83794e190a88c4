"""The KV budget of shapes whose requests go back to a number of tokens."""
import torch

from paper_2504_11320_amd import iteration as I


def test_a_token_takes_its_weights_too():
    """Such a shape holds 32 bits for each cached key beside its rows; the budget is
    what a server of that many tokens allocates."""
    for cache, row in ((torch.bfloat16, 2 * 64 * 2), (torch.int8, 2 * (64 + 4))):
        kw = dict(layers=3, heads=4, kv_heads=2, dim=64, ffn=32, cache=cache)
        assert I.Shape(**kw).token_bytes() == 3 * 2 * row
        shape = I.Shape(**kw, keep=8, recent=2)
        assert shape.token_bytes() == 3 * 2 * (row + 4)
        assert I.budget(shape, 160 * shape.token_bytes()) == 160
        server = I.Server(shape, tokens=160, positions=8, device="cpu")
        held = sum(t.nbytes for c in server.caches for t in c._tensors if t is not None)
        assert held + sum(w.nbytes for w in server.weights) == 160 * shape.token_bytes()
