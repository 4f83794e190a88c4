"""Batches, budgets and fits of the iteration measurement, without a GPU."""
import numpy as np
import pytest
import torch

from paper_2504_11320_amd import calibrate
from paper_2504_11320_amd import iteration as I


def test_budget():
    """524,288 bytes a token in 16 bits; 8 bits with their scales hold
    256 / 132 of that."""
    s = I.Shape()
    assert s.token_bytes() == 524288 and s.hidden == 4096
    assert I.budget(s, 1.37e5 * 524288) == 137000
    q = I.Shape(cache=torch.int8)
    assert q.token_bytes() == 32 * 2 * 32 * 132
    assert I.budget(q, 524288.0) == 1


def test_stage_batch_charges_the_simulated_tokens():
    """A batch with n requests at every stage holds n * S tokens, S the tokens a
    request holds summed over its stages."""
    for l, L, n in ((512, 20, 1), (256, 3, 4), (1, 1, 2)):
        new, old = I.stage_batch(l, L, n)
        assert sum(new) + sum(old) == n * calibrate.stage_work(l, L)
        assert len(new) == n * (L + 1)
        b = I.Batch(new, old, 16, device="cpu")
        assert b.tokens == n * calibrate.stage_work(l, L)


def test_batch_layout():
    b = I.Batch([3, 1, 0], [0, 16, 5], 16, device="cpu")
    assert b.pages_needed == 1 + 2 + 1
    assert b.pages.tolist() == [[0, -1], [1, 2], [3, -1]]
    assert b.slots.tolist() == [0, 1, 2, 32] and b.positions.tolist() == [0, 1, 2, 16]
    assert b.starts.tolist() == [0, 3, 4, 4] and b.kv_lens.tolist() == [3, 17, 5]
    assert (b.max_q, b.max_kv) == (3, 17)
    for bad in (([], []), ([1], [0, 1]), ([-1], [2]), ([0], [4])):
        with pytest.raises(ValueError):
            I.Batch(*bad, 16, device="cpu")


def test_fit():
    x = np.array([100.0, 500.0, 2000.0, 9000.0])
    f = I.fit(list(zip(x, 2.5 + 0.004 * x)))
    assert abs(f["d0"] - 2.5) < 1e-9 and abs(f["d1"] - 0.004) < 1e-12
    assert f["mape"] < 1e-9 and abs(f["r2"] - 1.0) < 1e-12
    g = I.fit([(0.0, 1.0), (1.0, 3.0), (2.0, 2.0)])
    assert abs(g["d0"] - 1.5) < 1e-12 and abs(g["d1"] - 0.5) < 1e-12
    assert abs(g["r2"] - 0.25) < 1e-12
    assert abs(g["mape"] - np.mean([0.5, 1.0 / 3.0, 0.25])) < 1e-12
    for bad in ([(1.0, 2.0)], [(1.0, 2.0), (1.0, 3.0)]):
        with pytest.raises(ValueError):
            I.fit(bad)
