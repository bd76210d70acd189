"""Attention over the 8-bit cache refuses operands whose gradient it would lose.
No GPU."""
import pytest
import torch

from paper_2605_07243_amd import kvcache


def plan():
    p = kvcache.Attention.__new__(kvcache.Attention)
    p._layers = 1
    p._fits = lambda t: False       # (the check that comes next)
    p.cache = type("Cache", (), {"shape": type("Shape", (), {"elem": torch.bfloat16})})
    p._rows_shape, p.device = torch.Size((2, 8, 64)), torch.device("cpu")
    return p


def test_operands_that_require_a_gradient():
    q = torch.zeros(2, 8, 64, dtype=torch.bfloat16)
    g = q.clone().requires_grad_()
    for args in ((g,), (g * 2,), (q, g), (g, q)):
        with pytest.raises(ValueError, match="no backward"):
            plan()(0, *args)
    for args in ((q,), (g.detach(),), (q, g.detach())):
        with pytest.raises(ValueError, match="contiguous"):
            plan()(0, *args)
    with torch.no_grad(), pytest.raises(ValueError, match="contiguous"):
        plan()(0, g)
    with torch.inference_mode(), pytest.raises(ValueError, match="contiguous"):
        plan()(0, q)
