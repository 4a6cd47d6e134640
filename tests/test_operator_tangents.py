"""Forward-mode tangents are refused before anything else (no GPU needed)."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2410_22697_amd import operators


def test_tangents_are_refused():
    x, w = torch.randn(6, 16), torch.randn(5, 16)
    ids = torch.zeros(3, dtype=torch.int32)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        for bad in (lambda: operators.linear(dual, w), lambda: operators.linear(x, w, x2=dual), lambda: operators.block_mean(dual, ids, ids),
                    lambda: operators.linear_backward(dual, x, w), lambda: operators.block_mean_backward(x, ids, ids, 3, add=dual)):
            with pytest.raises(ValueError, match="tangent"):
                bad()
        for fine in (lambda: operators.linear(x, w), lambda: operators.block_mean(x, ids, ids)):
            with pytest.raises(ValueError, match="device"):  # refused for where it lies, as outside
                fine()
