"""Tensors that share memory are found (no GPU needed)."""
import pytest
import torch

from paper_2410_22697_amd import operators


def test_tensors_that_share_memory_are_found():
    a = torch.zeros(40)
    for bad in ([a, a], [a[:20], a[19:]], [a[10:11], a[:30]], [a[5:], a[:5], a[39:]]):
        with pytest.raises(ValueError, match="share"):
            operators._disjoint(bad)
    operators._disjoint([a[:20], a[20:], None, a[:0], a[3:3], torch.zeros(40)])
    operators._disjoint([])
