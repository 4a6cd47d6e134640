"""AdamW with an eps of 0, and with one beneath what fp32 holds."""
import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2410_22697_amd import AdamW

pytestmark = pytest.mark.gpu
LR, B2 = 1e-3, 0.999


def cpu(t):
    return t.detach().float().cpu().numpy().astype(np.float64).reshape(-1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("size", [1.0, 1e-10, 1e-17, 1e-18, 3e-19, 1e-19])
def test_eps_of_zero(bits, size):
    """A first step is -lr sign(g) whatever g's size, as long as v can be held: v of 1e-41 (g of 1e-19) is a denormal of
    relative steps of 2^-13, whose root's are half of that; the moments', root's and quotient's own roundings are few."""
    p = torch.zeros(600, device="cuda")
    g = torch.randn(600, device="cuda")
    g = torch.where(g.abs() < 0.5, torch.sign(g), g) * size
    AdamW([p], lr=LR, eps=0.0, weight_decay=0.0, state_bits=bits).step([g])
    v = (1 - B2) * cpu(g) ** 2
    grain = 2.0 ** -149 * 2 / v  # g^2 and its product with 1 - b2 are rounded to denormals' steps
    want = -LR * np.sign(cpu(g))
    assert np.all(np.abs(cpu(p) - want) <= LR * (grain + 16 * plain.EPS))


def test_a_positive_eps_beneath_the_normal_range():
    """It counts as the least normal value: without gradient nothing moves, rather than 0 / 0."""
    for eps in (1e-40, 1e-60):
        p = torch.ones(300, device="cuda")
        AdamW([p], lr=LR, eps=eps, weight_decay=0.0).step([torch.zeros(300, device="cuda")])
        assert torch.all(p == 1)
