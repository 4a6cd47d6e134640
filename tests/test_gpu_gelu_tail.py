"""gelu and its slope where they are small, and over normal values, against 64 bits."""
import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2410_22697_amd import linear, linear_backward

pytestmark = pytest.mark.gpu


def through(z, dtype):
    """gelu(z) and its slope, by a layer of one weight of 1."""
    x = torch.from_numpy(z.astype(np.float32)).to(dtype).cuda()[:, None]
    one = torch.ones(1, 1, device="cuda", dtype=dtype)
    y = linear(x, one, act="gelu")
    slope = linear_backward(torch.ones_like(x), x, one, "gelu", x, bias=False, need_dw=False)[0]
    return [t[:, 0].double().cpu().numpy() for t in (x, y, slope)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [3001, 70_001])  # the form for few rows, and streamed rows
def test_the_negative_tail(dtype, n):
    """Relative: the exponential's argument, up to 26 in powers of two, is rounded twice (2.2e-6), the other factors' few
    roundings make it 1e-5 at most; 1e-12 of Phi and of the slope for the approximation."""
    z, y, slope = through(np.linspace(-6, -3, n), dtype)
    phi = plain.act(z, "gelu") / z
    half = plain.BF / 2 if dtype == torch.bfloat16 else 0.0
    for got, want, scale in ((y, plain.act(z, "gelu"), np.abs(z)), (slope, plain.slope(z, "gelu"), 1.0)):
        assert np.all(np.abs(got - want) <= (1e-5 + half) * np.abs(want) + 1e-12 * scale)
    assert np.all(phi > 9e-10)


def test_normal_values_in_fp32():
    """The root of the mean squared error: 2.45e-8 and 2.6e-8 for the formulas in fp32 operations rounded one by one; the
    bounds leave the hardware's exponential and reciprocal their unit in the last place."""
    z, y, slope = through(np.random.default_rng(0).standard_normal(300_000), torch.float32)
    rms = lambda e: np.sqrt(np.mean(e * e))  # noqa: E731
    assert rms(y - plain.act(z, "gelu")) <= 3.2e-8
    assert rms(slope - plain.slope(z, "gelu")) <= 4.8e-8
    assert np.abs(y - plain.act(z, "gelu")).max() <= 4e-7 and np.abs(slope - plain.slope(z, "gelu")).max() <= 3e-7


def test_the_ends():
    z = np.array([np.inf, 200.0, 38.0, 0.0, -0.0, -38.0, -200.0, np.nan, -1e-30, 1e-30, -1e-42, 1e-42])
    _, y, slope = through(z, torch.float32)
    assert y[0] == np.inf and y[1] == 200 and y[2] == 38 and y[3] == 0 and y[4] == 0 and abs(y[5]) < 1e-300 and y[6] == 0
    assert np.isnan(y[7]) and np.isnan(slope[7])
    assert np.allclose(y[8:10], [-5e-31, 5e-31], rtol=1e-6) and np.all(np.abs(y[10:]) <= 1e-42)
    assert np.allclose(slope[[0, 1, 2, 3, 4, 5, 6]], [1, 1, 1, 0.5, 0.5, 0, 0], atol=1e-7)
