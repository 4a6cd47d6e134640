"""A layer's gradients as documented: in bf16, dz is rounded to bf16 before the products with the weights and the inputs,
and to nothing less."""
import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2410_22697_amd import linear_backward

pytestmark = pytest.mark.gpu


def wide(t):
    return t.detach().double().cpu().numpy()


def to_bf16(a):
    return wide(torch.from_numpy(a).to(torch.bfloat16))


def make(rows, k, n, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    return new(rows, n), (2 * new(rows, n).float()).to(dtype), new(rows, k), new(n, k)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("size", [(70, 40, 33), (9_001, 130, 70)])  # the form for few rows, and streamed rows
def test_bf16_products_take_dz_in_bf16(act, size):
    """Against 64-bit products of dz rounded to bf16: a sum of K terms rounds K times at most, a result once. dz itself may
    round to either side where the slope's own error (4e-7 (1 + |pre|), and an operation's rounding) spans the middle
    between two bf16 values."""
    rows, k, n = size
    dy, pre, x, w = make(rows, k, n, torch.bfloat16, rows)
    dz = wide(dy) * plain.slope(wide(pre), act)
    off = (act != "relu") * (np.abs(wide(dy)) * 4e-7 * (1 + np.abs(wide(pre))) + 4 * plain.EPS * np.abs(dz))
    low, held, high = to_bf16(dz - off), to_bf16(dz), to_bf16(dz + off)
    either = np.maximum(np.abs(high - held), np.abs(held - low))
    dx, _, dw, _ = linear_backward(dy, x, w, act, pre)
    for got, want, slack in ((dx, held @ wide(w), either @ np.abs(wide(w)) + (n + 2) * plain.EPS * (np.abs(held) @ np.abs(wide(w)))),
                             (dw, held.T @ wide(x), either.T @ np.abs(wide(x)) + (rows + 2) * plain.EPS * (np.abs(held).T @ np.abs(wide(x))))):
        assert np.all(np.abs(wide(got) - want) <= slack + plain.BF / 2 * (np.abs(want) + slack))
