"""Autograd across types: an input's gradient has its input's precision."""
import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2410_22697_amd import block_mean, block_mean_backward, linear, linear_backward

pytestmark = pytest.mark.gpu


def test_gradients_of_a_mean_in_another_type():
    """x in fp32 and the mean in bf16: x's gradient is an fp32 sum, as exact as with a gradient in fp32."""
    rng = np.random.default_rng(0)
    lengths = rng.integers(0, 9, 400)
    indptr = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    indices = rng.integers(0, 60, indptr[-1]).astype(np.int32)
    x = torch.randn(60, 24, device="cuda", requires_grad=True)
    dout = torch.randn(400, 24, device="cuda").bfloat16()
    i, j = torch.from_numpy(indptr).cuda(), torch.from_numpy(indices).cuda()
    block_mean(x, i, j, dtype=torch.bfloat16).backward(dout)
    want, mag, count = plain.mean_backward(dout.double().cpu().numpy(), indptr, indices, 60)
    assert x.grad.dtype == torch.float32
    assert np.all(np.abs(x.grad.double().cpu().numpy() - want) <= (2 * count[:, None] + 3) * plain.EPS * mag)
    # and the other way round: summed in fp32, rounded once to the input's bf16
    y = x.detach().bfloat16().requires_grad_()
    up = torch.randn(400, 24, device="cuda")
    block_mean(y, i, j, dtype=torch.float32).backward(up)
    assert y.grad.dtype == torch.bfloat16 and torch.equal(y.grad, block_mean_backward(up, i, j, 60).bfloat16())


def test_a_layer_in_bf16():
    """Autograd's gradients are linear_backward's, also in bf16."""
    for act in ("none", "relu", "gelu", "silu"):
        x, w, b, x2, r = (torch.randn(s, device="cuda").bfloat16().requires_grad_() for s in ((90, 24), (33, 34), (33,), (90, 10), (90, 33)))
        dy = torch.randn(90, 33, device="cuda").bfloat16()
        linear(x, w, b, act=act, residual=r, x2=x2).backward(dy)
        with torch.no_grad():
            _, pre = linear(x, w, b, act=act, x2=x2, save_pre=True)
            want = linear_backward(dy, x, w, act, None if act == "none" else pre, x2)
        for got, u in zip((x.grad, x2.grad, w.grad, b.grad, r.grad), (*want, dy)):
            assert torch.equal(got, u)
