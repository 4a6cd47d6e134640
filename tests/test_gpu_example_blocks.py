"""The training example with residual blocks: a minibatch's loss and every gradient against plain torch in 64 bits on the same
sampled block and under the same masks."""
import os
import sys

import pytest
import torch

import plain_layers
from test_gpu_train_example import plain_mean

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("blocks,drop,width", [(1, 0.0, 96), (2, 0.3, 96), (1, 0.5, 33)])
def test_a_minibatch_against_plain_torch(blocks, drop, width):
    from train_sage import Setup, unpack_rows
    s = Setup(8, width=width, blocks=blocks, drop=drop)
    t = 3
    seeds, packed, (inner, outer) = s.sample(t)
    labels = s.labels[seeds.long()]
    loss = torch.nn.functional.cross_entropy(s.logits(packed, (inner, outer), t), labels)
    loss.backward()
    x = unpack_rows(packed, s.fmt).double()
    wide = [p.detach().double().requires_grad_() for p in s.params]
    w1, b1, w2, b2 = wide[:4]
    n0, n1 = inner[0].numel() - 1, outer[0].numel() - 1
    hidden = torch.relu(torch.cat([x[:n1], plain_mean(x, *outer)], 1) @ w1.t() + b1)
    for i in range(blocks):
        scale, both, back = wide[4 + 3 * i:7 + 3 * i]
        z = (hidden * torch.rsqrt(hidden.square().mean(1, keepdim=True) + 1e-6) * scale) @ both.t()
        n = both.shape[0] // 2
        y = (torch.nn.functional.silu(z[:, :n]) * z[:, n:]) @ back.t()
        keep = torch.from_numpy(plain_layers.kept(*y.shape, drop, t, i)).cuda()
        hidden = hidden + torch.where(keep, y / (1 - drop), 0.0)
    want = torch.nn.functional.cross_entropy(torch.cat([hidden[:n0], plain_mean(hidden, *inner)], 1) @ w2.t() + b2, labels)
    want.backward()
    assert abs(loss.item() - want.item()) <= 1e-5 * want.item()
    assert len(s.params) == 4 + 3 * blocks
    for p, q in zip(s.params, wide):
        # fp32 sums of a few hundred terms one after the other, and a relu whose argument may lie within their rounding of 0
        assert (p.grad - q.grad).norm() <= 1e-4 * q.grad.norm()
