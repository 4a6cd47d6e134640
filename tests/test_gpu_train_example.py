"""The training example: a minibatch's loss and gradients against plain torch on the same sampled block, and a run that
learns."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


def plain_mean(x, indptr, indices):
    n = indptr.numel() - 1
    lengths = (indptr[1:] - indptr[:-1]).long()
    of = torch.repeat_interleave(torch.arange(n, device=x.device), lengths)
    total = torch.zeros(n, x.shape[1], dtype=x.dtype, device=x.device).index_add(0, of, x[indices.long()])
    return total / lengths.clamp(min=1)[:, None]


@pytest.mark.parametrize("bits", [8, 4])
def test_a_minibatch_against_plain_torch(bits):
    from train_sage import Setup, unpack_rows
    s = Setup(bits, width=96)
    seeds, packed, (inner, outer) = s.sample(0)
    labels = s.labels[seeds.long()]
    loss = torch.nn.functional.cross_entropy(s.logits(packed, (inner, outer)), labels)
    loss.backward()
    x = unpack_rows(packed, s.fmt).double()
    w1, b1, w2, b2 = wide = [p.detach().double().requires_grad_() for p in s.params]
    n0, n1 = inner[0].numel() - 1, outer[0].numel() - 1
    hidden = torch.relu(torch.cat([x[:n1], plain_mean(x, *outer)], 1) @ w1.t() + b1)
    want = torch.nn.functional.cross_entropy(torch.cat([hidden[:n0], plain_mean(hidden, *inner)], 1) @ w2.t() + b2, labels)
    want.backward()
    assert abs(loss.item() - want.item()) <= 1e-5 * want.item()
    for p, q in zip(s.params, wide):
        # fp32 sums of a few hundred terms, and a relu whose argument may lie within their rounding of 0
        assert (p.grad - q.grad).norm() <= 1e-4 * q.grad.norm()


def test_it_learns():
    from train_sage import train
    losses = train(40, report=None)
    assert torch.isfinite(losses).all()
    assert losses[-5:].mean() < 0.7 * losses[:5].mean()
