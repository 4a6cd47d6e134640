"""AdamW counts each tensor's steps."""
import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2410_22697_amd import AdamW

pytestmark = pytest.mark.gpu
LR, B1, B2 = 1e-3, 0.9, 0.999


def cpu(t):
    return t.detach().float().cpu().numpy().astype(np.float64).reshape(-1)


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_are_counted_for_each_tensor(bits):
    """A tensor whose first gradient comes late takes its first step then, whatever the others have taken."""
    a, b = torch.randn(300, device="cuda"), torch.randn(500, device="cuda")
    start = b.clone()
    opt = AdamW([a, b], lr=LR, betas=(B1, B2), weight_decay=0.0, state_bits=bits)
    twin_p = a.clone()
    twin = AdamW([twin_p], lr=LR, betas=(B1, B2), weight_decay=0.0, state_bits=bits)
    gen = torch.Generator(device="cuda").manual_seed(0)
    for _ in range(6):
        g = torch.randn(300, device="cuda", generator=gen)
        opt.step([g, None])
        twin.step([g])
    assert torch.equal(b, start) and opt.t == 6
    last, g = torch.randn(300, device="cuda", generator=gen), torch.randn(500, device="cuda", generator=gen)
    opt.step([last, g])
    twin.step([last])
    assert torch.equal(a, twin_p) and opt.t == 7
    want, _, _ = plain.adamw(cpu(start), cpu(g), np.zeros(500), np.zeros(500), 1, LR, B1, B2, 1e-8, 0.0)
    assert np.all(np.abs(cpu(b) - want) <= 20 * plain.EPS * (np.abs(want) + LR))
    late = AdamW([start], lr=LR, betas=(B1, B2), weight_decay=0.0, state_bits=bits)
    late.step([g])
    assert torch.equal(b, start)
    for _ in range(3):  # and the next ones with both
        ga, gb = torch.randn(300, device="cuda", generator=gen), torch.randn(500, device="cuda", generator=gen)
        opt.step([ga, gb])
        twin.step([ga])
        late.step([gb])
        assert torch.equal(a, twin_p) and torch.equal(b, start)


def test_a_count_that_is_set_holds_for_every_tensor():
    g = torch.ones(10, device="cuda")
    p, q = torch.zeros(10, device="cuda"), torch.zeros(10, device="cuda")
    opt = AdamW([p, q], weight_decay=0.0)
    opt.step([g, None])
    opt.t = 0
    opt.m.zero_(), opt.v.zero_(), p.zero_()
    opt.step([g, g])
    assert opt.t == 1 and torch.equal(p, q)
