"""AdamW refuses tensors that share memory."""
import pytest
import torch

from paper_2410_22697_amd import AdamW

pytestmark = pytest.mark.gpu


def test_tensors_that_share_memory_are_refused():
    p = torch.zeros(100, device="cuda")
    half = torch.zeros(100, device="cuda", dtype=torch.bfloat16)
    q = torch.zeros(100, device="cuda", dtype=torch.bfloat16)
    empty = torch.zeros(0, device="cuda")
    for bad in (lambda: AdamW([p, p]), lambda: AdamW([p[:60], p[50:]]), lambda: AdamW([p[:50], p[50:], p[10:11]]),
                lambda: AdamW([q], copies=[q]), lambda: AdamW([p, torch.zeros(100, device="cuda")], copies=[half, half]),
                lambda: AdamW([p[:50], p[50:]], copies=[half[:50], half[49:99]])):
        with pytest.raises(ValueError, match="share"):
            bad()
    AdamW([p[:50], p[50:], empty, empty], copies=[half[:50], half[50:], None, None]).step([torch.ones(50, device="cuda")] * 2 + [empty] * 2)
    other = torch.zeros(100, device="cuda", requires_grad=True)
    third = torch.zeros(100, device="cuda", requires_grad=True)
    opt = AdamW([other, third])
    third.data = other.data
    with pytest.raises(ValueError, match="share"):
        opt.step([p, p])
