"""AdamW refuses gradients of another shape than their parameter's."""
import pytest
import torch

from paper_2410_22697_amd import AdamW

pytestmark = pytest.mark.gpu


def test_gradients_of_another_shape_are_refused():
    p = torch.zeros(4, 6, device="cuda")
    opt = AdamW([p, torch.zeros(5, device="cuda")])
    g = torch.ones(4, 6, device="cuda")
    one = torch.ones(5, device="cuda")
    for bad in (g.t().contiguous(), g.reshape(-1), g.reshape(2, 12), g[:, :5], g.t()):
        with pytest.raises(ValueError):
            opt.step([bad, one])
        assert opt.t == 0 and torch.all(p == 0)
    opt.step([g, one])
    # a parameter given another shape or layout on the same memory
    q = torch.zeros(4, 4, device="cuda", requires_grad=True)
    opt = AdamW([q])
    q.data = q.data.view(2, 8)
    opt.step([torch.ones(2, 8, device="cuda")])
    q.data = q.data.view(4, 4).t()
    with pytest.raises(ValueError):
        opt.step([torch.ones(4, 4, device="cuda")])
    q.data = q.data.t()[:2]
    with pytest.raises(ValueError):
        opt.step([torch.ones(2, 4, device="cuda")])
