"""AdamW on parameters that are given another view of their memory between steps."""
import pytest
import torch

from paper_2410_22697_amd import AdamW

pytestmark = pytest.mark.gpu


def test_views_of_the_same_memory():
    p, other = torch.zeros(2, 8, device="cuda", requires_grad=True), torch.zeros(3, device="cuda")
    opt = AdamW([p, other], weight_decay=0.0)
    for shape in ((2, 8), (4, 4), (16,), (1, 16), (4, 2, 2)):
        p.data = p.data.view(shape)
        for grads in ([torch.ones(shape, device="cuda"), None], [torch.ones(shape, device="cuda"), torch.ones(3, device="cuda")]):
            t = opt.t
            opt.step(grads)
            assert opt.t == t + 1 and torch.all(p == p.flatten()[0])
    p.data = p.data.view(4, 4).t()
    for grads in ([torch.ones(4, 4, device="cuda"), None], [torch.ones(4, 4, device="cuda"), torch.ones(3, device="cuda")]):
        with pytest.raises(ValueError, match="layout"):
            opt.step(grads)
    p.data = p.data.t()
    q = p.data.view(2, 2, 4)
    p.data = q
    opt.step([torch.ones(2, 2, 4, device="cuda"), None])
    p.data = q.transpose(0, 1)
    with pytest.raises(ValueError, match="layout"):
        opt.step([torch.ones(2, 2, 4, device="cuda"), None])
