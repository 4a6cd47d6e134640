"""Forward-mode tangents: refused, not dropped."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2410_22697_amd import AdamW, block_mean, block_mean_backward, linear, linear_backward

pytestmark = pytest.mark.gpu


def test_tangents_are_refused():
    x, w = torch.randn(6, 16, device="cuda"), torch.randn(5, 16, device="cuda")
    indptr, indices = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 2, 3], [0, 5, 1]))
    pre = torch.randn(6, 5, device="cuda")
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        wd = forward_ad.make_dual(w, torch.ones_like(w))
        d = forward_ad.make_dual(pre, torch.ones_like(pre))
        for bad in (lambda: linear(dual, w), lambda: linear(x, wd), lambda: linear(x, w, residual=d), lambda: linear(dual, w, save_pre=True),
                    lambda: block_mean(dual, indptr, indices), lambda: linear_backward(d, x, w), lambda: linear_backward(pre, x, wd),
                    lambda: block_mean_backward(dual[:2], indptr, indices, 6), lambda: AdamW([x]).step([dual])):
            with pytest.raises(ValueError, match="tangent"):
                bad()
        want = linear(x, w)
    assert torch.equal(linear(x, w), want)
