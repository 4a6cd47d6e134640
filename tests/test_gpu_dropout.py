"""Dropout and its gradient against the plain form in 64 bits."""
import os

import numpy as np
import pytest
import torch

import plain_layers
import plain_operators as plain
from paper_2410_22697_amd import dropout, dropout_backward, linear

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def wide(t):
    return t.detach().double().cpu().numpy()


def check(y, x, p, seed, draw, residual=None):
    """x times the fp32 scale is rounded, and so is its sum with the residual; the scale is half an ulp of fp32 off; a bf16
    result is rounded once."""
    keep = plain_layers.kept(*x.shape, p, seed, draw)
    scaled = np.where(keep, wide(x) / (1 - p) if p < 1 else 0.0, 0.0)
    want = scaled + (0 if residual is None else wide(residual))
    slack = 2 * plain.EPS * np.abs(scaled) + plain.EPS * np.abs(want) * (residual is not None) + 2.0 ** -149
    half = plain.BF / 2 if x.dtype == torch.bfloat16 else 0.0
    assert y.dtype == x.dtype
    assert np.all(np.abs(wide(y) - want) <= slack + half * (np.abs(want) + slack) * 1.01)
    if residual is None:
        assert np.array_equal(wide(y) == 0, ~keep | (wide(x) == 0))


def test_the_plain_generator_gives_the_known_answers():
    here = os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden", "philox4x32_10_kat.txt")
    lines = [[int(v, 16) for v in line.split()[-10:]] for line in open(here) if line.strip() and not line.startswith("#")]
    assert lines
    for v in lines:
        got = plain_layers.philox(*(np.array([c]) for c in v[:4]), v[4] + (v[5] << 32))
        assert [int(g[0]) for g in got] == v[6:10]


SIZES = [(1, 1), (1, 3), (3, 4), (2, 5), (7, 8), (300, 9), (33, 64), (129, 100), (16, 256), (5, 511), (64, 513), (3, 1100), (2, 5000), (70_001, 1)]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout(size, dtype):
    g = torch.Generator(device="cuda").manual_seed(size[0])
    new = lambda: torch.randn(size, generator=g, device="cuda").to(TYPES[dtype])  # noqa: E731
    for p, seed, draw in ((0.1, 1, 0), (0.5, 2 ** 64 - 5, 7), (0.9, -3, 2 ** 32 - 1), (0.0, 4, 1), (1.0, 5, 2), (1e-12, 6, 3)):
        x, res = new(), new()
        check(dropout(x, p, seed, draw), x, p, seed, draw)
        check(dropout(x, p, seed, draw=draw, residual=res), x, p, seed, draw, res)
        assert torch.equal(dropout_backward(x, p, seed, draw), dropout(x, p, seed, draw))
        at = torch.tensor(seed - 2 ** 64 if seed >= 2 ** 63 else seed, device="cuda")
        assert torch.equal(dropout(x, p, at, draw), dropout(x, p, seed, draw))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_any_stride_have_the_same_mask(dtype):
    wide_x = torch.randn(50, 301, device="cuda").to(TYPES[dtype])
    for a, d in ((0, 300), (1, 300), (3, 37), (5, 8), (2, 1)):
        x = wide_x[:, a:a + d]
        assert torch.equal(dropout(x, 0.3, 9, residual=x), dropout(x.contiguous(), 0.3, 9, residual=x.contiguous()))


def test_columns_that_drop_give_zero_whatever_they_hold():
    x = torch.randn(40, 64, device="cuda")
    keep = torch.from_numpy(plain_layers.kept(40, 64, 0.5, 3, 1)).cuda()
    for bad in (float("nan"), float("inf"), -float("inf")):
        y = dropout(torch.where(keep, x, bad), 0.5, 3, 1)
        assert torch.equal(y, torch.where(keep, x * 2, 0.0))
        y = dropout(torch.where(keep, bad, x), 0.5, 3, 1, residual=x)
        assert torch.equal(torch.isfinite(y), ~keep) and torch.equal(y[~keep], x[~keep])
    assert torch.equal(dropout(torch.full_like(x, float("nan")), 1.0, 3), torch.zeros_like(x))


def test_masks_of_other_draws_and_seeds_are_others_and_the_share_is_right():
    """2^20 columns: the share that drops is within six standard deviations of p, and two masks agree where chance lets them."""
    x = torch.ones(1024, 1024, device="cuda")
    n = x.numel()
    base = dropout(x, 0.3, 11, 0) == 0
    assert abs(base.sum().item() - 0.3 * n) < 6 * (0.21 * n) ** 0.5
    for seed, draw in ((12, 0), (11, 1), (11 + 2 ** 32, 0), (11, 2 ** 31)):
        other = dropout(x, 0.3, seed, draw) == 0
        assert abs((base & other).sum().item() - 0.09 * n) < 6 * (0.09 * 0.91 * n) ** 0.5


def test_gradients():
    """Dropout is linear: for any v, sum(dropout(v) w) is sum(v dx) with dx the gradient at w."""
    x, res, w = (torch.randn(130, 77, device="cuda") for _ in range(3))
    a, b = x.clone().requires_grad_(), res.clone().requires_grad_()
    at = torch.tensor([21], device="cuda")
    for seed in (21, at):
        y = dropout(a, 0.4, seed, 3, residual=b)
        a.grad = b.grad = None
        y.backward(w)
        assert torch.equal(b.grad, w) and torch.equal(a.grad, dropout_backward(w, 0.4, 21, 3))
        check(a.grad, w, 0.4, 21, 3)
    lhs, rhs = (wide(dropout(x, 0.4, 21, 3)) * wide(w)).sum(), (wide(x) * wide(a.grad)).sum()
    assert abs(lhs - rhs) <= 2 * plain.EPS * np.abs(wide(x) * wide(w)).sum() / 0.6 * 2
    only = dropout(x, 0.4, 21, 3, residual=b)
    b.grad = None
    only.backward(w.t().contiguous().t())
    assert torch.equal(b.grad, w)


def test_a_seed_that_changes_before_the_backward_pass_is_noticed():
    x, at = torch.randn(8, 8, device="cuda", requires_grad=True), torch.tensor([1], device="cuda")
    y = dropout(x, 0.5, at)
    at += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_replays_draw_by_the_seed_in_memory():
    x, at = torch.randn(300, 96, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    w = torch.randn(40, 96, device="cuda") * 0.1
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        linear(dropout(x, 0.5, at, 2), w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h = dropout(x, 0.5, at, 2, residual=x)
        y = linear(h, w)
        dx = dropout_backward(h, 0.5, at, 2)
        at += 1
    for step in range(5):
        x.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = dropout(x, 0.5, step, 2, residual=x)
        assert int(at) == step + 1
        assert torch.equal(h, want) and torch.equal(y, linear(want, w)) and torch.equal(dx, dropout_backward(want, 0.5, step, 2))


def test_on_another_stream():
    x = torch.randn(5000, 256, device="cuda")
    want = dropout(x, 0.2, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x2 = x * 1.0
        got = dropout(x2, 0.2, 5)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_empty():
    for shape in ((0, 5), (4, 0), (0, 0)):
        assert dropout(torch.empty(shape, device="cuda"), 0.5, 1).shape == shape
