"""The gated layer and its gradients, against the plain form in 64 bits."""
import numpy as np
import pytest
import torch

import plain_layers
import plain_operators as plain
from paper_2410_22697_amd import gated, gated_backward

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ["silu", "gelu", "relu", "none"]


def wide(t):
    return t.detach().double().cpu().numpy()


def make(rows, k, k2, n, dtype, seed=0, bias=True):
    g = torch.Generator(device="cuda").manual_seed(seed + rows * 7 + k * 3 + n)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    return dict(x=new(rows, k), x2=new(rows, k2) if k2 else None, weight=(new(2 * n, k + k2).float() / (k + k2) ** 0.5).to(dtype),
                bias=new(2 * n) if bias else None)


def inputs(a):
    return wide(a["x"]) if a["x2"] is None else np.concatenate([wide(a["x"]), wide(a["x2"])], 1)


def check_forward(got, pre, a, act, dtype):
    """A product of K terms rounds its sum K times at most; an activation's slope is 1.13 at most and its own error 4e-7 of its
    argument and 1; the product of both halves takes over what either is off; a bf16 result is rounded once."""
    x, w = inputs(a), wide(a["weight"])
    b = np.zeros(len(w)) if a["bias"] is None else wide(a["bias"])
    y, z = plain_layers.gated(x, w, b, act)
    n, half = y.shape[1], plain.BF / 2 if dtype == torch.bfloat16 else 0.0
    slack = (x.shape[1] + 4) * plain.EPS * (np.abs(x) @ np.abs(w).T + np.abs(b))
    if pre is not None:
        assert pre.dtype == dtype and np.all(np.abs(wide(pre) - z) <= slack + half * (np.abs(z) + slack))
    value = np.abs(plain.act(z[:, :n], act))
    off = 1.13 * slack[:, :n] + 4e-7 * (np.abs(z[:, :n]) + 1) * (act != "none")
    off = off * (np.abs(z[:, n:]) + slack[:, n:]) + value * slack[:, n:] + plain.EPS * np.abs(y)
    assert got.dtype == dtype and got.shape == y.shape
    assert np.all(np.abs(wide(got) - y) <= off + half * (np.abs(y) + off))


SIZES = [(1, 1, 0, 1), (1, 128, 128, 256), (2, 7, 5, 3), (5, 33, 0, 47), (16, 128, 128, 256), (64, 64, 64, 64), (65, 100, 100, 65),
         (129, 300, 0, 129), (200, 8, 16, 300), (1000, 50, 50, 172), (3, 1000, 1000, 17), (517, 257, 31, 1), (1, 600, 0, 1100)]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward(size, dtype):
    rows, k, k2, n = size
    for i, act in enumerate(ACTS):
        a = make(rows, k, k2, n, TYPES[dtype], i, bias=i != 1)
        check_forward(gated(a["x"], a["weight"], a["bias"], act=act, x2=a["x2"]), None, a, act, TYPES[dtype])
        y, pre = gated(a["x"], a["weight"], a["bias"], act=act, x2=a["x2"], save_pre=True)
        check_forward(y, pre, a, act, TYPES[dtype])


# enough results for the form of many rows: narrow and wide outputs, ragged tiles of rows and outputs, odd ends of either input
MANY = [(33_001, 64, 0, 40), (8201, 40, 33, 130), (9001, 1, 0, 257), (4097, 7, 3, 256), (70_003, 24, 0, 16), (3000, 511, 130, 353), (2100, 96, 0, 1024)]


@pytest.mark.parametrize("size", MANY)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_on_many_rows(size, dtype):
    rows, k, k2, n = size
    for i, act in enumerate(ACTS):
        a = make(rows, k, k2, n, TYPES[dtype], bias=i != 2)
        y, pre = gated(a["x"], a["weight"], a["bias"], act=act, x2=a["x2"], save_pre=True)
        check_forward(y, pre, a, act, TYPES[dtype])
        assert torch.equal(y, gated(a["x"], a["weight"], a["bias"], act=act, x2=a["x2"]))


def check_backward(got, dy, pre, a, act, dtype):
    """dg and du are rounded to bf16 for the bf16 products; the rest as in the forward pass. db sums them unrounded."""
    dx, dx2, dw, db = got
    x, w, k = inputs(a), wide(a["weight"]), a["x"].shape[1]
    d, p, n = wide(dy), wide(pre), dy.shape[1]
    dz = plain_layers.gated_dz(d, p, act)
    half = plain.BF / 2 if dtype == torch.bfloat16 else 0.0
    curve = 4e-7 * (act != "none") * np.concatenate([np.abs(d * p[:, n:]), np.abs(d)], 1) * (1 + np.abs(np.concatenate([p[:, :n]] * 2, 1)))
    own = curve + 4 * plain.EPS * np.abs(dz)
    off = own + half * (np.abs(dz) + own)

    def close(t, want, slack):
        assert t.dtype == dtype and t.shape == want.shape
        assert np.all(np.abs(wide(t) - want) <= slack + half * (np.abs(want) + slack))

    want, slack = dz @ w, off @ np.abs(w) + (len(w) + 2) * plain.EPS * (np.abs(dz) @ np.abs(w))
    close(dx, want[:, :k], slack[:, :k])
    if dx2 is not None:
        close(dx2, want[:, k:], slack[:, k:])
    close(dw, dz.T @ x, off.T @ np.abs(x) + (len(x) + 2) * plain.EPS * (np.abs(dz).T @ np.abs(x)))
    if db is not None:
        close(db, dz.sum(0), own.sum(0) + (len(x) + 2) * plain.EPS * np.abs(dz).sum(0))


@pytest.mark.parametrize("size", SIZES + MANY[1:4] + [(5000, 24, 0, 30), (2100, 130, 70, 140), (4100, 600, 0, 520)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward(size, dtype):
    rows, k, k2, n = size
    t = TYPES[dtype]
    for i, act in enumerate(ACTS):
        a = make(rows, k, k2, n, t, i)
        dy, pre = torch.randn(rows, n, device="cuda").to(t), (2 * torch.randn(rows, 2 * n, device="cuda")).to(t)
        got = gated_backward(dy, a["x"], a["weight"], pre, act, a["x2"])
        check_backward(got, dy, pre, a, act, t)
        only = gated_backward(dy, a["x"], a["weight"], pre, act, a["x2"], bias=False)
        assert only[3] is None
        assert all(u is None and v is None or torch.equal(u, v) for u, v in zip(only[:3], got[:3]))
        if i == 0:
            ask = dict(bias=False, need_dx=False, need_dx2=False, need_dw=False)
            for name, at in (("need_dx", 0), ("need_dx2", 1), ("need_dw", 2), ("bias", 3)):
                one = gated_backward(dy, a["x"], a["weight"], pre, act, a["x2"], **{**ask, name: True})
                assert all(u is None for j, u in enumerate(one) if j != at)
                if got[at] is not None:  # (a form for one input's columns may split its tiles in other places)
                    check = [got[0], got[1], got[2], got[3]]
                    check[at] = one[at]
                    check_backward(check, dy, pre, a, act, t)


def test_rows_of_any_stride():
    for dtype in TYPES.values():
        big = torch.randn(300, 1501, device="cuda").to(dtype)
        for rows, n in ((16, 40), (300, 40), (300, 200)):
            x, x2, w = big[:rows, 1:60], big[:rows, 3:40], big[:2 * n, 5:101] if 2 * n <= 300 else torch.randn(2 * n, 97, device="cuda").to(dtype)[:, 1:]
            dy, pre = big[:rows, 7:7 + n], big[:rows, 2:2 + 2 * n]
            b = torch.randn(2 * n, device="cuda").to(dtype)
            c = torch.Tensor.contiguous
            assert all(torch.equal(u, v) for u, v in zip(gated(x, w, b, x2=x2, save_pre=True), gated(c(x), c(w), b, x2=c(x2), save_pre=True)))
            assert all(torch.equal(u, v) for u, v in zip(gated_backward(dy, x, w, pre, x2=x2), gated_backward(c(dy), c(x), c(w), c(pre), x2=c(x2))))


@pytest.mark.parametrize("rows,n", [(40, 50), (9000, 200)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite_stays_in_its_row(rows, n, dtype):
    a = make(rows, 37, 20, n, TYPES[dtype])
    x = a["x"].clone()
    x[3, 5], x[17, 0], x[rows - 1, 36] = float("nan"), float("inf"), float("nan")
    y, pre = gated(x, a["weight"], a["bias"], x2=a["x2"], save_pre=True)
    want = gated(a["x"], a["weight"], a["bias"], x2=a["x2"])
    fine = torch.ones(rows, dtype=torch.bool, device="cuda")
    fine[torch.tensor([3, 17, rows - 1], device="cuda")] = False
    assert torch.equal(y[fine], want[fine]) and torch.isnan(y[3]).all() and torch.isnan(y[rows - 1]).all() and not torch.isfinite(pre[17]).any()
    dy = torch.randn(rows, n, device="cuda").to(TYPES[dtype])
    z = torch.nan_to_num(pre, nan=1.0, posinf=2.0, neginf=-2.0)
    good = gated_backward(dy, a["x"], a["weight"], z, x2=a["x2"])
    dy[3, 1] = float("nan")
    bad = gated_backward(dy, a["x"], a["weight"], z, x2=a["x2"])
    rest = torch.arange(rows, device="cuda") != 3
    for u, v in zip(bad[:2], good[:2]):
        assert torch.isnan(u[3]).all() and torch.equal(u[rest], v[rest])
    cols = (torch.arange(2 * n, device="cuda") % n) != 1
    for u, v in zip(bad[2:], good[2:]):
        assert torch.isnan(u[~cols]).all() and torch.equal(u[cols], v[cols])


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(act):
    """sum(y v) along a direction, by central differences of the plain form in 64 bits (h = 1e-6: off by h^2 times a third
    derivative and by 1e-16 / h, 1e-9 of the terms at most) and by autograd, in fp32."""
    a = make(30, 20, 10, 25, torch.float32, 3)
    v = torch.randn(30, 25, device="cuda")
    p = {k: t.clone().requires_grad_() for k, t in a.items()}
    y = gated(p["x"], p["weight"], p["bias"], act=act, x2=p["x2"])
    y.backward(v)
    t = {k: torch.randn_like(q) for k, q in a.items()}

    def loss(h):
        q = {k: wide(a[k]) + h * wide(t[k]) for k in a}
        return (plain_layers.gated(np.concatenate([q["x"], q["x2"]], 1), q["weight"], q["bias"], act)[0] * wide(v)).sum()

    want = (loss(1e-6) - loss(-1e-6)) / 2e-6
    terms = [wide(p[k].grad) * wide(t[k]) for k in a]
    # sums of 80 products at most, each of values that are themselves off by sums of 30: 200 roundings of terms 10 times a gradient's size
    if act == "relu":  # no value lies within h of the corner
        z = inputs(a) @ wide(a["weight"]).T + wide(a["bias"])
        assert np.abs(z).min() > 1e-5
    assert abs(sum(k.sum() for k in terms) - want) <= (2000 * plain.EPS + 1e-8) * sum(np.abs(k).sum() for k in terms)


def test_autograd_asks_for_what_is_needed():
    a = make(40, 30, 20, 24, torch.float32)
    v = torch.randn(24, 40, device="cuda").t()  # not contiguous
    y, pre = gated(a["x"], a["weight"], a["bias"], x2=a["x2"], save_pre=True)
    want = dict(zip(("x", "x2", "weight", "bias"), gated_backward(v.contiguous(), a["x"], a["weight"], pre, x2=a["x2"])))
    for names in (("x",), ("x2",), ("weight",), ("bias",), ("x", "weight", "bias", "x2"), ("x", "bias")):
        p = {k: t.clone().requires_grad_(k in names) for k, t in a.items()}
        out = gated(p["x"], p["weight"], p["bias"], x2=p["x2"])
        assert torch.equal(out, y)
        out.backward(v)
        for k in a:
            assert (p[k].grad is None) == (k not in names)
            assert p[k].grad is None or torch.allclose(p[k].grad, want[k], rtol=1e-4, atol=1e-4)
    with pytest.raises(ValueError, match="outside autograd"):
        gated(a["x"].clone().requires_grad_(), a["weight"], save_pre=True)


def test_replayed():
    a = make(4500, 64, 32, 300, torch.bfloat16)
    dy = torch.randn(4500, 300, device="cuda").to(torch.bfloat16)

    def step():
        y, pre = gated(a["x"], a["weight"], a["bias"], x2=a["x2"], save_pre=True)
        return (y, pre, *gated_backward(dy, a["x"], a["weight"], pre, x2=a["x2"]))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        for t in (a["x"], a["x2"], dy):
            t.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(out, step()))


def test_no_rows():
    for dtype in TYPES.values():
        a = make(0, 6, 3, 5, dtype)
        y, pre = gated(a["x"], a["weight"], a["bias"], x2=a["x2"], save_pre=True)
        assert y.shape == (0, 5) and pre.shape == (0, 10)
        dx, dx2, dw, db = gated_backward(y, a["x"], a["weight"], pre, x2=a["x2"])
        assert dx.shape == (0, 6) and dx2.shape == (0, 3) and not dw.any() and not db.any() and dw.shape == (10, 9) and db.shape == (10,)
