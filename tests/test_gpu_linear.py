"""A layer's product with its epilogue, and its gradients, against the plain form in 64 bits."""
import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2410_22697_amd import linear, linear_backward

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ["none", "relu", "gelu", "silu"]


def make(rows, k, k2, n, dtype, seed=0, bias=True, residual=True):
    g = torch.Generator(device="cuda").manual_seed(seed + rows * 7 + k * 3 + n)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    return dict(x=new(rows, k), x2=new(rows, k2) if k2 else None, weight=(new(n, k + k2).float() / (k + k2) ** 0.5).to(dtype),
                bias=new(n) if bias else None, residual=new(rows, n) if residual else None)


def wide(t):
    return None if t is None else t.detach().double().cpu().numpy()


def check_forward(got, pre, a, act, dtype):
    """A product of K terms rounds its sum K times at most; an activation's slope is 1.13 at most and its own error a few
    ulps; a bf16 result is rounded once."""
    x = wide(a["x"]) if a["x2"] is None else np.concatenate([wide(a["x"]), wide(a["x2"])], 1)
    w = wide(a["weight"])
    z = x @ w.T
    mag = np.abs(x) @ np.abs(w).T
    if a["bias"] is not None:
        z = z + wide(a["bias"])
        mag = mag + np.abs(wide(a["bias"]))
    slack = (x.shape[1] + 4) * plain.EPS * mag
    half = plain.BF / 2 if dtype == torch.bfloat16 else 0.0
    if pre is not None:
        assert np.all(np.abs(wide(pre) - z) <= slack + half * (np.abs(z) + slack))
    y = plain.act(z, act)
    slack = 1.13 * slack + 4e-7 * (np.abs(z) + 1) * (act != "none")
    if a["residual"] is not None:
        y = y + wide(a["residual"])
        slack = slack + 2 * plain.EPS * (np.abs(y) + np.abs(wide(a["residual"])))
    assert got.dtype == dtype
    assert np.all(np.abs(wide(got) - y) <= slack + half * (np.abs(y) + slack))


SIZES = [(1, 1, 0, 1), (1, 128, 128, 256), (2, 7, 5, 3), (5, 33, 0, 47), (16, 128, 128, 256), (64, 64, 64, 64), (65, 100, 100, 65),
         (129, 300, 0, 129), (200, 8, 16, 300), (1000, 50, 50, 172), (3, 1000, 1000, 17), (517, 257, 31, 1)]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward(size, dtype):
    rows, k, k2, n = size
    for i, act in enumerate(ACTS):
        a = make(rows, k, k2, n, TYPES[dtype], i, bias=i != 1, residual=i % 2 == 1)
        check_forward(linear(a["x"], a["weight"], a["bias"], act=act, residual=a["residual"], x2=a["x2"]), None, a, act, TYPES[dtype])
        y, pre = linear(a["x"], a["weight"], a["bias"], act=act, residual=a["residual"], x2=a["x2"], save_pre=True)
        check_forward(y, pre, a, act, TYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_on_many_rows(dtype):
    """Enough rows for the large tiles, narrow and wide, and a last tile of few rows."""
    for rows, k, k2, n in ((33_001, 64, 0, 40), (33_001, 40, 40, 130), (70_003, 24, 0, 70)):
        a = make(rows, k, k2, n, TYPES[dtype])
        check_forward(linear(a["x"], a["weight"], a["bias"], act="relu", residual=a["residual"], x2=a["x2"]), None, a, "relu", TYPES[dtype])


# enough results for rows to be streamed: weights that stay in LDS and that pass through it, one to many groups of
# outputs, segments that end inside a vector, a step or a chunk, inputs of a few columns, a last tile of one row
STREAMED = [(70_001, 5, 0, 30), (70_001, 3, 2, 33), (33_000, 64, 64, 64), (9_001, 100, 28, 256), (9_001, 129, 67, 257), (8_193, 700, 130, 256),
            (8_200, 1030, 0, 300), (33_025, 300, 300, 70), (2_300, 16, 0, 1000)]


@pytest.mark.parametrize("size", STREAMED)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_streamed(size, dtype):
    rows, k, k2, n = size
    for act, residual in (("gelu", False), ("relu", True)):
        a = make(rows, k, k2, n, TYPES[dtype], bias=residual, residual=residual)
        y, pre = linear(a["x"], a["weight"], a["bias"], act=act, residual=a["residual"], x2=a["x2"], save_pre=True)
        check_forward(y, pre, a, act, TYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_streamed_rows_of_any_stride(dtype):
    """As below, where rows are streamed: NaN around the operands reaches no result, and a row's own stays in it."""
    t = TYPES[dtype]
    rows, k, k2, n = 9_003, 133, 21, 270

    def inside(x, left, right):
        big = torch.full((x.shape[0] + 2, x.shape[1] + left + right), float("nan"), dtype=t, device="cuda")
        big[1:1 + x.shape[0], left:left + x.shape[1]] = x
        return big[1:1 + x.shape[0], left:left + x.shape[1]]

    a = make(rows, k, k2, n, t)
    b = dict(a, x=inside(a["x"], 1, 2), x2=inside(a["x2"], 3, 0), weight=inside(a["weight"], 1, 1), residual=inside(a["residual"], 5, 2))
    y, pre = linear(b["x"], b["weight"], b["bias"], act="silu", residual=b["residual"], x2=b["x2"], save_pre=True)
    check_forward(y, pre, a, "silu", t)
    dy = torch.randn(rows, n, device="cuda").to(t)
    got = linear_backward(inside(dy, 3, 2), b["x"], b["weight"], "silu", inside(pre, 2, 1), b["x2"])
    check_backward(got, dy, a, "silu", pre, t)
    a["x"][77, 132] = float("nan")
    a["x"][8_000, 0] = float("inf")
    y2 = linear(a["x"], a["weight"], a["bias"], act="silu", residual=a["residual"], x2=a["x2"])
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[[77, 8_000]] = False
    assert torch.equal(y2[keep], y[keep]) and torch.isnan(y2[77]).all()
    want = torch.isnan((a["x"][8_000:8_001].float() @ a["weight"][:, :k].float().t()))[0]
    assert not want.any() and not torch.isfinite(y2[8_000]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_any_stride_and_what_lies_around_them(dtype):
    """Columns and rows around the operands hold NaN: none of it may reach a result."""
    t = TYPES[dtype]

    def inside(x, left, right):
        big = torch.full((x.shape[0] + 3, x.shape[1] + left + right), float("nan"), dtype=t, device="cuda")
        big[1:1 + x.shape[0], left:left + x.shape[1]] = x
        return big[1:1 + x.shape[0], left:left + x.shape[1]]

    for rows, k, k2, n in ((70, 33, 21, 45), (130, 64, 8, 128), (16, 100, 28, 20)):
        a = make(rows, k, k2, n, t)
        b = dict(a, x=inside(a["x"], 1, 2), x2=inside(a["x2"], 3, 0), weight=inside(a["weight"], 1, 1), residual=inside(a["residual"], 5, 2))
        y, pre = linear(b["x"], b["weight"], b["bias"], act="gelu", residual=b["residual"], x2=b["x2"], save_pre=True)
        check_forward(y, pre, a, "gelu", t)
        dy = inside(torch.randn(rows, n, device="cuda").to(t), 1, 4)
        got = linear_backward(dy, b["x"], b["weight"], "gelu", inside(pre, 2, 1), b["x2"])
        check_backward(got, dy, a, "gelu", pre, t)


def test_values_that_are_not_finite_stay_in_their_rows():
    for t in TYPES.values():
        a = make(70, 40, 0, 50, t)
        a["x"][3, 5] = float("nan")
        a["x"][9, 0] = float("inf")
        y = linear(a["x"], a["weight"], a["bias"], act="relu")
        bad = torch.tensor([3, 9], device="cuda")
        keep = torch.ones(70, dtype=torch.bool, device="cuda")
        keep[bad] = False
        assert torch.isfinite(y[keep]).all()
        assert torch.isnan(y[3]).all()
        want = (a["x"][9:10].float() @ a["weight"].float().t()).clamp(min=0)
        assert torch.equal(torch.isinf(y[9]), torch.isinf(want[0])) and torch.equal(torch.isnan(y[9]), torch.isnan(want[0]))


# ------------------------------------------------------------------ backward
def check_backward(got, dy, a, act, pre, dtype):
    """dz is rounded to bf16 for the bf16 products unless it is dy or 0; the rest as in the forward pass."""
    dx, dx2, dw, db = got
    x = wide(a["x"]) if a["x2"] is None else np.concatenate([wide(a["x"]), wide(a["x2"])], 1)
    w = wide(a["weight"])
    dz = wide(dy) * (1.0 if act == "none" else plain.slope(wide(pre), act))
    half = plain.BF / 2 if dtype == torch.bfloat16 else 0.0
    curved = act in ("gelu", "silu")
    # an absolute error of 4e-7 in the slope, and a factor's rounding
    dz_slack = curved * (np.abs(wide(dy)) * 4e-7 * (1 + np.abs(wide(pre) if curved else 0)) + (half + 4 * plain.EPS) * np.abs(dz))

    def close(t, want, slack):
        assert t.dtype == dtype
        assert np.all(np.abs(wide(t) - want) <= slack + half * (np.abs(want) + slack))

    k = a["x"].shape[1]
    if dx is not None or dx2 is not None:
        want = dz @ w
        slack = dz_slack @ np.abs(w) + (w.shape[0] + 2) * plain.EPS * (np.abs(dz) @ np.abs(w))
        if dx is not None:
            close(dx, want[:, :k], slack[:, :k])
        if dx2 is not None:
            close(dx2, want[:, k:], slack[:, k:])
    if dw is not None:
        close(dw, dz.T @ x, dz_slack.T @ np.abs(x) + (len(x) + 2) * plain.EPS * (np.abs(dz).T @ np.abs(x)))
    if db is not None:
        close(db, dz.sum(0), dz_slack.sum(0) + (len(x) + 2) * plain.EPS * np.abs(dz).sum(0))


@pytest.mark.parametrize("size", SIZES + [(5000, 24, 0, 30), (2100, 130, 70, 140)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward(size, dtype):
    rows, k, k2, n = size
    t = TYPES[dtype]
    for i, act in enumerate(ACTS):
        a = make(rows, k, k2, n, t, i)
        dy = torch.randn(rows, n, device="cuda").to(t)
        pre = None if act == "none" else (3 * torch.randn(rows, n, device="cuda")).to(t)
        check_backward(linear_backward(dy, a["x"], a["weight"], act, pre, a["x2"]), dy, a, act, pre, t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_on_many_rows(dtype):
    t = TYPES[dtype]
    for rows, k, k2, n, act in ((40_003, 64, 64, 100, "relu"), (40_003, 33, 0, 140, "gelu"), (70_001, 20, 20, 10, "none")):
        a = make(rows, k, k2, n, t)
        dy = torch.randn(rows, n, device="cuda").to(t)
        pre = None if act == "none" else torch.randn(rows, n, device="cuda").to(t)
        got = linear_backward(dy, a["x"], a["weight"], act, pre, a["x2"])
        check_backward(got, dy, a, act, pre, t)
        again = linear_backward(dy, a["x"], a["weight"], act, pre, a["x2"])
        assert all(u is None and v is None or torch.equal(u, v) for u, v in zip(got, again))


@pytest.mark.parametrize("size", [(70_001, 30, 0, 5), (70_001, 33, 2, 3), (33_000, 64, 64, 64), (9_001, 128, 128, 256), (9_001, 257, 3, 129),
                                  (8_193, 256, 0, 700), (8_200, 70, 300, 1030), (2_300, 1000, 0, 16), (5_000, 9, 250, 300)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_streamed(size, dtype):
    """dx's forms and dw's tiles: one and several of each, columns that both inputs share a vector or a tile over."""
    rows, k, k2, n = size
    t = TYPES[dtype]
    for act in ("none", "gelu", "relu"):
        a = make(rows, k, k2, n, t)
        dy = torch.randn(rows, n, device="cuda").to(t)
        pre = None if act == "none" else (2 * torch.randn(rows, n, device="cuda")).to(t)
        check_backward(linear_backward(dy, a["x"], a["weight"], act, pre, a["x2"]), dy, a, act, pre, t)
    if k2:
        for ask in (dict(need_dx=False), dict(need_dx2=False)):
            got = linear_backward(dy, a["x"], a["weight"], act, pre, a["x2"], need_dw=False, bias=False, **ask)
            check_backward(got, dy, a, act, pre, t)


def test_each_gradient_alone():
    a = make(300, 40, 24, 70, torch.float32)
    dy, pre = torch.randn(2, 300, 70, device="cuda")
    every = linear_backward(dy, a["x"], a["weight"], "silu", pre, a["x2"])
    for i in range(4):
        ask = dict(need_dx=i == 0, need_dx2=i == 1, need_dw=i == 2, bias=i == 3)
        one = linear_backward(dy, a["x"], a["weight"], "silu", pre, a["x2"], **ask)
        assert [j for j in range(4) if one[j] is not None] == [i]
        # (another set of columns may take another tile: compare by the oracle's bounds)
        check_backward(one, dy, a, "silu", pre, torch.float32)
    check_backward(every, dy, a, "silu", pre, torch.float32)
    assert linear_backward(dy, a["x"], a["weight"], "silu", pre, a["x2"], bias=False, need_dx=False, need_dx2=False, need_dw=False) == (None,) * 4


def test_slopes_at_the_ends():
    """Where an activation is flat or the identity its slope is 0 or 1, also at infinities."""
    ends = torch.tensor([float("inf"), float("-inf"), 60.0, -60.0, 0.0, -0.0], device="cuda")
    for t in TYPES.values():
        for act, at0 in (("relu", 0.0), ("gelu", 0.5), ("silu", 0.5)):
            pre = ends[:, None].to(t)
            dx = linear_backward(torch.ones(6, 1, device="cuda", dtype=t), torch.ones(6, 1, device="cuda", dtype=t),
                                 torch.ones(1, 1, device="cuda", dtype=t), act, pre, bias=False, need_dw=False)[0]
            assert torch.allclose(dx[:, 0].float(), torch.tensor([1, 0, 1, 0, at0, at0], device="cuda"), atol=1e-6), act


def test_no_rows():
    for t in TYPES.values():
        a = make(0, 12, 4, 9, t)
        assert linear(a["x"], a["weight"], a["bias"], x2=a["x2"]).shape == (0, 9)
        dx, dx2, dw, db = linear_backward(torch.zeros(0, 9, device="cuda", dtype=t), a["x"], a["weight"], x2=a["x2"])
        assert dx.shape == (0, 12) and dx2.shape == (0, 4)
        assert torch.equal(dw, torch.zeros(9, 16, device="cuda", dtype=t)) and torch.equal(db, torch.zeros(9, device="cuda", dtype=t))


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(act):
    """Central differences of the plain form in 64 bits, along random directions; step 1e-4: their own error is ~1e-7."""
    rng = np.random.default_rng(2)
    x, w, b, dy = (rng.standard_normal(s).astype(np.float32) for s in ((40, 9), (13, 9), (13,), (40, 13)))
    f = lambda x, w, b: (plain.act(x @ w.T + b, act) * dy).sum()  # noqa: E731
    wide_in = [v.astype(np.float64) for v in (x, w, b)]
    z = wide_in[0] @ wide_in[1].T + wide_in[2]
    pre = None if act == "none" else torch.from_numpy(z.astype(np.float32)).cuda()
    dx, _, dw, db = linear_backward(*(torch.from_numpy(v).cuda() for v in (dy, x, w)), act, pre)
    for i, grad in enumerate((dx, dw, db)):
        for _ in range(4):
            v = rng.standard_normal(wide_in[i].shape)
            up, down = (f(*[u + s * 1e-4 * v if j == i else u for j, u in enumerate(wide_in)]) for s in (1, -1))
            got = (grad.double().cpu().numpy() * v).sum()
            # relu: an argument within 1e-4 |change| of 0 may lie on either side
            kink = 0.0
            if act == "relu":
                change = np.abs(v @ wide_in[1].T if i == 0 else wide_in[0] @ v.T if i == 1 else np.broadcast_to(v, z.shape))
                kink = (np.abs(dy) * change * (np.abs(z) <= 1e-4 * change)).sum()
            scale = np.abs(dy).sum() * 3
            assert abs((up - down) / 2e-4 - got) <= 2e-6 * scale + kink


@pytest.mark.parametrize("act", ACTS)
def test_autograd(act):
    a = make(90, 24, 10, 33, torch.float32)
    leaves = [t.requires_grad_() for t in (a["x"], a["weight"], a["bias"], a["residual"], a["x2"])]
    dy = torch.randn(90, 33, device="cuda")
    for residual in (None, a["residual"]):
        for t in leaves:
            t.grad = None
        linear(a["x"], a["weight"], a["bias"], act=act, residual=residual, x2=a["x2"]).backward(dy)
        with torch.no_grad():
            _, pre = linear(a["x"], a["weight"], a["bias"], act=act, x2=a["x2"], save_pre=True)
            dx, dx2, dw, db = linear_backward(dy, a["x"], a["weight"], act, None if act == "none" else pre, a["x2"])
        for got, want in zip((a["x"].grad, a["x2"].grad, a["weight"].grad, a["bias"].grad), (dx, dx2, dw, db)):
            assert torch.equal(got, want)
        assert residual is None or torch.equal(a["residual"].grad, dy)


def test_refusals():
    x, w, b = torch.zeros(4, 6, device="cuda"), torch.zeros(5, 6, device="cuda"), torch.zeros(5, device="cuda")
    dy = torch.zeros(4, 5, device="cuda")
    for bad in (lambda: linear(x, w[:, :5]), lambda: linear(x, w.bfloat16()), lambda: linear(x.half(), w.half()),
                lambda: linear(x, w, b[:4]), lambda: linear(x, w, b.bfloat16()), lambda: linear(x, w, act="tanh"),
                lambda: linear(x, w, residual=dy[:3]), lambda: linear(x, w, x2=x), lambda: linear(x.t(), w), lambda: linear(x[:1].expand(4, 6), w),
                lambda: linear(x, w.cpu()), lambda: linear_backward(dy, x, w, "relu"), lambda: linear_backward(dy, x, w, "none", dy),
                lambda: linear_backward(dy[:, :4], x, w), lambda: linear_backward(dy, x, w, "relu", dy.bfloat16()),
                lambda: linear(x.requires_grad_(), w, save_pre=True)):
        with pytest.raises(ValueError):
            bad()
