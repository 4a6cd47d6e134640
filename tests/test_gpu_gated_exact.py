"""The gated layer and its gradients in every form (gated_sizes), on small whole numbers whose products and sums are exact in
both types: the results are the wanted bits, whatever the order of the sums, so that a row, a column or a part that is lost,
taken twice or put in another's place shows.

Gates are far from 0 on either side, where every activation is z or 0 and its slope 1 or 0 exactly: the activations' own
values are tested elsewhere. Sums stay below 2^24 of their terms' common unit, so that fp32 holds each of them; a result in
bf16 is the exact one rounded once, to nearest even. Inputs lie between NaNs; outputs are larger than asked for, and what is
beside them stays as it was; the workspace begins as NaNs, and what follows it stays."""
import ctypes

import pytest
import torch

from gated_sizes import FORWARD, GRADIENTS
from paper_2410_22697_amd import gated, gated_backward, operators

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ["silu", "gelu", "relu", "none"]
NAN = float("nan")


class Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def whole(self, low, high, *shape):
        return torch.randint(low, high + 1, shape, generator=self.g, device="cuda")

    def one_of(self, values, *shape):
        return torch.tensor(values, device="cuda")[torch.randint(0, len(values), shape, generator=self.g, device="cuda")]


def among_nans(t, dtype, lead=0):
    """t as dtype, `lead` elements behind an aligned place, a unit of 16 bytes of NaNs between its rows and around them."""
    unit = 16 // dtype.itemsize
    rows, cols = t.shape
    step = -(-cols // unit) * unit + unit if lead == 0 and cols % unit == 0 else cols + unit
    flat = torch.full((2 * unit + lead + rows * step,), NAN, dtype=dtype, device="cuda")
    out = flat[unit + lead:unit + lead + rows * step].view(rows, step)[:, :cols]
    return out.copy_(t)


class Guarded:
    """Room for an output, three columns and a row more than it has, of a value that no result here is."""
    MARK = 0.6875

    def __init__(self, rows, cols, dtype):
        self.shape, self.all = (rows, cols), torch.full((rows + 1, cols + 3), self.MARK, dtype=dtype, device="cuda")
        self.stride, self.at = cols + 3, self.all.data_ptr()

    def take(self):
        rows, cols = self.shape
        assert (self.all[:, cols:] == self.MARK).all() and (self.all[rows:] == self.MARK).all()
        return self.all[:rows, :cols]


def act(z, name):
    return z if name == "none" else z.clamp(min=0)


def rounded(t, dtype):
    """Whole numbers (as float64) rounded to dtype."""
    assert t.abs().max() < 2 ** 24 * 32 and torch.equal(t.float().double(), t)
    return t.float().to(dtype)


def exactly(got, want, what):
    assert got.dtype == want.dtype and got.shape == want.shape, what
    wrong = got != want
    assert not wrong.any(), "%s: %d of %d differ, first at %s: %s, not %s" % (
        what, wrong.sum(), wrong.numel(), wrong.nonzero()[0].tolist(), got[wrong][0].item(), want[wrong][0].item())


@pytest.mark.parametrize("case", FORWARD, ids=lambda c: "-".join(map(str, c)).replace(" ", "-"))
def test_forward(case):
    dtype, (rows, k, k2, n, lead) = TYPES[case[0]], case[1:6]
    assert k + k2 <= 600  # gates stay at 1024 - 600 and beyond
    for i, name in enumerate(ACTS):
        d = Draw(i)
        x, w = d.whole(-1, 1, rows, k + k2), d.whole(-1, 1, 2 * n, k + k2)
        b = torch.cat([d.one_of([-1024, 1024], n), d.whole(-3, 3, n)])
        z = x.double() @ w.double().t() + b
        y = act(z[:, :n], name) * z[:, n:]
        a, a2 = among_nans(x[:, :k], dtype, lead), among_nans(x[:, k:], dtype, lead) if k2 else None
        c, bias = among_nans(w, dtype), b.to(dtype)
        got, pre = gated(a, c, bias, act=name, x2=a2, save_pre=True)
        exactly(got, rounded(y, dtype), name)
        exactly(pre, rounded(z, dtype), name + " pre")
        room, pre_room = Guarded(rows, n, dtype), Guarded(rows, 2 * n, dtype)
        for pre in (pre_room, None):
            args = operators._GatedArgs(a.data_ptr(), 0 if a2 is None else a2.data_ptr(), c.data_ptr(), bias.data_ptr(), room.at, pre.at if pre else None, rows,
                                        a.stride(0) if rows > 1 else k, a2.stride(0) if k2 else 0, c.stride(0), room.stride, pre.stride if pre else 0,
                                        n, k, k2, operators._TYPES[dtype], operators.ACTIVATIONS[name])
            room.all.fill_(Guarded.MARK)
            operators._check(operators._load().massive_gated(ctypes.byref(args), operators._stream(0)))
            exactly(room.take(), rounded(y, dtype), name + " into a larger array")
        exactly(pre_room.take(), rounded(z, dtype), name + " pre into a larger array")


@pytest.mark.parametrize("case", GRADIENTS, ids=lambda c: "-".join(map(str, c[:7])))
def test_gradients(case):
    dtype, (rows, k, k2, n, lead), ask = TYPES[case[0]], case[1:6], case[6]
    lib = operators._load()
    for i, name in enumerate(ACTS):
        d = Draw(i)
        x, w, dy = d.whole(-1, 1, rows, k + k2), d.whole(-1, 1, 2 * n, k + k2), d.whole(-2, 2, rows, n)
        # multiples of 32 with at most 3 bits, so that dy times them is exact in bf16, and the other half's are small
        pre = torch.cat([d.one_of([-256, -192, -128, 128, 160, 192, 256], rows, n), d.whole(-3, 3, rows, n)], 1)
        g, u, wide = pre[:, :n].double(), pre[:, n:].double(), dy.double()
        dz = torch.cat([wide * u * ((g > 0) if name != "none" else 1), wide * act(g, name)], 1)
        dx, dw, db = dz @ w.double(), dz.t().contiguous() @ x.double(), dz.sum(0)
        want = {"x": rounded(dx[:, :k], dtype), "2": rounded(dx[:, k:], dtype) if k2 else None, "w": rounded(dw, dtype), "b": rounded(db, dtype)}
        a, a2 = among_nans(x[:, :k], dtype, lead), among_nans(x[:, k:], dtype, lead) if k2 else None
        c, e, p = among_nans(w, dtype), among_nans(dy, dtype), among_nans(pre, dtype)
        got = gated_backward(e, a, c, p, name, a2, bias="b" in ask, need_dx="x" in ask, need_dx2="2" in ask, need_dw="w" in ask)
        for what, t in zip("x2wb", got):
            assert (t is not None) == (what in ask)
            if t is not None:
                exactly(t, want[what], "%s: d%s" % (name, what))
        room = {what: Guarded(*shape, dtype) if what in ask else None
                for what, shape in (("x", (rows, k)), ("2", (rows, k2)), ("w", (2 * n, k + k2)), ("b", (1, 2 * n)))}
        at = {what: r.at if r else None for what, r in room.items()}
        stride = {what: r.stride if r else 0 for what, r in room.items()}
        args = operators._GatedGrads(e.data_ptr(), p.data_ptr(), a.data_ptr(), a2.data_ptr() if k2 else None, c.data_ptr(), at["x"], at["2"], at["w"], at["b"],
                                     rows, e.stride(0), p.stride(0), a.stride(0), a2.stride(0) if k2 else 0, c.stride(0), stride["x"], stride["2"], stride["w"],
                                     n, k, k2, operators._TYPES[dtype], operators.ACTIVATIONS[name])
        need = ctypes.c_int64()
        operators._check(lib.massive_gated_workspace(ctypes.byref(args), ctypes.byref(need)))
        work = torch.full((need.value + 256,), 255, dtype=torch.uint8, device="cuda")  # NaNs in both types
        operators._check(lib.massive_gated_backward(ctypes.byref(args), work.data_ptr(), need.value, operators._stream(0)))
        for what, r in room.items():
            if r:
                t = r.take()
                exactly(t[0] if what == "b" else t, want[what], "%s: d%s into a larger array" % (name, what))
        assert (work[need.value:] == 255).all()
