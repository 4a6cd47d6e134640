"""Dropout, the norm and the gated layer on rows whose places pass 32 bits: rows 2^31 elements apart read and written, and
arrays of more than 2^32 elements, against the same rows close together."""
import ctypes

import pytest
import torch

from paper_2410_22697_amd import dropout, dropout_backward, gated, gated_backward, operators, rms_norm, rms_norm_backward

pytestmark = pytest.mark.gpu
FAR, ROWS = 2 ** 31 + 8, 3


@pytest.fixture(scope="module")
def room():
    """Memory for bf16 rows that far apart, for two arrays beside each other in each row (nothing but the rows is touched)."""
    yield torch.empty(2 * FAR + 2 ** 20, dtype=torch.bfloat16, device="cuda")
    torch.cuda.empty_cache()


def far(room, t, at):
    return room.as_strided(t.shape, (FAR, 1), at).copy_(t)


def test_rows_far_apart(room):
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    lib, stream = operators._load(), operators._stream(0)
    for d in (96, 100, 5000):
        x, r = new(ROWS, d), new(ROWS, d)
        fx, fr = far(room, x, 0), far(room, r, 2 ** 16)
        y = room.as_strided((ROWS, d), (FAR, 1), 2 ** 17)
        want = dropout(x, 0.3, 7, 2, residual=r)
        assert torch.equal(dropout(fx, 0.3, 7, 2, residual=fr), want) and torch.equal(dropout_backward(fx, 0.3, 7), dropout_backward(x, 0.3, 7))
        a = operators._DropoutArgs(fx.data_ptr(), fr.data_ptr(), y.data_ptr(), None, ROWS, FAR, FAR, FAR, 7, 0.3, 2, d, 1)
        operators._check(lib.massive_dropout(ctypes.byref(a), stream))
        assert torch.equal(y, want)
        w = new(d)
        want = rms_norm(x, w, residual=r)
        assert all(torch.equal(u, v) for u, v in zip(rms_norm(fx, w, residual=fr), want))
        s = room.as_strided((ROWS, d), (FAR, 1), 2 ** 18)
        a = operators._NormArgs(fx.data_ptr(), fr.data_ptr(), w.data_ptr(), s.data_ptr(), y.data_ptr(), None, None, 0, ROWS, FAR, FAR, FAR, FAR, 1e-6, d, 1)
        operators._check(lib.massive_rms_norm(ctypes.byref(a), stream))
        assert torch.equal(y, want[0]) and torch.equal(s, want[1])
        want = rms_norm_backward(r, x, w, ds=r)
        assert all(torch.equal(u, v) for u, v in zip(rms_norm_backward(fr, fx, w, ds=fr), want))
        need = ctypes.c_int64()
        dw = torch.empty_like(w)
        a = operators._NormGrads(fr.data_ptr(), fx.data_ptr(), w.data_ptr(), fr.data_ptr(), y.data_ptr(), dw.data_ptr(), ROWS, FAR, FAR, FAR, FAR, 1e-6, d, 1)
        operators._check(lib.massive_rms_norm_workspace(ctypes.byref(a), ctypes.byref(need)))
        work = torch.empty(need.value, dtype=torch.uint8, device="cuda")
        operators._check(lib.massive_rms_norm_backward(ctypes.byref(a), work.data_ptr(), need.value, stream))
        assert torch.equal(y, want[0]) and torch.equal(dw, want[1])
    for k, n in ((64, 40), (37, 33)):
        x, w, dy, pre = new(ROWS, k), new(2 * n, k), new(ROWS, n), new(ROWS, 2 * n)
        fx, fdy, fpre = far(room, x, 0), far(room, dy, 2 ** 16), far(room, pre, 2 ** 17)
        want = gated(x, w, save_pre=True)
        assert all(torch.equal(u, v) for u, v in zip(gated(fx, w, save_pre=True), want))
        y, z = room.as_strided((ROWS, n), (FAR, 1), 2 ** 18), room.as_strided((ROWS, 2 * n), (FAR, 1), 2 ** 19)
        a = operators._GatedArgs(fx.data_ptr(), None, w.data_ptr(), None, y.data_ptr(), z.data_ptr(), ROWS, FAR, 0, k, FAR, FAR, n, k, 0, 1, 3)
        operators._check(lib.massive_gated(ctypes.byref(a), stream))
        assert torch.equal(y, want[0]) and torch.equal(z, want[1])
        got, want = gated_backward(fdy, fx, w, fpre), gated_backward(dy, x, w, pre)
        assert all(u is None or torch.equal(u, v) for u, v in zip(got, want))


@pytest.mark.parametrize("k,n", [(8, 1024), (5, 1021)])
def test_more_than_32_bits_of_elements(k, n):
    """2.2 million rows of both halves, on whole numbers that every sum holds exactly (gates far from 0, so that the
    activation is z or 0): dz has over 2^32 elements on either way to dw."""
    rows = 2_200_003
    assert rows * 2 * n > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(k)
    small = lambda low, high, *s: torch.randint(low, high + 1, s, generator=g, device="cuda", dtype=torch.int8)  # noqa: E731
    x, w, dy = small(-1, 1, rows, k).bfloat16(), small(-1, 1, 2 * n, k).bfloat16(), small(-1, 1, rows, n).bfloat16()
    pre = small(-1, 1, rows, 2 * n).bfloat16()
    pre[:, :n].mul_(2).add_(1).mul_(128)  # -128, 128 and 384
    dx, _, dw, db = gated_backward(dy, x, w, pre)
    want_w, want_b = torch.zeros(2 * n, k, dtype=torch.float64, device="cuda"), torch.zeros(2 * n, dtype=torch.float64, device="cuda")
    for a in range(0, rows, 200_000):
        b = slice(a, a + 200_000)
        gate = pre[b, :n].float()
        dz = torch.cat([dy[b].float() * pre[b, n:].float() * (gate > 0), dy[b].float() * gate.clamp(min=0)], 1)
        # products of three values of at most 384 each, sums of 2 n of them: exact in fp32
        assert torch.equal(dx[b], (dz @ w.float()).bfloat16())
        want_w += dz.double().t().contiguous() @ x[b].double()
        want_b += dz.double().sum(0)
    # (of the gates' sums every term is a multiple of 128)
    assert want_w[n:].abs().max() < 2 ** 31 and want_w[:n].abs().max() < 2 ** 24
    assert torch.equal(dw, want_w.float().bfloat16()) and torch.equal(db, want_b.float().bfloat16())
    del dy, dx, dz
    y, z = gated(x, w, pre[0].contiguous() * 8, save_pre=True)
    assert torch.equal(z[-1000:], (x[-1000:].float() @ w.float().t() + pre[0].float() * 8).bfloat16())
    tail, head = gated(x[-1000:], w, pre[0].contiguous() * 8), gated(x[:1000], w, pre[0].contiguous() * 8)
    assert torch.equal(y[-1000:], tail) and torch.equal(y[:1000], head)
