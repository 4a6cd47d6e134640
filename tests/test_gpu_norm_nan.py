"""A NaN in a row of the norm: the whole row is NaN, for any eps (0 among them), and no other row."""
import pytest
import torch

from paper_2410_22697_amd import RowFormat, rms_norm, rms_norm_backward, unpack_rows

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-6, 1e30])
@pytest.mark.parametrize("d", [3, 200, 1500, 5000, 20_000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_with_a_nan(dtype, d, eps):
    g = torch.Generator(device="cuda").manual_seed(d)
    clean, dy, ds = (torch.randn(9, d, generator=g, device="cuda").to(TYPES[dtype]) for _ in range(3))
    x = clean.clone()
    x[1, 0], x[3, d - 1], x[4, d // 2] = NAN, NAN, NAN
    x[5, 0], x[5, d - 1] = INF, NAN
    x[6] = 0
    x[6, 1] = NAN
    x[7] = NAN
    bad = torch.tensor([1, 3, 4, 5, 6, 7], device="cuda")
    fine = torch.tensor([0, 2, 8], device="cuda")
    w = torch.randn(d, generator=g, device="cuda").to(TYPES[dtype])
    for weight in (w, None):
        y, want = rms_norm(x, weight, eps), rms_norm(clean, weight, eps)
        assert torch.isnan(y[bad]).all() and torch.equal(y[fine], want[fine])
        # the NaN may come from either of the two that are added
        y, s = rms_norm(clean, weight, eps, residual=x)
        assert torch.isnan(y[bad]).all() and torch.isfinite(y[fine]).all() and torch.equal(torch.isnan(s), torch.isnan(x))
    for bits in (8, 4):
        fmt = RowFormat(d, bits, 16)
        got = unpack_rows(rms_norm(x, w, eps, fmt=fmt), fmt)
        assert torch.isnan(got[bad]).all() and torch.equal(got[fine], unpack_rows(rms_norm(clean, w, eps, fmt=fmt), fmt)[fine])
    dx, dw = rms_norm_backward(dy, x, w, eps, ds)
    want, _ = rms_norm_backward(dy, clean, w, eps, ds)
    assert torch.isnan(dx[bad]).all() and torch.isnan(dw).all() and torch.equal(dx[fine], want[fine])
    assert torch.isfinite(rms_norm_backward(dy[fine], x[fine], w, eps, ds[fine])[1]).all()
