"""The norm's gradients of so many rows that a team would have over 64 one after the other (twice the blocks then, each with
a part of dweight), and of rows whose sums are exact: small whole numbers, so that a row lost or added twice shows."""
import pytest
import torch

from paper_2410_22697_amd import rms_norm_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d", [(270_001, 132), (262_145, 129), (17_000_003, 2)])
def test_dweight_counts_every_row_once(rows, d):
    """Rows of 1 and -1 have a mean square of 1 exactly and, without eps, a scale of 1 (the root's error is an ulp at most, and
    the rows' own sum tells it): dweight is then a sum of whole numbers, below 2^24."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    s = torch.randint(0, 2, (rows, d), generator=g, device="cuda", dtype=torch.int8).mul_(2).sub_(1)
    dy = torch.randint(-2, 3, (rows, d), generator=g, device="cuda", dtype=torch.int8)
    _, one = rms_norm_backward(torch.ones(1, d, device="cuda"), torch.ones(1, d, device="cuda"), torch.ones(d, device="cuda"), 0.0)
    r = one[0].item()  # the scale that the kernel has for such rows
    assert abs(r - 1) <= 2.0 ** -22
    _, dw = rms_norm_backward(dy.float(), s.float(), torch.ones(d, device="cuda"), 0.0, need_dx=False)
    want = torch.zeros(d, dtype=torch.int64, device="cuda")
    for a in range(0, rows, 1 << 20):
        want += (s[a:a + (1 << 20)] * dy[a:a + (1 << 20)]).sum(0, dtype=torch.int64)
    assert want.abs().max() < 2 ** 24
    if r == 1:
        assert torch.equal(dw.double(), want.double())
    else:  # every product is rounded once by r, and every sum
        assert (dw.double() - want).abs().max() <= 2 ** -22 * 2 * rows


def test_rows_past_each_teams_width():
    """A row of one wave, of several turns of it and of a block, on either side of each line: dx of rows of 1 and -1 with dy the
    row itself is r (s - s r^2), zero but for the root's error (an ulp, twice) and three roundings, and dweight the rows'
    number, rounded once (a row more or less is 1 in 37)."""
    for t, units in ((torch.float32, 4), (torch.bfloat16, 8), (torch.bfloat16, 4)):
        for width in (64, 128, 256, 512, 1024):
            for d in (width * units - units, width * units, width * units + units):
                s = torch.randint(0, 2, (37, d), device="cuda").mul_(2).sub_(1).to(t)
                dx, dw = rms_norm_backward(s, s, torch.ones(d, device="cuda", dtype=t), 0.0)
                assert torch.allclose(dw.float(), torch.full((d,), 37.0, device="cuda"), rtol=2.0 ** -8, atol=0)
                assert dx.float().abs().max() <= 2.0 ** -20
