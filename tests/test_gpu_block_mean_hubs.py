"""The mean's gradient where few sources have all of the edges, on both sides of where its form changes."""
import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2410_22697_amd import block_mean_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,most,rows", [(1, 128, 1), (1, 129, 1), (8, 16, 1), (9, 15, 1), (16, 2000, 2), (250, 8, 244), (250, 8, 245), (2048, 1, 256),
                                         (2048, 1, 255), (300, 40, 3)])
def test_few_sources(n, most, rows, dtype):
    """A sum of c products rounds twice for each at most, the share once."""
    rng = np.random.default_rng(n + rows)
    indptr = (np.arange(n + 1) * most).astype(np.int32)
    indices = (rng.random(indptr[-1]) ** 2 * rows).astype(np.int32)
    dout = torch.from_numpy(rng.standard_normal((n, 36)).astype(np.float32)).to(dtype).cuda()
    got = block_mean_backward(dout, torch.from_numpy(indptr).cuda(), torch.from_numpy(indices).cuda(), rows).double().cpu().numpy()
    want, mag, count = plain.mean_backward(dout.double().cpu().numpy(), indptr, indices, rows)
    slack = (2 * count[:, None] + 3) * plain.EPS * mag
    assert np.all(np.abs(got - want) <= slack + (plain.BF / 2 * (np.abs(want) + slack) if dtype == torch.bfloat16 else 0.0))
