"""out and slots of the norm are for packed rows: without a format they are refused, whether or not a tensor requires a
gradient (before any device call; no GPU needed)."""
import os

import pytest
import torch

from paper_2410_22697_amd import RowFormat, massive, rms_norm

pytestmark = pytest.mark.skipif(not os.path.exists(massive.LIB_PATH), reason="libmassive.so not built")
SLOTS, TABLE = torch.arange(6, dtype=torch.int32), torch.zeros(6, 20, dtype=torch.uint8)


@pytest.mark.parametrize("needs", ["", "x", "weight", "residual"])
@pytest.mark.parametrize("grads", [True, False])
def test_without_a_format(needs, grads):
    x, w, r = torch.randn(6, 16).requires_grad_(needs == "x"), torch.ones(16).requires_grad_(needs == "weight"), \
        torch.randn(6, 16).requires_grad_(needs == "residual")
    with torch.set_grad_enabled(grads):
        for more in (dict(slots=SLOTS), dict(out=TABLE), dict(out=TABLE, slots=SLOTS)):
            with pytest.raises(ValueError, match="for packed rows"):
                rms_norm(x, w, residual=r, **more)
        with pytest.raises(ValueError, match="no gradient" if needs and grads else "device"):
            rms_norm(x, w, residual=r, fmt=RowFormat(16), slots=SLOTS, out=TABLE)
