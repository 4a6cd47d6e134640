"""A refusal comes before anything is enqueued (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2410_22697_amd import massive, operators
from paper_2410_22697_amd.massive import EINVAL

pytestmark = pytest.mark.skipif(not os.path.exists(massive.LIB_PATH), reason="libmassive.so not built")
P = 4096  # an address that is aligned and never followed


@pytest.mark.parametrize("k,n", [(1 << 20, 1 << 20), (1 << 16, 1 << 15)])
def test_a_layer_too_large_for_its_weights_gradient_is_refused_before_dx(k, n):
    """With dx asked for too, which is refused with the rest rather than enqueued first."""
    for ask in (dict(dw=P), dict(dw=P, dbias=P)):
        a = operators._LinearGrads(dy=P, x=P, w=P, dx=P, rows=4, dy_stride=n, x_stride=k, w_stride=k, dx_stride=k, dw_stride=k,
                                   n=n, k=k, type=0, act=0, **ask)
        assert operators._load().massive_linear_backward(ctypes.byref(a), P, 1 << 62, None) == EINVAL
        assert "too many" in operators._load().massive_last_error(None).decode()
