"""The gradient of a layer's bias alone: it needs neither inputs nor weights."""
import ctypes

import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2410_22697_amd import operators

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def wide(t):
    return t.detach().double().cpu().numpy()


def make(rows, k, n, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    return new(rows, n), (2 * new(rows, n).float()).to(dtype), new(rows, k), new(n, k)


@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 3, 1), (70, 40, 33), (5_003, 12, 300), (9_001, 300, 70)])
def test_bias_gradient_without_inputs(act, dtype, size):
    """Only dbias asked for, and no x and no w given."""
    rows, k, n = size
    t = TYPES[dtype]
    dy, pre, _, _ = make(rows, k, n, t, n)
    db = torch.full((n + 2,), 7.0, device="cuda").to(t)
    g = operators._LinearGrads(dy=dy.data_ptr(), pre=None if act == "none" else pre.data_ptr(), dbias=db.data_ptr(), rows=rows,
                               dy_stride=n, pre_stride=n, x_stride=k, w_stride=k, n=n, k=k,
                               type=operators._TYPES[t], act=operators.ACTIVATIONS[act])
    lib, need = operators._load(), ctypes.c_int64()
    assert lib.massive_linear_workspace(ctypes.byref(g), ctypes.byref(need)) == 0
    work = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    rc = lib.massive_linear_backward(ctypes.byref(g), work.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream)
    assert rc == 0, lib.massive_last_error(None)
    slope = 1.0 if act == "none" else plain.slope(wide(pre), act)
    dz = wide(dy) * slope
    slack = (act == "gelu") * (np.abs(wide(dy)) * 4e-7 * (1 + np.abs(wide(pre)))).sum(0) + (rows + 2) * plain.EPS * np.abs(dz).sum(0)
    want, half = dz.sum(0), plain.BF / 2 if dtype == "bf16" else 0.0
    assert np.all(np.abs(wide(db)[:n] - want) <= slack + half * (np.abs(want) + slack))
    assert torch.all(db[n:] == 7)
