"""Which form the mean's gradient takes, seen by its workspace: none for the one launch in which a source adds up its list
alone, which many edges of few sources make long (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2410_22697_amd import massive, operators

pytestmark = pytest.mark.skipif(not os.path.exists(massive.LIB_PATH), reason="libmassive.so not built")


def workspace(n, edges, rows, d=128):
    size = ctypes.c_int64()
    b = operators._Block(4096, 4096, n, edges, rows)
    assert operators._load().massive_block_mean_workspace(ctypes.byref(b), d, ctypes.byref(size)) == massive.OK
    return size.value


@pytest.mark.parametrize("n,edges,rows", [(8, 64, 1), (37, 296, 16), (125, 1000, 64), (250, 2000, 256), (250, 2000, 8192), (1, 0, 1)])
def test_short_lists_take_one_launch(n, edges, rows):
    assert workspace(n, edges, rows) == 0


@pytest.mark.parametrize("n,edges,rows", [(37, 296, 1), (125, 1000, 16), (250, 2000, 1), (250, 2000, 64), (250, 2049, 8192), (250, 2000, 8193)])
def test_long_lists_are_sorted(n, edges, rows):
    assert workspace(n, edges, rows) > 0
