"""The gated layer's results hang neither on where its arrays lie and on their strides nor (but for the split of dx's sums,
which goes by the columns asked for) on which gradients are asked for: the same bits."""
import pytest
import torch

from paper_2410_22697_amd import gated, gated_backward

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def moved(t, lead, pad):
    """t's values `lead` elements behind an aligned place, rows `pad` elements further apart."""
    if t is None:
        return None
    rows, cols = t.shape
    flat = torch.full((lead + rows * (cols + pad),), float("nan"), dtype=t.dtype, device="cuda")
    out = flat[lead:].view(rows, cols + pad)[:, :cols]
    return out.copy_(t)


def other(got, want):
    """Which results are there and not the wanted bits."""
    return [i for i, (u, v) in enumerate(zip(got, want)) if u is not None and not torch.equal(u, v)]


# inputs in whole units of 16 bytes: one row and few, ragged ends of rows, one part of them and many, one and two inputs,
# outputs in whole units or not and less than one, and more columns than a tile has
SIZES = [(1, 64, 0, 40), (7, 8, 8, 8), (33, 64, 32, 40), (300, 64, 32, 40), (300, 128, 128, 9), (1000, 64, 0, 7), (1001, 40, 24, 70), (5000, 64, 32, 200),
         (9001, 256, 0, 33), (40_003, 128, 0, 64), (700, 256, 64, 130)]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_same_bits(size, dtype):
    rows, k, k2, n = size
    t = TYPES[dtype]
    for i, act in enumerate(("silu", "gelu", "relu", "none")):
        g = torch.Generator(device="cuda").manual_seed(i)
        new = lambda *s: torch.randn(s, generator=g, device="cuda").to(t)  # noqa: E731
        x, x2, w, b, dy, pre = new(rows, k), new(rows, k2) if k2 else None, new(2 * n, k + k2), new(2 * n), new(rows, n), new(rows, 2 * n)
        forward = gated(x, w, b, act=act, x2=x2, save_pre=True)
        want = gated_backward(dy, x, w, pre, act, x2)
        for lead, pad in ((1, 0), (0, 1), (16 // x.element_size(), 3), (3, 5)):
            differs = other(gated(moved(x, lead, pad), moved(w, lead, pad), b, act=act, x2=moved(x2, lead, pad), save_pre=True), forward)
            assert not differs, (act, lead, pad)
            for there in ("x", "x2", "w", "dy", "pre", "all"):
                a = {name: moved(v, lead, pad) if there in (name, "all") else v for name, v in (("x", x), ("x2", x2), ("w", w), ("dy", dy), ("pre", pre))}
                differs = other(gated_backward(a["dy"], a["x"], a["w"], a["pre"], act, a["x2"]), want)
                assert not differs, (act, lead, pad, there)
        for ask in (dict(need_dw=False), dict(bias=False), dict(need_dx=False, need_dx2=False), dict(need_dx=False, need_dx2=False, need_dw=False),
                    dict(need_dx=False, need_dx2=False, bias=False)):
            for xs in ((x, x2), (moved(x, 1, 0), moved(x2, 1, 0))):
                differs = other(gated_backward(dy, xs[0], w, pre, act, xs[1], **ask), want)
                assert not differs, (act, ask)
