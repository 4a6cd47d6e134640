"""Plain forms, in 64 bits, of what stands between a training step's layers, and their gradients. numpy only."""
import numpy as np

import plain_operators as plain


def philox(c0, c1, c2, c3, key):
    """Philox4x32-10 of counter words (arrays of uint64 below 2^32) under a 64-bit key: four words."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, np.uint64) + np.zeros(np.broadcast_shapes(*map(np.shape, (c0, c1, c2, c3))), np.uint64) for v in (c0, c1, c2, c3)]
    k0, k1 = key % 2 ** 32, key // 2 ** 32
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    return c


def kept(rows, d, p, seed, draw):
    words = philox(np.arange(-(-d // 4))[None, :], np.arange(rows)[:, None], draw, 0, seed % 2 ** 64)
    words = np.stack(words, 2).reshape(rows, -1)[:, :d]
    return words >= np.uint64(round(p * 2 ** 32))


def norm(s, weight, eps):
    """(y, n, r) of rows of s."""
    with np.errstate(all="ignore"):
        r = 1 / np.sqrt((s * s).mean(1, keepdims=True) + eps)
        n = s * r
        return n * weight, n, r


def norm_backward(dy, s, weight, eps, ds):
    """(dx, dweight, what the rounding of their sums goes by)."""
    _, n, r = norm(s, weight, eps)
    g = dy * weight
    dx = r * (g - n * (g * n).mean(1, keepdims=True)) + ds
    return dx, (dy * n).sum(0), r * (np.abs(g) + np.abs(n) * np.abs(g * n).mean(1, keepdims=True)) + np.abs(ds), np.abs(dy * n).sum(0)


def gated(x, w, b, act):
    """(y, pre) of rows of x."""
    z = x @ w.T + b
    n = w.shape[0] // 2
    return plain.act(z[:, :n], act) * z[:, n:], z


def gated_dz(dy, pre, act):
    n = dy.shape[1]
    g, u = pre[:, :n], pre[:, n:]
    return np.concatenate([dy * u * plain.slope(g, act), dy * plain.act(g, act)], 1)
