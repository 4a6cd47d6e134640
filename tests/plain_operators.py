"""Plain forms of the operators in 64 bits (and, for what is held in 8 or 4
bits, the formula's own fp32 steps one by one), for the tests. numpy only."""
import numpy as np

F32 = np.float32
EPS = 2.0 ** -24  # half an ulp of fp32 (24 significant bits), relative
BF = 2.0 ** -7    # an ulp of bf16 (8 significant bits), relative: a rounding is half of one off at most


def groups_of(d, group):
    g = group if group and group < d else d
    return [(a, min(d, a + g)) for a in range(0, d, g)]


def pack(x, bits, group):
    """(codes [n, d] int, lo [n, groups], step [n, groups]) of fp32 rows, each operation rounded to fp32."""
    x = np.asarray(x, F32)
    n, d = x.shape
    gs = groups_of(d, group)
    codes, lo, step = np.zeros((n, d), np.int64), np.zeros((n, len(gs)), F32), np.zeros((n, len(gs)), F32)
    with np.errstate(all="ignore"):
        for g, (a, b) in enumerate(gs):
            part = x[:, a:b]
            bad = ~np.isfinite(part).all(1)
            low = part.min(1) if bits == 4 else np.zeros(n, F32)
            r = (np.abs(part).max(1) if bits == 8 else part.max(1) - low).astype(F32)
            bad |= ~np.isfinite(r)
            s = (r * F32(1 / (127 if bits == 8 else 15))).astype(F32)
            inv = (F32(1) / s).astype(F32)
            flat = ~(r >= F32(2.0 ** -119))
            s[flat] = 0
            inv[flat] = 0
            c = np.rint(((part - low[:, None]).astype(F32) * inv[:, None]).astype(F32))
            c[flat | bad] = 0
            codes[:, a:b] = np.clip(c, *((-127, 127) if bits == 8 else (0, 15))).astype(np.int64)
            s[bad] = np.nan
            low = np.where(bad & (bits == 4), F32(np.nan), low)
            lo[:, g], step[:, g] = low, s
    return codes, lo, step


def stand_for(codes, lo, step, group):
    """The values of packed rows, in 64 bits."""
    out = np.zeros(codes.shape)
    for g, (a, b) in enumerate(groups_of(codes.shape[1], group)):
        out[:, a:b] = lo[:, g:g + 1].astype(np.float64) + codes[:, a:b] * step[:, g:g + 1].astype(np.float64)
    return out


def to_bytes(codes, lo, step, bits):
    n, d = codes.shape
    used = 4 * -(-d * bits // 32)
    row = np.zeros((n, used), np.uint8)
    if bits == 8:
        row[:, :d] = codes.astype(np.int8).view(np.uint8)
        floats = step
    else:
        even, odd = codes[:, 0::2].astype(np.uint8), codes[:, 1::2].astype(np.uint8)
        row[:, :even.shape[1]] = even
        row[:, :odd.shape[1]] |= odd << 4
        floats = np.stack([lo, step], 2).reshape(n, 2 * step.shape[1])
    return np.concatenate([row, np.ascontiguousarray(floats.astype(F32)).view(np.uint8).reshape(n, 4 * floats.shape[1])], 1)


def mean(x, indptr, indices):
    """(mean, mean of magnitudes, lengths) in 64 bits; an index outside x is a row of zeros."""
    n, d = len(indptr) - 1, x.shape[1]
    out, mag, lengths = np.zeros((n, d)), np.zeros((n, d)), np.zeros(n, np.int64)
    for i in range(n):
        j = indices[max(indptr[i], 0):min(indptr[i + 1], len(indices))].astype(np.int64)
        lengths[i] = len(j)
        if len(j):
            rows = np.where(((j >= 0) & (j < len(x)))[:, None], x[np.clip(j, 0, len(x) - 1)], 0.0)
            out[i] = rows.sum(0) / len(j)
            mag[i] = np.abs(rows).sum(0) / len(j)
    return out, mag, lengths


def mean_backward(dout, indptr, indices, rows):
    """(dx, sum of magnitudes, entries) in 64 bits."""
    dx, mag, count = np.zeros((rows, dout.shape[1])), np.zeros((rows, dout.shape[1])), np.zeros(rows, np.int64)
    for i in range(len(indptr) - 1):
        j = indices[max(indptr[i], 0):min(indptr[i + 1], len(indices))].astype(np.int64)
        length = len(j)
        j = j[(j >= 0) & (j < rows)]
        if len(j):
            np.add.at(dx, j, dout[i] / length)
            np.add.at(mag, j, np.abs(dout[i]) / length)
            np.add.at(count, j, 1)
    return dx, mag, count


def act(z, name):
    import torch
    t = torch.from_numpy(z)
    if name == "relu":
        return np.where(z > 0, z, 0.0)
    if name == "gelu":
        return (t * torch.special.ndtr(t)).numpy()
    if name == "silu":
        return (t * torch.sigmoid(t)).numpy()
    return z


def slope(z, name):
    import torch
    t = torch.from_numpy(z)
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "gelu":
        return (torch.special.ndtr(t) + t * torch.exp(-t * t / 2) / np.sqrt(2 * np.pi)).numpy()
    if name == "silu":
        q = torch.sigmoid(t)
        return (q * (1 + t * (1 - q))).numpy()
    return np.ones_like(z)


# ------------------------------------------------------------------- AdamW
def blocks(x):
    return np.pad(x, (0, -len(x) % 256)).reshape(-1, 256)


def encode(x, power):
    """(codes, scales) of flat fp32 values, each operation rounded to fp32."""
    b = blocks(np.asarray(x, F32))
    top, least = (127.0 ** 2, 2.0 ** -112) if power == 2 else (255.0 ** 4, 2.0 ** -94)
    with np.errstate(all="ignore"):
        bad = ~np.isfinite(b).all(1)
        a = np.abs(b).max(1)
        scale = (a * F32(1 / top)).astype(F32)
        inv = (F32(1) / scale).astype(F32)
        flat = ~(a >= F32(least))
        scale[flat] = 0
        inv[flat] = 0
        t = (np.abs(b) * inv[:, None]).astype(F32)
        root = np.sqrt(t) if power == 2 else np.sqrt(np.sqrt(t))
        c = np.rint(root)
        if power == 2:
            c = np.minimum(c, 127) * np.sign(b)
        else:
            c = np.where(t > 0, np.clip(c, 1, 255), 0)
        c[bad | flat] = 0
        scale[bad] = np.nan
    return c.astype(np.int64).reshape(-1)[:len(x)], scale


def decode(c, scale, power):
    """fp32 values of codes, the products rounded one by one."""
    s = np.repeat(scale, 256)[:len(c)]
    q = (c * np.abs(c)).astype(F32) if power == 2 else ((c * c).astype(F32) * (c * c).astype(F32)).astype(F32)
    return (q * s).astype(F32)


def adamw(p, g, m, v, t, lr, b1, b2, eps, wd):
    """One step in 64 bits, from fp32 states: (p, m, v)."""
    p, g, m, v = (np.asarray(x, np.float64) for x in (p, g, m, v))
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    p = p * (1 - lr * wd) - lr / (1 - b1 ** t) * m / (np.sqrt(v) / np.sqrt(1 - b2 ** t) + eps)
    return p, m, v


def moments32(g, m, v, b1, b2):
    """The new moments as fp32 rounds them, operation by operation."""
    g, m, v = (np.asarray(x, F32) for x in (g, m, v))
    m = (m * F32(b1)).astype(F32) + (g * F32(1 - b1)).astype(F32)
    v = (v * F32(b2)).astype(F32) + ((g * g).astype(F32) * F32(1 - b2)).astype(F32)
    return m.astype(F32), v.astype(F32)
