"""What stands between a training step's layers, as cases that can be timed.

  dropout  residual + dropout(x) with a mask from a counter-based generator, never stored (`dropout`), and its
           gradient (`dropout_backward`)
  norm     the root-mean-square norm of x + residual, in x's type or as packed rows (`rms_norm`), and its gradients
           (`rms_norm_backward`)
  gated    act(x Wg^T + bg) * (x Wu^T + bu), weights and biases of both halves below each other (`gated`), and its
           gradients (`gated_backward`)

`run` computes them with elementary torch operations in 32 bits, or, where `own` is true, through the library's
entry points. Sizes are those of this repository's workloads (feature widths 64, 100 and 128, batches of 16 to
4096 seeds, frontiers of up to 854K rows) with hidden widths of 256 and 1024.
"""
import math

import torch

own = False

GELU, SILU = "gelu", "silu"


def listed():
    return [
        # the hidden rows of a few seeds
        _dropout("dropout_seeds", 16, 256, "f32", 0.5, False, False),
        # a residual layer's end over a papers-sized frontier
        _dropout("dropout_residual_bf16", 242_000, 256, "bf16", 0.1, True, False),
        # the gradient through a wide hidden layer's mask
        _dropout("dropout_wide_backward", 110_000, 1024, "f32", 0.5, False, True),
        # a serving request: the rows of 16 seeds before the next layer
        _norm("norm_serve", 16, 256, "f32", True, 0, False),
        # a papers-sized frontier's rows normed and handed to the next layer in 8 bits
        _norm("norm_packed_8", 242_000, 256, "bf16", True, 8, False),
        # a stress minibatch's feature rows, of an odd width
        _norm("norm_stress_f32", 854_001, 100, "f32", False, 0, False),
        # its gradients inside a residual layer
        _norm("norm_backward_bf16", 242_000, 256, "bf16", True, 0, True),
        # a serving request through one gated layer
        _gated("gated_serve_bf16", 16, 256, 0, 1024, "bf16", SILU, False, False),
        # a gated layer on a papers-sized frontier's own rows and their neighbours' means
        _gated("gated_layer_bf16", 110_000, 128, 128, 1024, "bf16", SILU, True, False),
        # the gradients of one
        _gated("gated_backward_bf16", 110_000, 256, 0, 1024, "bf16", SILU, True, True),
        # an odd number of rows, features and outputs in 32 bits
        _gated("gated_odd_f32", 16_391, 100, 100, 323, "f32", GELU, True, False),
        _gated("gated_odd_backward_f32", 16_391, 100, 100, 323, "f32", GELU, True, True),
    ]


def draw(rng):
    """One more case between the smallest and the largest listed ones."""
    def spread(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    op = rng.choice(["dropout", "norm", "gated"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    backward = rng.random() < 0.5
    if op == "dropout":
        d = rng.choice([spread(1, 1100), rng.choice([64, 100, 128, 256, 1024])])
        rows = min(spread(1, 900_000), 110_000_000 // max(d, 16))
        return _dropout(None, rows, d, dtype, rng.choice([0.1, 0.5, round(rng.uniform(0.01, 0.9), 3)]), not backward and rng.random() < 0.5, backward)
    if op == "norm":
        d = rng.choice([spread(1, 4096), rng.choice([64, 100, 128, 256, 1024])])
        rows = min(spread(1, 900_000), 80_000_000 // max(d, 16))
        # one or a few columns leave nothing of the norm's own gradient but rounding: there the residual's is added to it
        return _norm(None, rows, d, dtype, d < 16 or rng.random() < 0.7, 0 if backward else rng.choice([0, 0, 8]), backward)
    k, n = spread(8, 600), spread(1, 1100)
    k2 = rng.choice([0, 0, k])
    rows = min(spread(1, 242_000), int((1.1e11 if dtype == "bf16" else 2e10) / (4 * (k + k2) * n)) + 1, 110_000_000 // max(k + k2, n))
    return _gated(None, rows, k, k2, n, dtype, rng.choice(["none", "relu", GELU, SILU, SILU]), rng.random() < 0.5, backward)


def _named(name, **case):
    return case if name is None else dict(name=name, **case)


def _dropout(name, rows, d, dtype, p, residual, backward):
    return _named(name, op="dropout", rows=rows, d=d, dtype=dtype, p=p, residual=residual, backward=backward)


def _norm(name, rows, d, dtype, residual, bits, backward):
    return _named(name, op="norm", rows=rows, d=d, dtype=dtype, residual=residual, bits=bits, backward=backward)


def _gated(name, rows, k, k2, n, dtype, act, bias, backward):
    return _named(name, op="gated", rows=rows, k=k, k2=k2, n=n, dtype=dtype, act=act, bias=bias, backward=backward)


_SIZE = {"f32": 4, "bf16": 2}
_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-6


def work(case):
    m, s = case["rows"], _SIZE[case["dtype"]]
    if case["op"] == "dropout":
        return {"bytes": s * m * case["d"] * (3 if case["residual"] else 2), "flops": 2 * m * case["d"]}
    if case["op"] == "norm":
        d = case["d"]
        if case["backward"]:  # dy, s and ds read, the gradients written
            return {"bytes": s * (m * d * (4 if case["residual"] else 3) + 2 * d), "flops": 10 * m * d}
        # x and residual read; the sum and the norm written, packed rows read again as bf16 values
        y = m * (4 * -(-d // 4) + 4) * 2 + 2 * m * d if case["bits"] else s * m * d
        return {"bytes": s * (m * d * (3 if case["residual"] else 1) + d) + y, "flops": 5 * m * d}
    n, k = case["n"], case["k"] + case["k2"]
    flops = 4 * m * n * k
    if case["backward"]:  # dy, both halves' arguments, x and weights read; the gradients written
        return {"bytes": s * (3 * m * n + 2 * m * k + 4 * n * k + (2 * n if case["bias"] else 0)), "flops": 2 * flops}
    return {"bytes": s * (m * k + 2 * n * k + m * n + (2 * n if case["bias"] else 0)), "flops": flops}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = _TYPE[case["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    s = {"case": case}
    if own:
        from paper_2410_22697_amd import operators
        s["lib"] = operators
    if case["op"] == "dropout":
        s["x"] = normal(case["rows"], case["d"]).to(t)
        s["residual"] = normal(case["rows"], case["d"]).to(t) if case["residual"] else None
        # a key of 64 bits for the step, a number for the layer
        s["key"], s["layer"] = (seed * 0x9E3779B97F4A7C15 + 0x1234567) % 2 ** 64, seed % 7
    elif case["op"] == "norm":
        m, d = case["rows"], case["d"]
        s["x"] = (normal(m, d) * (0.1 + normal(m, 1).abs())).to(t)  # rows of unlike size
        s["weight"] = (1 + 0.1 * normal(d)).to(t)
        if case["backward"]:
            s["dy"] = normal(m, d).to(t)
            s["ds"] = normal(m, d).to(t) if case["residual"] else None
        else:
            s["residual"] = normal(m, d).to(t) if case["residual"] else None
            if own:
                s["format"] = s["lib"].RowFormat(d, case["bits"]) if case["bits"] else None
    else:
        m, n, k, k2 = case["rows"], case["n"], case["k"], case["k2"]
        s["x"] = normal(m, k).to(t)
        s["x2"] = normal(m, k2).to(t) if k2 else None
        s["w"] = (normal(2 * n, k + k2) / math.sqrt(k + k2)).to(t)
        s["b"] = normal(2 * n).to(t) if case["bias"] else None
        if case["backward"]:
            s["dy"] = normal(m, n).to(t)
            s["pre"] = normal(m, 2 * n).to(t)  # what the forward pass kept
    return s


# ------------------------------------------------------------------ the passes
def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


def _dropout_own(s):
    lib, case = s["lib"], s["case"]
    if case["backward"]:
        return lib.dropout_backward(s["x"], case["p"], s["key"], draw=s["layer"])
    return lib.dropout(s["x"], case["p"], s["key"], draw=s["layer"], residual=s["residual"])


def _norm_own(s):
    lib, case = s["lib"], s["case"]
    if case["backward"]:
        return lib.rms_norm_backward(s["dy"], s["x"], s["weight"], eps=_EPS, ds=s["ds"])
    got = lib.rms_norm(s["x"], s["weight"], eps=_EPS, residual=s["residual"], fmt=s["format"])
    if not case["bits"]:
        return got
    table, total = got if case["residual"] else (got, None)
    return lib.unpack_rows(table, s["format"], dtype=torch.bfloat16), total


def _gated_own(s):
    lib, case = s["lib"], s["case"]
    if case["backward"]:
        return lib.gated_backward(s["dy"], s["x"], s["w"], s["pre"], act=case["act"], x2=s["x2"], bias=case["bias"])
    return lib.gated(s["x"], s["w"], s["b"], act=case["act"], x2=s["x2"])


_OWN = {"dropout": _dropout_own, "norm": _norm_own, "gated": _gated_own}

_LOW = 0xFFFFFFFF


def _philox(c, key):
    """Philox4x32-10 of four counter words (tensors of int64, below 2^32) under a 64-bit key."""
    k0, k1 = key & _LOW, key >> 32
    c0, c1, c2, c3 = c
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # 64 bits; the shift's sign is cut off below
        c0, c1, c2, c3 = ((b >> 32) & _LOW) ^ c1 ^ k0, b & _LOW, ((a >> 32) & _LOW) ^ c3 ^ k1, a & _LOW
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    return c0, c1, c2, c3


def _dropout_plain(s):
    """Column j of row i is kept if word j % 4 of the generator at (j / 4, i, layer, 0) is at least p 2^32."""
    case, x = s["case"], s["x"]
    m, d = x.shape
    j, i = torch.arange(-(-d // 4), device="cuda"), torch.arange(m, device="cuda")[:, None]
    zero = torch.zeros(m, j.numel(), dtype=torch.int64, device="cuda")
    words = torch.stack(_philox((zero + j, zero + i, zero + s["layer"], zero), s["key"]), 2).view(m, -1)[:, :d]
    y = torch.where(words >= round(case["p"] * 2 ** 32), x.float() * (1 / (1 - case["p"])), 0.0)
    return (y if s["residual"] is None else y + s["residual"].float()).to(x.dtype)


def _packed_8(y):
    """A row's codes of 8 bits and its step, and the values that they stand for."""
    r = y.abs().amax(1, keepdim=True)
    step = r * (1 / 127)
    inv = torch.where(r >= 2.0 ** -119, step.reciprocal(), 0.0)
    code = (y * inv).round().clamp(-127, 127).to(torch.int8)
    return (code.float() * torch.where(r >= 2.0 ** -119, step, 0.0)).to(torch.bfloat16)


def _norm_plain(s):
    case, t, w = s["case"], s["x"].dtype, s["weight"].float()
    x = s["x"].float()
    if not case["backward"]:
        if s["residual"] is not None:
            x = x + s["residual"].float()
        y = x * torch.rsqrt(x.square().mean(1, keepdim=True) + _EPS) * w
        y = _packed_8(y) if case["bits"] else y.to(t)
        return (y, x.to(t)) if case["residual"] else (y, None) if case["bits"] else y
    r = torch.rsqrt(x.square().mean(1, keepdim=True) + _EPS)
    dy, n = s["dy"].float(), x * r
    g = dy * w
    dx = r * (g - n * (g * n).mean(1, keepdim=True))
    if s["ds"] is not None:
        dx = dx + s["ds"].float()
    return dx.to(t), (dy * n).sum(0).to(t)


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == GELU:
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z * torch.sigmoid(z) if act == SILU else z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == GELU:
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == SILU:
        q = torch.sigmoid(z)
        return q * (1 + z * (1 - q))
    return torch.ones_like(z)


def _gated_plain(s):
    case, t, n = s["case"], s["x"].dtype, s["case"]["n"]
    x, w = s["x"].float(), s["w"].float()
    if s["x2"] is not None:
        x = torch.cat([x, s["x2"].float()], 1)
    if not case["backward"]:
        z = x @ w.t()
        if s["b"] is not None:
            z = z + s["b"].float()
        return (_act(z[:, :n], case["act"]) * z[:, n:]).to(t)
    dy, g, u = s["dy"].float(), s["pre"][:, :n].float(), s["pre"][:, n:].float()
    dz = torch.cat([dy * u * _act_slope(g, case["act"]), dy * _act(g, case["act"])], 1)
    dx, k = dz @ w, case["k"]
    return (dx[:, :k].to(t), dx[:, k:].to(t) if case["k2"] else None, (dz.t() @ x).to(t), dz.sum(0).to(t) if case["bias"] else None)


_PLAIN = {"dropout": _dropout_plain, "norm": _norm_plain, "gated": _gated_plain}


# ------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"dropout": _dropout_exact, "norm": _norm_exact, "gated": _gated_exact}[case["op"]](s)


def _halves(x, by):
    """The high and the low 32 bits of x (below 2^32) times a constant, from products of 16 bits."""
    b1, b0 = divmod(by, 65536)
    x1, x0 = x // 65536, x % 65536
    low = x0 * b0
    mid = x1 * b0 + low // 65536
    cross = x0 * b1 + mid % 65536
    return x1 * b1 + mid // 65536 + cross // 65536, (cross % 65536) * 65536 + low % 65536


def _dropout_exact(s):
    case, x = s["case"], s["x"].double()
    m, d = x.shape
    kept = torch.empty(m, 4 * -(-d // 4), dtype=torch.bool, device="cuda")
    rows = max(1, (1 << 22) // kept.shape[1])
    for a in range(0, m, rows):
        here = min(rows, m - a)
        v = [torch.arange(kept.shape[1] // 4, device="cuda").repeat(here, 1),
             torch.arange(a, a + here, device="cuda").view(-1, 1).repeat(1, kept.shape[1] // 4),
             torch.full((here, kept.shape[1] // 4), s["layer"], device="cuda"), torch.zeros(here, kept.shape[1] // 4, dtype=torch.int64, device="cuda")]
        for r in range(10):
            k0, k1 = (s["key"] % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (s["key"] // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32
            (h0, l0), (h1, l1) = _halves(v[0], 0xD2511F53), _halves(v[2], 0xCD9E8D57)
            v = [h1 ^ v[1] ^ k0, l1, h0 ^ v[3] ^ k1, l0]
        for q in range(4):
            kept[a:a + here, q::4] = v[q].double() >= case["p"] * 2.0 ** 32
    y = x / (1 - case["p"]) * kept[:, :d]
    return y if s["residual"] is None else y + s["residual"].double()


def _norm_exact(s):
    case, x, w = s["case"], s["x"].double(), s["weight"].double()
    if case["backward"]:
        # through the norm as a quotient: x / q, q^2 = mean of x^2 + eps
        q = torch.sqrt((x * x).sum(1, keepdim=True) / case["d"] + _EPS)
        up = s["dy"].double() * w
        dx = up / q - x * ((up * x).sum(1, keepdim=True) / (case["d"] * q ** 3))
        return dx if s["ds"] is None else dx + s["ds"].double(), (s["dy"].double() * (x / q)).sum(0)
    if s["residual"] is not None:
        x = x + s["residual"].double()
    y = x / torch.sqrt((x * x).sum(1, keepdim=True) / case["d"] + _EPS) * w
    if case["bits"]:
        step = torch.maximum(y.max(1, keepdim=True)[0], -y.min(1, keepdim=True)[0]) / 127
        y = torch.round(y / step.clamp(min=1e-300)) * step
    return (y, x) if case["residual"] else (y, None) if case["bits"] else y


def _gated_exact(s):
    case, n, k = s["case"], s["case"]["n"], s["case"]["k"]
    x = s["x"].double() if s["x2"] is None else torch.cat([s["x"].double(), s["x2"].double()], 1)
    w = s["w"].double()

    def value(z):
        if case["act"] == GELU:
            return z * torch.special.ndtr(z)
        return torch.where(z > 0, z, 0.0) if case["act"] == "relu" else z / (1 + torch.exp(-z)) if case["act"] == SILU else z

    def slope(z):
        if case["act"] == GELU:
            return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        e = torch.exp(-z)
        return torch.where(z > 0, 1.0, 0.0).double() if case["act"] == "relu" else (1 + e + z * e) / (1 + e) ** 2 if case["act"] == SILU else torch.ones_like(z)

    if not case["backward"]:
        g, u = (torch.matmul(x, h.t().contiguous()) for h in (w[:n], w[n:]))
        if s["b"] is not None:
            g, u = g + s["b"][:n].double(), u + s["b"][n:].double()
        return value(g) * u
    dy, g, u = s["dy"].double(), s["pre"][:, :n].double(), s["pre"][:, n:].double()
    dg, du = dy * u * slope(g), dy * value(g)
    dx = torch.matmul(dg, w[:n]) + torch.matmul(du, w[n:])
    dw = torch.cat([torch.matmul(h.t().contiguous(), x) for h in (dg, du)])
    return dx[:, :k], dx[:, k:] if case["k2"] else None, dw, torch.cat([dg.sum(0), du.sum(0)]) if case["bias"] else None
