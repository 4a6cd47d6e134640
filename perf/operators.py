"""The operators of a training step on sampled minibatches, as cases that can be timed.

  rows    rows written to a table in 8 or 4 bits (`pack_rows`) and rows read back from it (`unpack_rows`)
  mean    the mean over each row's sampled neighbours (`block_mean`) and its gradient (`block_mean_backward`)
  linear  act([x | x2] W^T + b) + residual (`linear`) and its gradients (`linear_backward`)
  adamw   an AdamW step over all of a model's tensors (`AdamW.step`), states in 32 or 8 bits

`run` computes them with elementary torch operations in 32 bits, or, where `own` is true, through the library's
entry points. Sizes are those of this repository's workloads (feature widths 64, 100 and 128, batches of 16 to
4096 seeds, frontiers of up to 854K rows, partitions of up to 15.6M nodes) with hidden widths of 256 and 1024.
"""
import math

import torch

own = False

GELU, SILU = "gelu", "silu"


def listed():
    return [
        # a serving request: a few embeddings written to the cache, a small frontier read from it
        _rows("rows_serve_8", 170_000, 16, 1500, 128, 8, 0, "f32", "f32"),
        # a minibatch's embeddings pushed to a cache of every node's (its offsets pass 32 bits), the next one's pulled
        _rows("rows_push_pull_8", 15_578_155, 110_000, 242_000, 256, 8, 0, "bf16", "bf16"),
        # feature rows of an odd width in 4 bits, groups of 32 with a ragged last one, a stress minibatch's frontier
        _rows("rows_stress_4", 1_599_230, 86_016, 854_001, 100, 4, 32, "f32", "f32"),
        # a serving request's first hop
        _mean("mean_serve", 16, 15, 250, 128, "f32", "f32", False),
        # the last hop of a papers-sized minibatch, its features held in 8 bits
        _mean("mean_packed_8", 110_000, 5, 242_000, 128, "q8", "f32", False),
        # the gradient through the last hop of a papers-sized minibatch, hidden width 256
        _mean("mean_backward", 110_000, 5, 242_000, 256, "f32", "f32", True),
        # a serving request through one layer: 16 seeds, their own rows and their neighbours' means
        _linear("linear_serve_f32", 16, 128, 128, 256, "f32", "relu", True, False, False),
        # the first layer over a papers-sized frontier
        _linear("linear_layer_bf16", 242_000, 128, 128, 256, "bf16", "relu", True, False, False),
        # gradients of a wide layer
        _linear("linear_wide_backward_bf16", 110_000, 128, 0, 1024, "bf16", GELU, True, False, True),
        # gradients of the classifier in 32 bits: an odd number of rows and of classes
        _linear("linear_classes_backward_f32", 16_391, 256, 256, 47, "f32", "none", True, False, True),
        # the weights of a three-layer model, one step
        _adamw("adamw_model", 9, 131_072, "f32", "f32", 32),
        # a model with an embedding for each of a partition's own nodes, states in 8 bits
        _adamw("adamw_embeddings_8", 12, 160_000_000, "f32", "f32", 8),
    ]


def draw(rng):
    """One more case between the smallest and the largest listed ones."""
    def spread(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    op = rng.choice(["rows", "rows", "mean", "mean", "mean", "linear", "linear", "linear", "adamw", "adamw"])
    if op == "rows":
        d, bits = rng.choice([spread(1, 256), rng.choice([64, 100, 128, 256])]), rng.choice([8, 4])
        reads = min(spread(1, 900_000), 80_000_000 // max(d, 16))
        return _rows(None, spread(100, 8_000_000), min(spread(1, 200_000), 25_000_000 // max(d, 16)), reads, d, bits,
                     rng.choice([0, 0, 16, 32, 64, 128]), rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"]))
    if op == "mean":
        n, fanout = spread(1, 200_000), rng.randint(1, 30)
        d = rng.choice([spread(4, 256), rng.choice([64, 100, 128, 256])])
        n = min(n, max(1, 140_000_000 // (fanout * max(d, 32))))
        out = rng.choice(["f32", "f32", "bf16"])
        backward = rng.random() < 0.5
        x = out if backward else rng.choice([out, "q8", "q4"])
        return _mean(None, n, fanout, n + spread(1, 1 + 3 * n), d, x, out, backward)
    if op == "linear":
        dtype = rng.choice(["f32", "bf16", "bf16"])
        k, k2, n = spread(8, 600), rng.choice([0, -1, -1]), spread(1, 1100)
        k2 = k if k2 else 0
        rows = min(spread(1, 242_000), int((2.8e10 if dtype == "bf16" else 1e10) / (2 * (k + k2) * n)) + 1,
                   240_000_000 // max(k + k2, n))
        backward = rng.random() < 0.5
        return _linear(None, rows, k, k2, n, dtype, rng.choice(["none", "relu", "relu", GELU, SILU]), rng.random() < 0.8,
                       not backward and rng.random() < 0.5, backward)
    return _adamw(None, spread(1, 400), spread(1000, 100_000_000), rng.choice(["f32", "f32", "bf16"]),
                  rng.choice(["f32", "bf16"]), rng.choice([32, 8]))


def _named(name, **case):
    return case if name is None else dict(name=name, **case)


def _rows(name, table, writes, reads, d, bits, group, src, dst):
    return _named(name, op="rows", table=table, writes=min(writes, table), reads=reads, d=d, bits=bits, group=group, src=src, dst=dst)


def _mean(name, n, fanout, rows, d, x, out, backward):
    return _named(name, op="mean", n=n, fanout=fanout, rows=rows, d=d, x=x, out=out, backward=backward)


def _linear(name, rows, k, k2, n, dtype, act, bias, residual, backward):
    return _named(name, op="linear", rows=rows, k=k, k2=k2, n=n, dtype=dtype, act=act, bias=bias, residual=residual, backward=backward)


def _adamw(name, tensors, total, param, grad, bits):
    return _named(name, op="adamw", tensors=tensors, total=total, param=param, grad=grad, bits=bits)


_SIZE = {"f32": 4, "bf16": 2}
_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _ceil(a, b):
    return -(-a // b)


def _row_bytes(d, bits, group):
    """Codes padded to four bytes, then each group's step (8 bits) or lowest value and step (4 bits) as f32."""
    groups = _ceil(d, group) if group else 1
    return 4 * _ceil(d * bits, 32) + 4 * groups * (1 if bits == 8 else 2)


def _x_bytes(case):
    """Bytes of one of block_mean's rows."""
    if case["x"] in _SIZE:
        return case["d"] * _SIZE[case["x"]]
    return _row_bytes(case["d"], int(case["x"][1]), 0)


def work(case):
    op = case["op"]
    if op == "rows":
        rb = _row_bytes(case["d"], case["bits"], case["group"])
        return {"bytes": case["writes"] * (case["d"] * _SIZE[case["src"]] + rb + 4) + case["reads"] * (case["d"] * _SIZE[case["dst"]] + rb + 4),
                "flops": 4 * (case["writes"] + case["reads"]) * case["d"]}
    if op == "mean":
        edges = _edges(case)
        index = 4 * (edges + case["n"] + 1)
        out = case["n"] * case["d"] * _SIZE[case["out"]]
        if case["backward"]:
            return {"bytes": out + index + case["rows"] * case["d"] * _SIZE[case["out"]], "flops": 2 * edges * case["d"]}
        return {"bytes": out + index + min(edges, case["rows"]) * _x_bytes(case), "flops": 2 * edges * case["d"]}
    if op == "linear":
        m, n, k, s = case["rows"], case["n"], case["k"] + case["k2"], _SIZE[case["dtype"]]
        flops = 2 * m * n * k
        if not case["backward"]:
            return {"bytes": s * (m * k + n * k + m * n * (2 if case["residual"] else 1) + (n if case["bias"] else 0)), "flops": flops}
        return {"bytes": s * (2 * m * k + 2 * n * k + m * n * (1 if case["act"] == "none" else 2) + (n if case["bias"] else 0)), "flops": 2 * flops}
    n = case["total"]
    states = 16 if case["bits"] == 32 else 4 + 8  # in 8 bits the states are read, written, and returned as values
    return {"bytes": n * (2 * _SIZE[case["param"]] + _SIZE[case["grad"]] + states), "flops": 14 * n}


def _edges(case):
    """Sampled edges: rows take turns of `fanout`, half of it, all of it, one and none."""
    return sum(_LENGTHS[i](case["fanout"]) * ((case["n"] - i + 7) // 8) for i in range(min(8, case["n"])))


# most rows are longer than the fanout and keep `fanout` edges; some are shorter, and one in eight rows is empty
_LENGTHS = [lambda f: f, lambda f: f, lambda f: (f + 1) // 2, lambda f: f, lambda f: 1, lambda f: f, lambda f: f, lambda f: 0]


def _plain_rows(table, case, gen):
    """Rows of a table as they are in use: any codes, steps of around 2^-5."""
    d, bits, group = case["d"], case["bits"], case.get("group", 0)
    groups = _ceil(d, group) if group else 1
    at = 4 * _ceil(d * bits, 32)
    t = torch.randint(0, 256, (table, _row_bytes(d, bits, group)), generator=gen, dtype=torch.uint8, device="cuda")
    if bits == 8:
        t[:, :d] = t[:, :d].clamp(min=1).bitwise_xor(128)  # -127..127
        t[:, d:at] = 0
    else:
        used = _ceil(d, 2)
        t[:, used:at] = 0
        if d % 2:
            t[:, used - 1] &= 15
    p = torch.rand((table, groups * (1 if bits == 8 else 2)), generator=gen, device="cuda") * 0.03 + 0.01
    t[:, at:] = p.view(torch.uint8).view(table, -1)
    return t


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    op = case["op"]
    s = {"case": case}
    if own:
        from paper_2410_22697_amd import operators
        s["lib"] = operators
    if op == "rows":
        s["table"] = _plain_rows(case["table"], case, gen)
        x = normal(case["writes"], case["d"]) * (0.1 + normal(case["writes"], 1).abs())
        s["x"] = (x.relu() if case["bits"] == 4 else x).to(_TYPE[case["src"]])  # 4 bits: values after an activation too
        s["slots"] = torch.randperm(case["table"], generator=gen, device="cuda")[:case["writes"]].to(torch.int32)
        s["index"] = torch.randint(0, case["table"], (case["reads"],), generator=gen, device="cuda", dtype=torch.int32)
        most = min(case["writes"], case["reads"])
        s["index"][:most] = s["slots"][torch.randperm(case["writes"], generator=gen, device="cuda")[:most]]
        if own:
            s["format"] = s["lib"].RowFormat(case["d"], case["bits"], case["group"])
    elif op == "mean":
        n, rows, edges = case["n"], case["rows"], _edges(case)
        lengths = torch.tensor([f(case["fanout"]) for f in _LENGTHS], device="cuda").repeat(_ceil(n, 8))[:n]
        s["indptr"] = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        s["indptr"][1:] = lengths.cumsum(0)
        # neighbours in proportion to their degrees: a few hubs in many rows, most nodes in few
        at = (torch.rand(edges, generator=gen, device="cuda", dtype=torch.float64).square() * rows).to(torch.int64)
        s["indices"] = torch.randperm(rows, generator=gen, device="cuda")[at].to(torch.int32)
        if case["backward"]:
            s["dout"] = normal(n, case["d"]).to(_TYPE[case["out"]])
        elif case["x"] in _TYPE:
            s["x"] = normal(rows, case["d"]).to(_TYPE[case["x"]])
        else:
            s["x"] = _plain_rows(rows, {"d": case["d"], "bits": int(case["x"][1])}, gen)
            if own:
                s["format"] = s["lib"].RowFormat(case["d"], int(case["x"][1]))
    elif op == "linear":
        m, n, k, k2, t = case["rows"], case["n"], case["k"], case["k2"], _TYPE[case["dtype"]]
        s["x"] = normal(m, k).to(t)
        s["x2"] = normal(m, k2).to(t) if k2 else None
        s["w"] = (normal(n, k + k2) / math.sqrt(k + k2)).to(t)
        s["b"] = normal(n).to(t) if case["bias"] else None
        s["residual"] = normal(m, n).to(t) if case["residual"] else None
        if case["backward"]:
            s["dy"] = normal(m, n).to(t)
            s["pre"] = normal(m, n).to(t) if case["act"] != "none" else None  # what the forward pass kept
    else:
        # tensors of spread sizes; each takes whole blocks of 256 in the flat arrays, the rest of its last block is zero
        sizes = _sizes(case)
        starts = [0]
        for z in sizes:
            starts.append(starts[-1] + 256 * _ceil(z, 256))
        spread = (lambda v: v) if starts[-1] == sum(sizes) else (lambda v, live=_live(sizes, starts): v * live)
        s["params"] = spread(normal(starts[-1]) * 0.1).to(_TYPE[case["param"]])
        s["grads"] = spread(normal(starts[-1]) * normal(starts[-1]).abs() * 1e-3).to(_TYPE[case["grad"]])
        s["t"] = 0
        if own:
            views = [s["params"][a:a + z] for a, z in zip(starts, sizes)]
            s["gradients"] = [s["grads"][a:a + z] for a, z in zip(starts, sizes)]
            s["optimizer"] = s["lib"].AdamW(views, state_bits=case["bits"], **_HYPER)
        else:
            s["m"], s["v"] = (_zero_state(starts[-1], case["bits"]) for _ in range(2))
    return s


def _live(sizes, starts):
    live = torch.zeros(starts[-1], device="cuda")
    for a, z in zip(starts, sizes):
        live[a:a + z] = 1
    return live


def _zero_state(n, bits):
    if bits == 32:
        return torch.zeros(n, device="cuda")
    return torch.zeros(n, dtype=torch.int16, device="cuda"), torch.zeros(n // 256, 1, device="cuda")


def _sizes(case):
    """Sizes of a model's tensors: one holds about half of the values, weights the rest, every third is a bias."""
    n, count = case["total"], case["tensors"]
    if count == 1:
        return [n]
    weights = [1.0 if i == 0 else (0.004 if i % 3 == 2 else 1.0 / (count - 1)) for i in range(count)]
    got = [max(1, int(n * w / (2 * sum(weights[1:]) if i else 2))) for i, w in enumerate(weights)]
    got[0] = max(1, got[0] + n - sum(got))
    return got


_HYPER = dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)


# ------------------------------------------------------------------ the passes
def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


def _rows_own(s):
    lib = s["lib"]
    lib.pack_rows(s["x"], s["format"], out=s["table"], slots=s["slots"])
    return lib.unpack_rows(s["table"], s["format"], index=s["index"], dtype=_TYPE[s["case"]["dst"]])


def _mean_own(s):
    lib, case = s["lib"], s["case"]
    if case["backward"]:
        return lib.block_mean_backward(s["dout"], s["indptr"], s["indices"], case["rows"])
    return lib.block_mean(s["x"], s["indptr"], s["indices"], fmt=s.get("format"), dtype=_TYPE[case["out"]])


def _linear_own(s):
    lib, case = s["lib"], s["case"]
    if not case["backward"]:
        return lib.linear(s["x"], s["w"], s["b"], act=case["act"], residual=s["residual"], x2=s["x2"])
    return lib.linear_backward(s["dy"], s["x"], s["w"], act=case["act"], pre=s["pre"], x2=s["x2"], bias=case["bias"])


def _adamw_own(s):
    s["optimizer"].step(s["gradients"])
    return (s["params"], *s["optimizer"].states())


_OWN = {"rows": _rows_own, "mean": _mean_own, "linear": _linear_own, "adamw": _adamw_own}


def _grouped(x, group):
    """x's columns as [rows, groups, group], the last group filled up with its own first value."""
    d = x.shape[1]
    g = group or d
    short = _ceil(d, g) * g - d
    if short:
        x = torch.cat([x, x[:, d - d % g:d - d % g + 1].expand(-1, short)], 1)
    return x.view(x.shape[0], -1, g)


def _rows_encode(x, case):
    d, bits = case["d"], case["bits"]
    x = _grouped(x.float(), case["group"])
    if bits == 8:
        r, lo = x.abs().amax(2, keepdim=True), None
        step = r * (1 / 127)
    else:
        lo = x.amin(2, keepdim=True)
        r = x.amax(2, keepdim=True) - lo
        step = r * (1 / 15)
    some, fine = r >= 2.0 ** -119, torch.isfinite(r)
    inv = torch.where(some & fine, step.reciprocal(), 0.0)
    step = torch.where(fine, torch.where(some, step, 0.0), float("nan"))
    code = ((x if lo is None else x - lo) * inv).round()
    code = (code.clamp(-127, 127) if bits == 8 else code.clamp(0, 15)).view(x.shape[0], -1)[:, :d]
    used = 4 * _ceil(d * bits, 32)
    if bits == 8:
        code = torch.nn.functional.pad(code.to(torch.int8).view(torch.uint8), (0, used - d))
        scales = step
    else:
        code = torch.nn.functional.pad(code.to(torch.uint8), (0, 2 * used - d))
        code = code[:, 0::2] | (code[:, 1::2] << 4)
        scales = torch.cat([lo, step], 2)
    return torch.cat([code, scales.reshape(x.shape[0], -1).view(torch.uint8)], 1)


def _rows_decode(rows, d, bits, group):
    used = 4 * _ceil(d * bits, 32)
    p = rows[:, used:].contiguous().view(torch.float32)
    groups = _ceil(d, group) if group else 1
    if bits == 8:
        code = rows[:, :d].view(torch.int8).float()
        if groups == 1:
            return code * p
        return code * p.repeat_interleave(group, 1)[:, :d]
    code = torch.stack([rows[:, :used] & 15, rows[:, :used] >> 4], 2).view(rows.shape[0], -1)[:, :d].float()
    if groups == 1:
        return p[:, :1] + code * p[:, 1:]
    return p[:, 0::2].repeat_interleave(group, 1)[:, :d] + code * p[:, 1::2].repeat_interleave(group, 1)[:, :d]


def _rows_plain(s):
    case = s["case"]
    s["table"][s["slots"].long()] = _rows_encode(s["x"], case)
    return _rows_decode(s["table"][s["index"].long()], case["d"], case["bits"], case["group"]).to(_TYPE[case["dst"]])


def _mean_plain(s):
    case = s["case"]
    n, edges = case["n"], s["indices"].numel()
    lengths = (s["indptr"][1:] - s["indptr"][:-1]).long()
    of = torch.repeat_interleave(torch.arange(n, device="cuda"), lengths, output_size=edges)
    share = 1.0 / lengths.clamp(min=1).float()[:, None]
    index = s["indices"].long()
    if case["backward"]:
        dx = torch.zeros(case["rows"], case["d"], device="cuda")
        return dx.index_add_(0, index, (s["dout"].float() * share)[of]).to(_TYPE[case["out"]])
    if case["x"] in _TYPE:
        x = s["x"][index].float()
    else:
        x = _rows_decode(s["x"][index], case["d"], int(case["x"][1]), 0)
    return (torch.zeros(n, case["d"], device="cuda").index_add_(0, of, x) * share).to(_TYPE[case["out"]])


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
    q = torch.sigmoid(z)
    return q * (1 + z * (1 - q))


def _linear_in(s, wide):
    """Both outputs' formulas in one width: the plain form's 32 bits, or 64."""
    case = s["case"]
    x = s["x"].to(wide)
    if s["x2"] is not None:
        x = torch.cat([x, s["x2"].to(wide)], 1)
    return case, x, s["w"].to(wide), _TYPE[case["dtype"]]


def _linear_plain(s):
    case, x, w, t = _linear_in(s, torch.float32)
    if not case["backward"]:
        y = x @ w.t()
        if s["b"] is not None:
            y = y + s["b"].float()
        y = _act(y, case["act"])
        return (y if s["residual"] is None else y + s["residual"].float()).to(t)
    dz = s["dy"].float()
    if case["act"] != "none":
        dz = dz * _act_slope(s["pre"].float(), case["act"])
    dx, dw = dz @ w, dz.t() @ x
    k = case["k"]
    return (dx[:, :k].to(t), dx[:, k:].to(t) if case["k2"] else None, dw.to(t), dz.sum(0).to(t) if case["bias"] else None)


def _coded(x, power):
    """Blocks of 256 as 8-bit codes of a square (signed) or fourth power (from zero up) law, and their scales."""
    x = x.view(-1, 256)
    a = x.abs().amax(1, keepdim=True)
    top = 127.0 ** 2 if power == 2 else 255.0 ** 4
    some, fine = a >= (2.0 ** -112 if power == 2 else 2.0 ** -94), torch.isfinite(a)
    scale = a * (1 / top)
    t = x.abs() * torch.where(some & fine, scale.reciprocal(), 0.0)
    if power == 2:
        code = t.sqrt().round().clamp(max=127) * torch.sign(x)
    else:
        code = t.sqrt().sqrt().round().clamp(min=1, max=255) * (t > 0)
    scale = torch.where(fine, torch.where(some, scale, 0.0), float("nan"))
    return torch.where(fine, code, 0.0).to(torch.int16).view(-1), scale


def _decoded(code, scale, power):
    c = code.view(-1, 256).float()
    c = c * c.abs() if power == 2 else (c * c) * (c * c)
    return (c * scale).view(-1)


def _adamw_plain(s):
    bits = s["case"]["bits"]
    (b1, b2), lr = _HYPER["betas"], _HYPER["lr"]
    s["t"] += 1
    g, p = s["grads"].float(), s["params"].float()
    m, v = (s["m"], s["v"]) if bits == 32 else (_decoded(*s["m"], 2), _decoded(*s["v"], 4))
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    p = p * (1 - lr * _HYPER["weight_decay"])
    p = p - (m * (lr / (1 - b1 ** s["t"]))) / (v.sqrt() * (1 / math.sqrt(1 - b2 ** s["t"])) + _HYPER["eps"])
    s["params"].copy_(p)
    if bits == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return s["params"], s["m"], s["v"]
    s["m"], s["v"] = _coded(m, 2), _coded(v, 4)
    return s["params"], _decoded(*s["m"], 2), _decoded(*s["v"], 4)


_PLAIN = {"rows": _rows_plain, "mean": _mean_plain, "linear": _linear_plain, "adamw": _adamw_plain}


# ------------------------------------------------------------- in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"rows": _rows_exact, "mean": _mean_exact, "linear": _linear_exact, "adamw": _adamw_exact}[case["op"]](s)


def _values(rows, d, bits, group):
    """What packed rows stand for: column j's code, times (and from) what its group's floats say."""
    used, j = 4 * _ceil(d * bits, 32), torch.arange(d, device="cuda")
    p = rows[:, used:].contiguous().view(torch.float32).double()
    at = j // (group or d)
    if bits == 8:
        c = rows[:, :d].double()
        return torch.where(c > 127, c - 256, c) * p[:, at]
    c = (rows[:, j // 2].int() >> (4 * (j % 2))) & 15
    return p[:, 2 * at] + c.double() * p[:, 2 * at + 1]


def _rows_exact(s):
    case = s["case"]
    d, group = case["d"], case["group"] or case["d"]
    read = s["index"].long()
    out = _values(s["table"][read], d, case["bits"], case["group"])
    written = torch.full((case["table"],), -1, dtype=torch.int64, device="cuda")
    written[s["slots"].long()] = torch.arange(case["writes"], device="cuda")
    x = s["x"].double()
    stands = torch.empty_like(x)
    for a in range(0, d, group):
        part = x[:, a:a + group]
        lo, hi = part.min(1, keepdim=True)[0], part.max(1, keepdim=True)[0]
        if case["bits"] == 8:
            step = torch.maximum(hi, -lo) / 127
            lo = torch.zeros_like(lo)
        else:
            step = (hi - lo) / 15
        stands[:, a:a + group] = lo + torch.round((part - lo) / step.clamp(min=1e-300)) * step
    fresh = written[read]
    return torch.where((fresh >= 0)[:, None], stands[fresh.clamp(min=0)], out)


def _mean_exact(s):
    case = s["case"]
    d, n = case["d"], case["n"]
    ends = s["indptr"].long()
    lengths = ends[1:] - ends[:-1]
    of = torch.searchsorted(ends[1:].contiguous(), torch.arange(s["indices"].numel(), device="cuda"), right=True)
    index = s["indices"].long()
    total = torch.zeros(case["rows"] if case["backward"] else n, d, dtype=torch.float64, device="cuda")
    for a in range(0, index.numel(), 1 << 20):
        i, j = of[a:a + (1 << 20)], index[a:a + (1 << 20)]
        if case["backward"]:
            total.index_add_(0, j, s["dout"][i].double() / lengths[i][:, None])
        else:
            x = s["x"][j]
            x = x.double() if case["x"] in _TYPE else _values(x, d, int(case["x"][1]), 0)
            total.index_add_(0, i, x / lengths[i][:, None])
    return total


def _linear_exact(s):
    case, x, w, _ = _linear_in(s, torch.float64)
    if not case["backward"]:
        z = torch.matmul(x, w.t().contiguous())
        if s["b"] is not None:
            z += s["b"].double()
        if case["act"] == "relu":
            z = torch.where(z > 0, z, 0.0)
        elif case["act"] == GELU:
            z = z * torch.special.ndtr(z)
        elif case["act"] == SILU:
            z = z / (1 + torch.exp(-z))
        return z if s["residual"] is None else z + s["residual"].double()
    dz = s["dy"].double()
    if s["pre"] is not None:
        z = s["pre"].double()
        if case["act"] == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        elif case["act"] == GELU:
            dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        else:
            e = torch.exp(-z)
            dz = dz * (1 + e + z * e) / (1 + e) ** 2
    dx = torch.matmul(dz, w)
    dw = torch.matmul(dz.t().contiguous(), x)
    k = case["k"]
    return (dx[:, :k], dx[:, k:] if case["k2"] else None, dw, dz.sum(0) if case["bias"] else None)


def _adamw_exact(s):
    """One step from states of zero."""
    (b1, b2), lr = _HYPER["betas"], _HYPER["lr"]
    g, p = s["grads"].double(), s["params"].double()
    m, v = (1 - b1) * g, (1 - b2) * g * g
    p = p * (1 - lr * _HYPER["weight_decay"]) - lr * (m / (1 - b1)) / (torch.sqrt(v / (1 - b2)) + _HYPER["eps"])
    if s["case"]["bits"] == 32:
        return p, m, v

    def held(x, top, root):
        x = x.view(-1, 256)
        a = x.abs().max(1, keepdim=True)[0].clamp(min=1e-300)
        c = torch.round(top * (x.abs() / a) ** (1 / root))
        if root == 4:
            c = torch.where(x > 0, c.clamp(min=1), 0.0)
        return (torch.sign(x) * a * (c / top) ** root).view(-1)
    return p, held(m, 127, 2), held(v, 255, 4)
