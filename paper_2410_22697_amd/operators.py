"""What a training step does with the rows that `Massive` gathers (the
operators of include/massive.h): rows held in few bits, the mean over a sampled
block, a layer, a gated layer, the norm and the dropout between them, and the
step on their weights.

As in the rest of the binding, Python only checks and marshals arguments: every
operator runs in the library's HIP kernels, on the current stream of the
tensors' device, and returns without waiting. Outputs and workspaces come from
torch's allocator. `linear`, `gated`, `rms_norm`, `dropout` and `block_mean`
take part in autograd (once, in reverse: their gradients are not differentiated
again, and tensors with forward-mode tangents are refused), and their gradients
are also there as calls of their own. What a call changes in place counts as changed there: a
backward pass that would read it raises. Wrong arguments raise ValueError here,
or MassiveError where the library refuses them.
"""
import ctypes
import operator
from typing import List, Optional, Sequence, Tuple

import numpy as np
import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable
from torch.autograd.graph import increment_version

from . import massive
from .massive import OK, MassiveError

F32, BF16, PACKED = 0, 1, 2
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
_TYPES = {torch.float32: F32, torch.bfloat16: BF16}

_vp, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class _Format(ctypes.Structure):
    _fields_ = [("d", _i32), ("bits", _i32), ("group", _i32), ("reserved", _i32), ("row_bytes", _i64)]


class _Block(ctypes.Structure):
    _fields_ = [("indptr", _vp), ("indices", _vp), ("n", _i64), ("edges", _i64), ("rows", _i64)]


class _LinearArgs(ctypes.Structure):
    _fields_ = [(f, _vp) for f in ("x", "x_second", "w", "bias", "residual", "y", "pre")] + [("rows", _i64)] + \
        [(f, _i64) for f in ("x_stride", "x_second_stride", "w_stride", "residual_stride", "y_stride", "pre_stride")] + \
        [(f, _i32) for f in ("n", "k", "k_second", "type", "act")]


class _LinearGrads(ctypes.Structure):
    _fields_ = [(f, _vp) for f in ("dy", "pre", "x", "x_second", "w", "dx", "dx_second", "dw", "dbias")] + [("rows", _i64)] + \
        [(f, _i64) for f in ("dy_stride", "pre_stride", "x_stride", "x_second_stride", "w_stride", "dx_stride",
                             "dx_second_stride", "dw_stride")] + \
        [(f, _i32) for f in ("n", "k", "k_second", "type", "act")]


class _DropoutArgs(ctypes.Structure):
    _fields_ = [(f, _vp) for f in ("x", "residual", "y", "seed_at")] + \
        [(f, _i64) for f in ("rows", "x_stride", "residual_stride", "y_stride")] + \
        [("seed", ctypes.c_uint64), ("p", ctypes.c_double), ("draw", ctypes.c_uint32), ("d", _i32), ("type", _i32)]


class _NormArgs(ctypes.Structure):
    _fields_ = [(f, _vp) for f in ("x", "residual", "weight", "sum", "y")] + [("fmt", ctypes.POINTER(_Format)), ("slots", _vp)] + \
        [(f, _i64) for f in ("table_rows", "rows", "x_stride", "residual_stride", "sum_stride", "y_stride")] + \
        [("eps", ctypes.c_double), ("d", _i32), ("type", _i32)]


class _NormGrads(ctypes.Structure):
    _fields_ = [(f, _vp) for f in ("dy", "s", "weight", "ds", "dx", "dweight")] + \
        [(f, _i64) for f in ("rows", "dy_stride", "s_stride", "ds_stride", "dx_stride")] + \
        [("eps", ctypes.c_double), ("d", _i32), ("type", _i32)]


class _GatedArgs(ctypes.Structure):
    _fields_ = [(f, _vp) for f in ("x", "x_second", "w", "bias", "y", "pre")] + [("rows", _i64)] + \
        [(f, _i64) for f in ("x_stride", "x_second_stride", "w_stride", "y_stride", "pre_stride")] + \
        [(f, _i32) for f in ("n", "k", "k_second", "type", "act")]


class _GatedGrads(ctypes.Structure):
    _fields_ = _LinearGrads._fields_


class _AdamwTensor(ctypes.Structure):
    _fields_ = [(f, _vp) for f in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")] + [("n", _i64)]


_ADAMW_ROW = np.dtype([(f, np.uint64) for f in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")] + [("n", np.int64)])


class _AdamwArgs(ctypes.Structure):
    _fields_ = [(f, ctypes.c_double) for f in ("lr", "beta_first", "beta_second", "eps", "weight_decay")] + \
        [("t", _i64)] + [(f, _i32) for f in ("state_bits", "param_type", "grad_type", "reserved")]


_lib = None


def _load():
    global _lib
    if _lib is None:
        lib = massive.load()
        p = ctypes.POINTER
        lib.massive_row_layout.argtypes = [p(_Format), p(_i64), p(_i64)]
        lib.massive_pack_rows.argtypes = [p(_Format), _vp, _i32, _i64, _i64, _vp, _vp, _i64, _vp]
        lib.massive_unpack_rows.argtypes = [p(_Format), _vp, _i64, _vp, _i64, _vp, _i32, _i64, _vp]
        lib.massive_block_mean.argtypes = [p(_Block), _vp, _i32, _i64, p(_Format), _i32, _vp, _i32, _i64, _vp]
        lib.massive_block_mean_workspace.argtypes = [p(_Block), _i32, p(_i64)]
        lib.massive_block_mean_backward.argtypes = [p(_Block), _vp, _i32, _i64, _i32, _vp, _i64, _i64, _vp, _i64, _vp, _i64, _vp]
        lib.massive_linear.argtypes = [p(_LinearArgs), _vp]
        lib.massive_linear_workspace.argtypes = [p(_LinearGrads), p(_i64)]
        lib.massive_linear_backward.argtypes = [p(_LinearGrads), _vp, _i64, _vp]
        lib.massive_dropout.argtypes = [p(_DropoutArgs), _vp]
        lib.massive_rms_norm.argtypes = [p(_NormArgs), _vp]
        lib.massive_rms_norm_workspace.argtypes = [p(_NormGrads), p(_i64)]
        lib.massive_rms_norm_backward.argtypes = [p(_NormGrads), _vp, _i64, _vp]
        lib.massive_gated.argtypes = [p(_GatedArgs), _vp]
        lib.massive_gated_workspace.argtypes = [p(_GatedGrads), p(_i64)]
        lib.massive_gated_backward.argtypes = [p(_GatedGrads), _vp, _i64, _vp]
        lib.massive_adamw.argtypes = [p(_AdamwTensor), _i64, p(_AdamwArgs), _vp]
        lib.massive_adamw_states.argtypes = [_vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp]
        _lib = lib
    return _lib


def _check(rc):
    if rc != OK:
        raise MassiveError(rc, _lib.massive_last_error(None).decode())


def _stream(device: int) -> int:
    """The current stream of a GPU, as the library takes it."""
    return torch._C._cuda_getCurrentRawStream(device)


def _on_gpu(*tensors) -> int:
    """The GPU on which all tensors given (not None) lie, which must be the current one: the library launches there."""
    there = None
    for t in tensors:
        if t is not None:
            at = t.get_device()
            if at < 0 or not t.is_cuda:
                raise ValueError("operators take device (cuda) tensors, not one on %s" % t.device)
            if there is not None and at != there:
                raise ValueError("tensors lie on cuda:%d and on cuda:%d" % (there, at))
            there = at
    here = torch.cuda.current_device()
    if there is not None and there != here:
        raise ValueError("a tensor lies on cuda:%d, and cuda:%d is the current device" % (there, here))
    return here


def _no_tangent(*tensors):
    """Forward-mode derivatives are not there: a tensor that carries a tangent is refused, rather than the tangent lost."""
    if forward_ad._current_level >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise ValueError("operators have no forward-mode derivatives, and a tensor carries a tangent")


def _matrix(t, name, cols=None, rows=None, dtype=None) -> int:
    """The row stride of a 2-d tensor whose rows are contiguous; checks its shape and type."""
    if t.dim() != 2:
        raise ValueError("%s must be a 2-d tensor" % name)
    if t.dtype not in _TYPES or (dtype is not None and t.dtype != dtype):
        raise ValueError("%s is %s, and must be %s" % (name, t.dtype, dtype or "float32 or bfloat16"))
    n, d = t.shape
    if (cols is not None and d != cols) or (rows is not None and n != rows):
        raise ValueError("%s has shape %s, expected %s" % (name, (n, d), ("any" if rows is None else rows, "any" if cols is None else cols)))
    if n <= 1 and d <= 1 or not n or not d:
        return d
    step, one = t.stride()
    if d > 1 and one != 1:
        raise ValueError("%s must have contiguous rows" % name)
    if n > 1 and step < d:
        raise ValueError("%s has rows that overlap" % name)
    return step if n > 1 else d  # of a single row the stride says nothing


def _ids(t, name) -> int:
    if t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous():
        raise ValueError("%s must be a contiguous 1-d int32 tensor" % name)
    return t.numel()


# ------------------------------------------------------------------ packed rows
class RowFormat:
    """Rows of d values in 8 or 4 bits: `group` columns share a step (8 bits) or
    a least value and a step (4 bits); 0 for the whole row, else a power of two
    from 16 to 512. row_bytes, a multiple of 4, is the bytes of a row of a
    table (the least by default), and what `Massive` is given as its row_bytes
    for features held this way."""

    def __init__(self, d: int, bits: int = 8, group: int = 0, row_bytes: int = 0):
        for name, value in (("d", d), ("bits", bits), ("group", group)):
            if not -2 ** 31 <= int(value) < 2 ** 31:
                raise ValueError("%s is out of range" % name)
        self.c = _Format(int(d), int(bits), int(group), 0, int(row_bytes))
        least, floats_at = _i64(), _i64()
        lib = _load()
        _check(lib.massive_row_layout(ctypes.byref(self.c), ctypes.byref(least), ctypes.byref(floats_at)))
        self.d, self.bits, self.group = int(d), int(bits), int(group)
        self.least_bytes, self.floats_at = int(least.value), int(floats_at.value)
        self.row_bytes = self.c.row_bytes = int(row_bytes) or self.least_bytes

    def __repr__(self):
        return "RowFormat(d=%d, bits=%d, group=%d, row_bytes=%d)" % (self.d, self.bits, self.group, self.row_bytes)


def _table(t, fmt, name="table", pinned=False) -> int:
    """Rows of a table: a contiguous uint8 tensor [rows, row_bytes], on the GPU or (to be read) pinned."""
    if t.dtype != torch.uint8 or t.dim() != 2 or t.shape[1] != fmt.row_bytes or not t.is_contiguous():
        raise ValueError("%s must be a contiguous uint8 tensor of rows of %d bytes" % (name, fmt.row_bytes))
    if not (pinned and not t.is_cuda and t.is_pinned()):
        _on_gpu(t)
    return t.shape[0]


def _read_later(table):
    """The current stream reads a pinned table after the call has returned: a copy of its first byte, which torch's
    allocator of pinned memory waits for before it hands the memory out again. (A captured graph's tables are the
    program's to keep, as all that it reads.)"""
    if not table.is_cuda and table.numel() and not torch.cuda.is_current_stream_capturing():
        table.view(-1)[:1].to("cuda", non_blocking=True)


def pack_rows(x, fmt: RowFormat, out=None, slots=None):
    """Writes x's rows (float32 or bfloat16, [n, d]) in fmt to rows slots[i]
    (int32, distinct; one outside the table is left out) of the uint8 table
    `out`, or to its first n rows without slots. Without out, a new table of n
    rows. Returns the table."""
    stride = _matrix(x, "x", cols=fmt.d)
    here = _on_gpu(x, slots)
    n = x.shape[0]
    if slots is not None and _ids(slots, "slots") != n:
        raise ValueError("x has %d rows, and there are %d slots" % (n, slots.numel()))
    if out is None:
        if slots is not None:
            raise ValueError("slots without a table to write to")
        out = torch.empty((n, fmt.row_bytes), dtype=torch.uint8, device=x.device)
        if fmt.row_bytes != fmt.least_bytes:
            out[:, fmt.least_bytes:] = 0
    rows = _table(out, fmt, "out")
    if slots is None and rows < n:
        raise ValueError("out has %d rows, and x %d" % (rows, n))
    _check(_load().massive_pack_rows(ctypes.byref(fmt.c), x.data_ptr(), _TYPES[x.dtype], stride, n,
                                     None if slots is None else slots.data_ptr(), out.data_ptr(), rows, _stream(here)))
    increment_version(out)
    return out


def unpack_rows(table, fmt: RowFormat, index=None, dtype=torch.float32, out=None):
    """Reads rows index[i] (int32; one outside the table reads as zeros), or
    every row without an index, of a table on the GPU or in pinned memory, to
    a new tensor of dtype, or to `out`. A pinned table is read when the stream
    comes to it: until then it may be dropped, but not written to."""
    rows = _table(table, fmt, pinned=True)
    here = _on_gpu(index, out)
    n = rows if index is None else _ids(index, "index")
    if out is None:
        if dtype not in _TYPES:
            raise ValueError("dtype must be float32 or bfloat16, not %s" % dtype)
        out = torch.empty((n, fmt.d), dtype=dtype, device="cuda")
    elif out.requires_grad and torch.is_grad_enabled():
        raise ValueError("out requires a gradient, which rows read from a table have not")
    stride = _matrix(out, "out", cols=fmt.d, rows=n)
    _check(_load().massive_unpack_rows(ctypes.byref(fmt.c), table.data_ptr(), rows, None if index is None else index.data_ptr(), n,
                                       out.data_ptr(), _TYPES[out.dtype], stride, _stream(here)))
    _read_later(table)
    increment_version(out)
    return out


# ------------------------------------------------------------------- block mean
def _block(indptr, indices, rows) -> _Block:
    n = _ids(indptr, "indptr") - 1
    if n < 0:
        raise ValueError("indptr needs a row's end at least")
    return _Block(indptr.data_ptr(), indices.data_ptr(), n, _ids(indices, "indices"), int(rows))


def _block_mean(x, indptr, indices, fmt, dtype):
    here = _on_gpu(indptr, indices)
    if fmt is not None:
        rows, d, kind, stride, c = _table(x, fmt, "x", pinned=True), fmt.d, PACKED, 0, ctypes.byref(fmt.c)
        dtype = dtype or torch.float32
    else:
        stride = _matrix(x, "x")
        _on_gpu(x)
        (rows, d), kind, c = x.shape, _TYPES[x.dtype], None
        dtype = dtype or x.dtype
    if dtype not in _TYPES:
        raise ValueError("dtype must be float32 or bfloat16, not %s" % dtype)
    b = _block(indptr, indices, rows)
    out = torch.empty((b.n, d), dtype=dtype, device="cuda")
    _check(_load().massive_block_mean(ctypes.byref(b), x.data_ptr(), kind, stride, c, d, out.data_ptr(), _TYPES[dtype], d,
                                      _stream(here)))
    _read_later(x)
    return out


class _BlockMean(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, indptr, indices, dtype):
        ctx.save_for_backward(indptr, indices)
        ctx.rows, ctx.dtype = x.shape[0], x.dtype
        return _block_mean(x, indptr, indices, None, dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        indptr, indices = ctx.saved_tensors
        # sums are fp32, and rounded to dout's type: a gradient of bfloat16 for an fp32 input is widened before them
        wider = torch.promote_types(dout.dtype, ctx.dtype)
        return block_mean_backward(dout.to(wider).contiguous(), indptr, indices, ctx.rows).to(ctx.dtype), None, None, None


def block_mean(x, indptr, indices, fmt: Optional[RowFormat] = None, dtype=None):
    """[n, d]: the mean of x's rows indices[indptr[i]:indptr[i + 1]], zeros for
    an empty list. indptr (n + 1) and indices are int32, such as hop k's of a
    batch: `bb.indptr[k][:n + 1]`, `bb.indices[k][:e]`, with x the rows of the
    next frontier. x is float32 or bfloat16, or with fmt a table of packed
    rows, pinned ones as in unpack_rows. The result has x's type (float32 for
    packed rows) unless dtype says otherwise. An index outside x stands for a
    row of zeros."""
    _no_tangent(x)
    if fmt is None and x.requires_grad and torch.is_grad_enabled():
        return _BlockMean.apply(x, indptr, indices, dtype)
    return _block_mean(x, indptr, indices, fmt, dtype)


def block_mean_backward(dout, indptr, indices, rows: int, add=None):
    """The gradient [rows, d] of block_mean's x, in dout's type: row j sums
    dout[i] / length(i) over the rows i that list j, in their order; plus
    add[j] for the first len(add) rows."""
    _no_tangent(dout, add)
    stride = _matrix(dout, "dout")
    here = _on_gpu(dout, indptr, indices, add)
    b = _block(indptr, indices, rows)
    if dout.shape[0] != b.n:
        raise ValueError("dout has %d rows, and the block %d" % (dout.shape[0], b.n))
    d = dout.shape[1]
    add_stride = 0 if add is None else _matrix(add, "add", cols=d, dtype=dout.dtype)
    add_rows = 0 if add is None else add.shape[0]
    if add_rows > rows:
        raise ValueError("add has %d rows, more than the %d of the gradient" % (add_rows, rows))
    lib = _load()
    dx = torch.empty((int(rows), d), dtype=dout.dtype, device=dout.device)
    need = _i64()
    _check(lib.massive_block_mean_workspace(ctypes.byref(b), d, ctypes.byref(need)))
    work = torch.empty(need.value, dtype=torch.uint8, device=dout.device) if need.value else None
    _check(lib.massive_block_mean_backward(ctypes.byref(b), dout.data_ptr(), _TYPES[dout.dtype], stride, d,
                                           add.data_ptr() if add_rows else None, add_stride, add_rows, dx.data_ptr(), d,
                                           _ptr(work), need.value, _stream(here)))
    return dx


# ----------------------------------------------------------------------- linear
def _activation(act) -> int:
    if act not in ACTIVATIONS:
        raise ValueError("act must be one of %s, not %r" % (", ".join(ACTIVATIONS), act))
    return ACTIVATIONS[act]


def _layer(x, weight, x2):
    """Checks the inputs and weights of a layer; (rows, n, k, k2) and the strides of x, x2 and weight."""
    x_stride = _matrix(x, "x")
    rows, k = x.shape
    k2 = x2_stride = 0
    if x2 is not None:
        x2_stride = _matrix(x2, "x2", rows=rows, dtype=x.dtype)
        k2 = x2.shape[1]
    w_stride = _matrix(weight, "weight", cols=k + k2, dtype=x.dtype)
    return rows, weight.shape[0], k, k2, x_stride, x2_stride, w_stride


def _vector(t, name, n, dtype):
    if t.dim() != 1 or t.numel() != n or t.dtype != dtype or not t.is_contiguous():
        raise ValueError("%s must be a contiguous 1-d tensor of %d values of %s" % (name, n, dtype))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _linear(x, weight, bias, act, residual, x2, save_pre):
    code = _activation(act)
    rows, n, k, k2, x_stride, x2_stride, w_stride = _layer(x, weight, x2)
    here = _on_gpu(x, weight, bias, residual, x2)
    dtype = x.dtype
    if bias is not None:
        _vector(bias, "bias", n, dtype)
    res_stride = 0 if residual is None else _matrix(residual, "residual", cols=n, rows=rows, dtype=dtype)
    y = torch.empty((rows, n), dtype=dtype, device="cuda")
    pre = torch.empty_like(y) if save_pre else None
    a = _LinearArgs(x.data_ptr(), _ptr(x2), weight.data_ptr(), _ptr(bias), _ptr(residual), y.data_ptr(), _ptr(pre), rows,
                    x_stride, x2_stride, w_stride, res_stride, n, n, n, k, k2, _TYPES[dtype], code)
    _check(_load().massive_linear(ctypes.byref(a), _stream(here)))
    return y, pre


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, act, residual, x2):
        # relu's own output says where its slope is 1, unless a residual was added to it
        keep = act in ("gelu", "silu") or (act == "relu" and residual is not None)
        y, pre = _linear(x, weight, bias, act, residual, x2, keep)
        ctx.save_for_backward(x, weight, x2, pre if keep else (y if act == "relu" else None))
        ctx.act, ctx.bias = act, bias is not None
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, x2, pre = ctx.saved_tensors
        need = ctx.needs_input_grad
        dy = dy.contiguous()
        dx, dx2, dw, db = linear_backward(dy, x, weight, ctx.act, pre, x2, bias=ctx.bias and need[2], need_dx=need[0],
                                          need_dx2=need[5], need_dw=need[1])
        return dx, dw, db, None, dy if need[4] else None, dx2


def linear(x, weight, bias=None, act: str = "none", residual=None, x2=None, save_pre: bool = False):
    """act([x | x2] weight^T + bias) + residual, with act "none", "relu",
    "gelu" (z times the normal distribution's Phi(z)) or "silu". x [rows, k],
    x2 [rows, k2], weight [n, k + k2], bias [n], residual [rows, n]; all of one
    type, float32 or bfloat16, rows of any stride. With save_pre, returns the
    activation's argument too, for linear_backward."""
    _no_tangent(x, weight, bias, residual, x2)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, bias, residual, x2)):
        if save_pre:
            raise ValueError("save_pre is for calls outside autograd")
        return _Linear.apply(x, weight, bias, act, residual, x2)
    y, pre = _linear(x, weight, bias, act, residual, x2, save_pre)
    return (y, pre) if save_pre else y


def linear_backward(dy, x, weight, act: str = "none", pre=None, x2=None, bias: bool = True, need_dx: bool = True,
                    need_dx2: bool = True, need_dw: bool = True):
    """(dx, dx2, dweight, dbias) of `linear`, None for those not asked for or
    not there. pre is what linear returned with save_pre (for relu without a
    residual, y serves as well), None for act "none". The residual's gradient
    is dy. In bfloat16, dy times the activation's slope is rounded to bfloat16
    before it is multiplied by the weights and by the inputs; dbias sums it
    unrounded."""
    _no_tangent(dy, x, weight, pre, x2)
    code = _activation(act)
    rows, n, k, k2, x_stride, x2_stride, w_stride = _layer(x, weight, x2)
    here = _on_gpu(dy, x, weight, x2, pre)
    dtype = x.dtype
    dy_stride = _matrix(dy, "dy", cols=n, rows=rows, dtype=dtype)
    if (pre is None) != (code == 0):
        raise ValueError("pre goes with an activation, and only with one")
    pre_stride = 0 if pre is None else _matrix(pre, "pre", cols=n, rows=rows, dtype=dtype)
    new = lambda *shape: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    dx = new(rows, k) if need_dx else None
    dx2 = new(rows, k2) if need_dx2 and x2 is not None else None
    dw = new(n, k + k2) if need_dw else None
    db = new(n) if bias else None
    g = _LinearGrads(dy.data_ptr(), _ptr(pre), x.data_ptr(), _ptr(x2), weight.data_ptr(), _ptr(dx), _ptr(dx2), _ptr(dw), _ptr(db),
                     rows, dy_stride, pre_stride, x_stride, x2_stride, w_stride, k, k2, k + k2, n, k, k2, _TYPES[dtype], code)
    lib = _load()
    need = _i64()
    _check(lib.massive_linear_workspace(ctypes.byref(g), ctypes.byref(need)))
    work = torch.empty(need.value, dtype=torch.uint8, device="cuda") if need.value else None
    _check(lib.massive_linear_backward(ctypes.byref(g), _ptr(work), need.value, _stream(here)))
    return dx, dx2, dw, db


def _like(x):
    """A new tensor of x's shape and type, contiguous whatever x is."""
    return torch.empty_like(x, memory_format=torch.contiguous_format)


# ---------------------------------------------------------------------- dropout
def _seed(seed, draw):
    """The seed as 64 bits or the tensor that holds them, and draw, checked."""
    if not hasattr(draw, "__index__") or not 0 <= operator.index(draw) < 2 ** 32:
        raise ValueError("draw must be a whole number in 0..2^32 - 1, not %r" % (draw,))
    if isinstance(seed, torch.Tensor):
        if seed.dtype != torch.int64 or seed.numel() != 1:
            raise ValueError("a seed in a tensor must be one int64 value")
        return 0, seed, operator.index(draw)
    if not hasattr(seed, "__index__") or not -2 ** 63 <= operator.index(seed) < 2 ** 64:
        raise ValueError("seed must be a whole number of 64 bits, or an int64 tensor, not %r" % (seed,))
    return operator.index(seed) % 2 ** 64, None, operator.index(draw)


def _dropout(x, p, seed, draw, residual):
    bits, at, draw = _seed(seed, draw)
    stride = _matrix(x, "x")
    here = _on_gpu(x, residual, at)
    rows, d = x.shape
    res_stride = 0 if residual is None else _matrix(residual, "residual", cols=d, rows=rows, dtype=x.dtype)
    if not 0 <= p <= 1:
        raise ValueError("p must be in [0, 1], not %r" % (p,))
    y = _like(x)
    a = _DropoutArgs(x.data_ptr(), _ptr(residual), y.data_ptr(), _ptr(at), rows, stride, res_stride, d, bits, p, draw, d, _TYPES[x.dtype])
    if d:
        _check(_load().massive_dropout(ctypes.byref(a), _stream(here)))
    return y


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, p, seed, draw, residual):
        at = seed if isinstance(seed, torch.Tensor) else None
        ctx.save_for_backward(at)  # a seed changed before the backward pass would draw another mask: autograd raises
        ctx.how = p, seed if at is None else None, draw
        return _dropout(x, p, seed, draw, residual)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        at, = ctx.saved_tensors
        p, seed, draw = ctx.how
        dx = _dropout(dy.contiguous(), p, seed if at is None else at, draw, None) if ctx.needs_input_grad[0] else None
        return dx, None, None, None, dy if ctx.needs_input_grad[4] else None


def dropout(x, p: float, seed, draw: int = 0, residual=None):
    """residual + dropout(x): x / (1 - p) where a column is kept, 0 where it is
    not, whatever it held. x [rows, d] and residual are float32 or bfloat16, rows
    of any stride. Column j of row i is kept if word j % 4 of Philox4x32-10 at
    the counter (j / 4, i, draw, 0) under the seed is at least p 2^32, so the
    mask is the same wherever it is drawn, and none is stored. draw (0 to
    2^32 - 1) tells a seed's masks apart: a number for each layer, say, and a
    seed for each step. seed is a whole number of 64 bits, or an int64 tensor
    of one value on the GPU, which is read when the stream comes to it (replays
    of a captured call can have masks of their own) and stays as it is until
    the backward pass has read it too."""
    _no_tangent(x, residual)
    if torch.is_grad_enabled() and (x.requires_grad or (residual is not None and residual.requires_grad)):
        return _Dropout.apply(x, p, seed, draw, residual)
    return _dropout(x, p, seed, draw, residual)


def dropout_backward(dy, p: float, seed, draw: int = 0):
    """The gradient of dropout's x: dy under the mask of the same p, seed and
    draw. The residual's gradient is dy."""
    _no_tangent(dy)
    return _dropout(dy, p, seed, draw, None)


# ------------------------------------------------------------------------- norm
def _rms_norm(x, weight, eps, residual, fmt, out, slots):
    stride = _matrix(x, "x")
    rows, d = x.shape
    here = _on_gpu(x, weight, residual, slots)
    dtype = x.dtype
    if weight is not None:
        _vector(weight, "weight", d, dtype)
    res_stride = 0 if residual is None else _matrix(residual, "residual", cols=d, rows=rows, dtype=dtype)
    if slots is not None and _ids(slots, "slots") != rows:
        raise ValueError("x has %d rows, and there are %d slots" % (rows, slots.numel()))
    table_rows = 0
    if fmt is None:
        y = _like(x)
    else:
        if fmt.d != d:
            raise ValueError("x has %d columns, and the row format %d" % (d, fmt.d))
        if out is None:
            if slots is not None:
                raise ValueError("slots without a table to write to")
            out = torch.empty((rows, fmt.row_bytes), dtype=torch.uint8, device=x.device)
            if fmt.row_bytes != fmt.least_bytes:
                out[:, fmt.least_bytes:] = 0
        table_rows = _table(out, fmt, "out")
        if slots is None and table_rows < rows:
            raise ValueError("out has %d rows, and x %d" % (table_rows, rows))
        y = out
    total = None if residual is None else _like(x)
    a = _NormArgs(x.data_ptr(), _ptr(residual), _ptr(weight), _ptr(total), y.data_ptr(), None if fmt is None else ctypes.pointer(fmt.c), _ptr(slots),
                  table_rows, rows, stride, res_stride, d, d, eps, d, _TYPES[dtype])
    if d:
        _check(_load().massive_rms_norm(ctypes.byref(a), _stream(here)))
    if fmt is not None:
        increment_version(out)
    return y, total


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, eps, residual):
        y, total = _rms_norm(x, weight, eps, residual, None, None, None)
        ctx.save_for_backward(x if total is None else total, weight)
        ctx.eps = eps
        ctx.set_materialize_grads(False)
        return y if total is None else (y, total)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, ds=None):
        s, weight = ctx.saved_tensors
        need = ctx.needs_input_grad
        if dy is None:
            dx, dw = ds, None
        else:
            dx, dw = rms_norm_backward(dy.contiguous(), s, weight, ctx.eps, None if ds is None else ds.contiguous(), need_dx=need[0] or need[3],
                                       need_dweight=need[1])
        return dx if need[0] else None, dw, None, dx if need[3] else None


def rms_norm(x, weight=None, eps: float = 1e-6, residual=None, fmt: Optional[RowFormat] = None, out=None, slots=None):
    """s / sqrt(mean(s^2) + eps) * weight over each row of s = x + residual; with
    a residual, (that, s). x [rows, d], weight [d] and residual are of one type,
    float32 or bfloat16, rows of any stride; the mean is float32, of s before it
    is rounded. With fmt the normed rows are packed, before they are rounded to
    anything else, and written to a table as pack_rows does: to a new one, or
    to `out`, its rows slots[i] or its first ones; packed rows have no gradient,
    and tensors that ask for one are refused."""
    _no_tangent(x, weight, residual)
    if fmt is None and (out is not None or slots is not None):
        raise ValueError("out and slots are for packed rows, which fmt asks for")
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, residual)):
        if fmt is not None:
            raise ValueError("packed rows have no gradient, and a tensor requires one")
        return _RmsNorm.apply(x, weight, eps, residual)
    y, total = _rms_norm(x, weight, eps, residual, fmt, out, slots)
    return y if total is None else (y, total)


def rms_norm_backward(dy, s, weight=None, eps: float = 1e-6, ds=None, need_dx: bool = True, need_dweight: bool = True):
    """(dx, dweight) of rms_norm, None for those not asked for, dweight without
    a weight too. s is what rms_norm returned beside the norm (without a
    residual, x), ds the gradient that s gets from elsewhere, which is added to
    dx. dx is the gradient of x and of the residual."""
    _no_tangent(dy, s, weight, ds)
    stride = _matrix(s, "s")
    rows, d = s.shape
    here = _on_gpu(dy, s, weight, ds)
    dtype = s.dtype
    dy_stride = _matrix(dy, "dy", cols=d, rows=rows, dtype=dtype)
    ds_stride = 0 if ds is None else _matrix(ds, "ds", cols=d, rows=rows, dtype=dtype)
    if weight is not None:
        _vector(weight, "weight", d, dtype)
    dx = _like(s) if need_dx else None
    dw = torch.empty(d, dtype=dtype, device="cuda") if need_dweight and weight is not None else None
    if d and (dx is not None or dw is not None):
        g = _NormGrads(dy.data_ptr(), s.data_ptr(), _ptr(weight), _ptr(ds), _ptr(dx), _ptr(dw), rows, dy_stride, stride, ds_stride, d, eps, d,
                       _TYPES[dtype])
        lib = _load()
        need = _i64()
        _check(lib.massive_rms_norm_workspace(ctypes.byref(g), ctypes.byref(need)))
        work = torch.empty(need.value, dtype=torch.uint8, device="cuda") if need.value else None
        _check(lib.massive_rms_norm_backward(ctypes.byref(g), _ptr(work), need.value, _stream(here)))
    return dx, dw


# ------------------------------------------------------------------ gated layer
def _gated_layer(x, weight, x2):
    """_layer()'s, with n the outputs of a half."""
    rows, both, *rest = _layer(x, weight, x2)
    if both % 2 or not both:
        raise ValueError("weight has %d rows, and must have two for each output" % both)
    return rows, both // 2, *rest


def _gated(x, weight, bias, act, x2, save_pre):
    code = _activation(act)
    rows, n, k, k2, x_stride, x2_stride, w_stride = _gated_layer(x, weight, x2)
    here = _on_gpu(x, weight, bias, x2)
    dtype = x.dtype
    if bias is not None:
        _vector(bias, "bias", 2 * n, dtype)
    y = torch.empty((rows, n), dtype=dtype, device="cuda")
    pre = torch.empty((rows, 2 * n), dtype=dtype, device="cuda") if save_pre else None
    a = _GatedArgs(x.data_ptr(), _ptr(x2), weight.data_ptr(), _ptr(bias), y.data_ptr(), _ptr(pre), rows, x_stride, x2_stride, w_stride, n, 2 * n,
                   n, k, k2, _TYPES[dtype], code)
    _check(_load().massive_gated(ctypes.byref(a), _stream(here)))
    return y, pre


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, act, x2):
        y, pre = _gated(x, weight, bias, act, x2, True)
        ctx.save_for_backward(x, weight, x2, pre)
        ctx.act, ctx.bias = act, bias is not None
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, x2, pre = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx, dx2, dw, db = gated_backward(dy.contiguous(), x, weight, pre, ctx.act, x2, bias=ctx.bias and need[2], need_dx=need[0],
                                         need_dx2=need[4], need_dw=need[1])
        return dx, dw, db, None, dx2


def gated(x, weight, bias=None, act: str = "silu", x2=None, save_pre: bool = False):
    """act(g) * u, [g | u] = [x | x2] weight^T + bias, with linear's activations.
    x [rows, k], x2 [rows, k2], weight [2 n, k + k2], its first n rows the
    gate's, bias [2 n]; all of one type, float32 or bfloat16, rows of any
    stride. With save_pre, returns [g | u] too, for gated_backward."""
    _no_tangent(x, weight, bias, x2)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, bias, x2)):
        if save_pre:
            raise ValueError("save_pre is for calls outside autograd")
        return _Gated.apply(x, weight, bias, act, x2)
    y, pre = _gated(x, weight, bias, act, x2, save_pre)
    return (y, pre) if save_pre else y


def gated_backward(dy, x, weight, pre, act: str = "silu", x2=None, bias: bool = True, need_dx: bool = True, need_dx2: bool = True,
                   need_dw: bool = True):
    """(dx, dx2, dweight, dbias) of `gated`, None for those not asked for or not
    there. pre is what gated returned with save_pre. In bfloat16, the gradients
    of g and u are rounded to bfloat16 before they are multiplied by the
    weights and by the inputs; dbias sums them unrounded."""
    _no_tangent(dy, x, weight, pre, x2)
    code = _activation(act)
    rows, n, k, k2, x_stride, x2_stride, w_stride = _gated_layer(x, weight, x2)
    here = _on_gpu(dy, x, weight, x2, pre)
    dtype = x.dtype
    dy_stride = _matrix(dy, "dy", cols=n, rows=rows, dtype=dtype)
    pre_stride = _matrix(pre, "pre", cols=2 * n, rows=rows, dtype=dtype)
    new = lambda *shape: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    dx = new(rows, k) if need_dx else None
    dx2 = new(rows, k2) if need_dx2 and x2 is not None else None
    dw = new(2 * n, k + k2) if need_dw else None
    db = new(2 * n) if bias else None
    g = _GatedGrads(dy.data_ptr(), pre.data_ptr(), x.data_ptr(), _ptr(x2), weight.data_ptr(), _ptr(dx), _ptr(dx2), _ptr(dw), _ptr(db),
                    rows, dy_stride, pre_stride, x_stride, x2_stride, w_stride, k, k2, k + k2, n, k, k2, _TYPES[dtype], code)
    lib = _load()
    need = _i64()
    _check(lib.massive_gated_workspace(ctypes.byref(g), ctypes.byref(need)))
    work = torch.empty(need.value, dtype=torch.uint8, device="cuda") if need.value else None
    _check(lib.massive_gated_backward(ctypes.byref(g), _ptr(work), need.value, _stream(here)))
    return dx, dx2, dw, db


# ------------------------------------------------------------------------ AdamW
_dtype_of, _shape_of = operator.attrgetter("dtype"), operator.attrgetter("shape")


def _pointers(tensors):
    return list(map(torch.Tensor.data_ptr, tensors))


def _disjoint(tensors):
    """Refuses tensors (contiguous, or None) that share memory: a call's blocks would write it at the same time."""
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors if t is not None and t.numel())
    for (_, end), (begin, _) in zip(spans, spans[1:]):
        if begin < end:
            raise ValueError("parameters or copies share memory")


class AdamW:
    """AdamW over a list of tensors, contiguous, of one type (float32 or
    bfloat16) and in memory of their own, updated in place by `step`. state_bits 32 keeps the two moments
    as float32, 8 as bytes with a float32 scale for each 256 values. copies: for
    each parameter a bfloat16 tensor of its shape that receives the new values,
    or None.

    The states of all tensors lie in flat arrays, each tensor's from a multiple
    of 256 values on (`starts`). Steps are counted for each tensor; `t` is the
    largest count, and sets all of them where it is assigned."""

    def __init__(self, params: Sequence, lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 0.01, state_bits: int = 32, copies: Optional[Sequence] = None):
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        if state_bits not in (32, 8):
            raise ValueError("state_bits must be 32 or 8")
        self.copies = [None] * len(self.params) if copies is None else list(copies)
        if len(self.copies) != len(self.params):
            raise ValueError("%d parameters, and %d copies" % (len(self.params), len(self.copies)))
        self.dtype = self.params[0].dtype
        if self.dtype not in _TYPES:
            raise ValueError("parameters must be float32 or bfloat16, not %s" % self.dtype)
        _on_gpu(*self.params, *self.copies)
        for p, c in zip(self.params, self.copies):
            if p.dtype != self.dtype or not p.is_contiguous():
                raise ValueError("parameters must be contiguous and of one type")
            if c is not None and (c.dtype != torch.bfloat16 or c.shape != p.shape or not c.is_contiguous()):
                raise ValueError("a copy must be a contiguous bfloat16 tensor of its parameter's shape")
        _disjoint(self.params + self.copies)
        self.lr, self.betas, self.eps, self.weight_decay = lr, betas, eps, weight_decay
        self.state_bits, self._counts = state_bits, np.zeros(len(self.params), np.int64)
        device = self.params[0].device
        self.starts: List[int] = []
        total = 0
        for p in self.params:
            self.starts.append(total)
            total += -(-p.numel() // 256) * 256
        self.total = total
        if state_bits == 32:
            self.m, self.v = (torch.zeros(total, device=device) for _ in range(2))
            self.m_scale = self.v_scale = None
        else:
            self.m = torch.zeros(total, dtype=torch.int8, device=device)
            self.v = torch.zeros(total, dtype=torch.uint8, device=device)
            self.m_scale, self.v_scale = (torch.zeros(total // 256, device=device) for _ in range(2))
        self._list = (_AdamwTensor * len(self.params))()
        self._table = np.frombuffer(self._list, dtype=_ADAMW_ROW)  # the same memory, by columns
        size = self.m.element_size()
        starts = np.array(self.starts, np.uint64)
        self._table["m"], self._table["v"] = self.m.data_ptr() + starts * size, self.v.data_ptr() + starts * size
        if state_bits == 8:
            self._table["m_scale"] = self.m_scale.data_ptr() + starts // 256 * 4
            self._table["v_scale"] = self.v_scale.data_ptr() + starts // 256 * 4
        self._sizes = np.array([p.numel() for p in self.params], np.int64)
        self._own_layout()
        self._memory = self._table["param"] = _pointers(self.params)
        self._table["copy"] = [0 if c is None else c.data_ptr() for c in self.copies]
        self._copy_memory = _pointers(c for c in self.copies if c is not None)
        self._changed = self._written(range(len(self.params)))

    def _written(self, at):
        """The tensors that a step of the parameters `at` writes."""
        states = [s for s in (self.m, self.v, self.m_scale, self.v_scale) if s is not None]
        return [self.params[i] for i in at] + [self.copies[i] for i in at if self.copies[i] is not None] + states

    @property
    def t(self) -> int:
        return int(self._counts.max())

    @t.setter
    def t(self, steps: int):
        self._counts[:] = steps

    def _own_memory(self):
        """The parameters' and copies' memory may have been replaced since it was last seen."""
        now = _pointers(self.params)
        if now != self._memory or not all(map(torch.Tensor.is_contiguous, self._even)):
            self._own_layout()
            _on_gpu(*self.params)
            _disjoint(self.params + self.copies)
            self._memory = self._table["param"] = now
        if _pointers(c for c in self.copies if c is not None) != self._copy_memory:
            raise ValueError("a copy's memory was replaced")

    def _own_layout(self):
        """The parameters still have the type, size and layout that they began with; takes over their shapes."""
        for p, n in zip(self.params, self._sizes):
            if p.dtype != self.dtype or p.numel() != n or not p.is_contiguous():
                raise ValueError("a parameter's memory was replaced by another type, size or layout")
        self._shapes = list(map(_shape_of, self.params))
        # those of which a transposition has the same shape
        self._even = [p for p in self.params if p.dim() > 1 and len(set(p.shape)) < p.dim()]

    def _shaped(self, grads, there) -> bool:
        """Whether the gradients have their parameters' shapes."""
        now = list(map(_shape_of, grads))
        at = np.arange(len(self.params))[there]
        if now == (self._shapes if len(at) == len(self.params) else [self._shapes[i] for i in at]):
            return True
        self._own_layout()  # a parameter may have been given another view of its memory
        return now == [self._shapes[i] for i in at]

    def step(self, grads: Optional[Sequence] = None):
        """One step. grads: a contiguous tensor of each parameter's shape, all
        of one type (float32 or bfloat16); by default the parameters' .grad.
        A parameter whose gradient is None stays as it is, its count of steps
        too. A step captured into a graph keeps its lr and its counts: replays
        neither count nor correct the moments for the steps between, so while
        1 - beta^t is not 1 yet a step belongs outside the graph."""
        grads = [p.grad for p in self.params] if grads is None else list(grads)
        if len(grads) != len(self.params):
            raise ValueError("%d parameters, and %d gradients" % (len(self.params), len(grads)))
        there, changed = slice(None), self._changed
        if any(g is None for g in grads):
            there = np.array([i for i, g in enumerate(grads) if g is not None], np.int64)
            grads = [grads[i] for i in there]
            if not grads:
                return
            changed = self._written(there)
        if forward_ad._current_level >= 0:
            _no_tangent(*self.params, *grads)
        here = _on_gpu(self.params[0])
        types = set(map(_dtype_of, grads))
        if len(types) != 1 or not types <= _TYPES.keys():
            raise ValueError("gradients must be of one type, float32 or bfloat16")
        self._own_memory()
        if set(map(torch.Tensor.get_device, grads)) != {here} or not all(map(torch.Tensor.is_contiguous, grads)) or \
                not self._shaped(grads, there):
            raise ValueError("a gradient must be a contiguous tensor of its parameter's shape, on cuda:%d" % here)
        self._table["grad"][there] = np.fromiter(map(torch.Tensor.data_ptr, grads), np.uint64, len(grads))
        grad_type, stream = _TYPES[types.pop()], _stream(here)
        counts = self._counts[there] + 1
        groups = set(counts.tolist())  # one, unless some tensors went without a gradient before
        for t in groups:
            at = there if len(groups) == 1 else np.arange(len(self.params))[there][counts == t]
            self._table["n"] = 0
            self._table["n"][at] = self._sizes[at]
            a = _AdamwArgs(self.lr, self.betas[0], self.betas[1], self.eps, self.weight_decay, t, self.state_bits,
                           _TYPES[self.dtype], grad_type, 0)
            _check(_load().massive_adamw(self._list, len(self._list), ctypes.byref(a), stream))
            self._counts[at] = t
        increment_version(changed)

    def states(self):
        """(m, v), flat float32 arrays of what the states stand for (`starts`
        says where each tensor's begin). With state_bits 32 they are the
        states themselves."""
        if self.state_bits == 32:
            return self.m, self.v
        m, v = (torch.empty(self.total, device=self.m.device) for _ in range(2))
        _check(_load().massive_adamw_states(self.m.data_ptr(), self.v.data_ptr(), self.m_scale.data_ptr(), self.v_scale.data_ptr(),
                                            self.total, m.data_ptr(), v.data_ptr(), _stream(_on_gpu(m))))
        return m, v
