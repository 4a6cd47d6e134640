"""The operators' C entry points refuse arguments outside their documented ranges before any device call (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2410_22697_amd import RowFormat, massive, operators
from paper_2410_22697_amd.massive import ECAPACITY, EINVAL, OK

pytestmark = pytest.mark.skipif(not os.path.exists(massive.LIB_PATH), reason="libmassive.so not built")
P = 4096  # an address that is aligned and never followed: every call here is refused, or has nothing to do


def lib():
    return operators._load()


def refused(rc, word, code=EINVAL):
    message = lib().massive_last_error(None).decode()
    assert rc == code and word in message, (rc, message)


def fmt(d=16, bits=8, group=0, reserved=0, row_bytes=0):
    return operators._Format(d, bits, group, reserved, row_bytes)


@pytest.mark.parametrize("bad,word", [(dict(d=0), "d must"), (dict(d=(1 << 20) + 1), "d must"), (dict(bits=2), "bits"),
                                      (dict(group=8), "group"), (dict(group=24), "group"), (dict(group=1024), "group"),
                                      (dict(group=-16), "group"), (dict(reserved=1), "reserved"), (dict(row_bytes=16), "row_bytes"),
                                      (dict(row_bytes=22), "row_bytes"), (dict(row_bytes=-4), "row_bytes")])
def test_row_format(bad, word):
    f = fmt(**bad)
    refused(lib().massive_row_layout(ctypes.byref(f), None, None), word)
    refused(lib().massive_pack_rows(ctypes.byref(f), P, 0, 64, 1, None, P, 1, None), word)
    refused(lib().massive_unpack_rows(ctypes.byref(f), P, 1, None, 1, P, 0, 64, None), word)


@pytest.mark.parametrize("d,bits,group,least,floats_at", [(1, 8, 0, 8, 4), (128, 8, 0, 132, 128), (100, 8, 32, 116, 100), (100, 4, 32, 84, 52),
                                                          (1, 4, 0, 12, 4), (9, 4, 0, 16, 8), (64, 8, 64, 68, 64), (65, 8, 64, 76, 68)])
def test_row_layout(d, bits, group, least, floats_at):
    f = RowFormat(d, bits, group)
    assert (f.least_bytes, f.floats_at, f.row_bytes) == (least, floats_at, least)
    assert RowFormat(d, bits, group, row_bytes=least + 8).row_bytes == least + 8
    refused(lib().massive_row_layout(None, None, None), "NULL")


def test_rows():
    f = fmt()
    call = lib().massive_pack_rows
    for args, word in (((P, 2, 16, 1, None, P, 1), "src_type"), ((P, 0, 15, 1, None, P, 1), "stride"), ((None, 0, 16, 1, None, P, 1), "NULL"),
                       ((P, 0, 16, 1, None, None, 1), "NULL"), ((P, 0, 16, -1, None, P, 1), "negative"), ((P + 2, 0, 16, 1, None, P, 1), "aligned"),
                       ((P, 0, 16, 1, P + 1, P, 1), "aligned"), ((P, 0, 16, 1, None, P + 2, 1), "aligned")):
        refused(call(ctypes.byref(f), *args, None), word)
    assert call(ctypes.byref(f), None, 0, 16, 0, None, None, 0, None) == OK
    call = lib().massive_unpack_rows
    for args, word in (((P, 1, None, 1, P, 7, 16), "out_type"), ((P, 1, None, 1, P, 0, 15), "stride"), ((None, 1, None, 1, P, 0, 16), "NULL"),
                       ((P, 1, None, 1, None, 0, 16), "NULL"), ((P, -1, None, 1, P, 0, 16), "negative"), ((P, 1, None, 1, P + 2, 0, 16), "aligned")):
        refused(call(ctypes.byref(f), *args, None), word)
    assert call(ctypes.byref(f), None, 0, None, 0, None, 0, 16, None) == OK


def block(indptr=P, indices=P, n=4, edges=5000, rows=10):
    return operators._Block(indptr, indices, n, edges, rows)


BLOCKS = [(dict(n=-1), "negative"), (dict(edges=-1), "negative"), (dict(rows=-1), "negative"), (dict(edges=(1 << 30) + 1), "2^30"),
          (dict(rows=(1 << 30) + 1), "2^30"), (dict(n=(1 << 30) + 1), "2^30"), (dict(indptr=None), "indptr"), (dict(indices=None), "indices"), (dict(indptr=P + 2), "aligned")]


@pytest.mark.parametrize("bad,word", BLOCKS)
def test_block(bad, word):
    b = block(**bad)
    size = ctypes.c_int64()
    refused(lib().massive_block_mean(ctypes.byref(b), P, 0, 16, None, 16, P, 0, 16, None), word)
    refused(lib().massive_block_mean_workspace(ctypes.byref(b), 16, ctypes.byref(size)), word)
    refused(lib().massive_block_mean_backward(ctypes.byref(b), P, 0, 16, 16, None, 0, 0, P, 16, P, 1 << 40, None), word)


def test_block_mean():
    b, f = block(), fmt()
    call = lib().massive_block_mean
    for args, word in (((P, 3, 16, None, 16, P, 0, 16), "x_type"), ((P, 0, 16, None, 16, P, 2, 16), "out_type"), ((P, 0, 15, None, 16, P, 0, 16), "x_stride"),
                       ((P, 0, 16, None, 16, P, 0, 15), "out_stride"), ((P, 0, 16, None, 0, P, 0, 16), "d must"), ((None, 0, 16, None, 16, P, 0, 16), "NULL"),
                       ((P, 2, 0, None, 16, P, 0, 16), "format"), ((P, 2, 0, ctypes.byref(f), 17, P, 0, 17), "format"),
                       ((P, 0, 16, ctypes.byref(f), 16, P, 0, 16), "format"), ((P + 2, 0, 16, None, 16, P, 0, 16), "aligned")):
        refused(call(ctypes.byref(b), *args, None), word)
    none = block(indptr=None, n=0)
    assert call(ctypes.byref(none), None, 0, 16, None, 16, None, 0, 16, None) == OK
    refused(call(None, P, 0, 16, None, 16, P, 0, 16, None), "NULL")


def test_block_mean_backward():
    b, size = block(), ctypes.c_int64()
    assert lib().massive_block_mean_workspace(ctypes.byref(b), 16, ctypes.byref(size)) == OK and size.value > 0
    refused(lib().massive_block_mean_workspace(ctypes.byref(b), 16, None), "NULL")
    refused(lib().massive_block_mean_workspace(ctypes.byref(b), 0, ctypes.byref(size)), "d must")
    call = lib().massive_block_mean_backward
    need = size.value
    for args, word, code in (((P, 5, 16, 16, None, 0, 0, P, 16, P, need), "type", EINVAL), ((P, 0, 15, 16, None, 0, 0, P, 16, P, need), "stride", EINVAL),
                             ((P, 0, 16, 16, P, 15, 4, P, 16, P, need), "add_stride", EINVAL), ((P, 0, 16, 16, P, 16, 11, P, 16, P, need), "add_rows", EINVAL),
                             ((P, 0, 16, 16, None, 0, 0, P, 16, P, need - 1), "workspace", ECAPACITY),
                             ((P, 0, 16, 16, None, 0, 0, P, 16, None, need), "workspace", ECAPACITY),
                             ((P, 0, 16, 16, None, 0, 0, P, 16, P + 4, need), "aligned", EINVAL),
                             ((None, 0, 16, 16, None, 0, 0, P, 16, P, need), "NULL", EINVAL)):
        refused(call(ctypes.byref(b), *args, None), word, code)


def layer(**more):
    a = dict(x=P, w=P, y=P, rows=4, x_stride=6, w_stride=6, y_stride=5, n=5, k=6, k_second=0, type=0, act=0)
    return operators._LinearArgs(**{**a, **more})


@pytest.mark.parametrize("bad,word", [(dict(type=2), "type"), (dict(act=4), "act"), (dict(act=-1), "act"), (dict(rows=-1), "rows"), (dict(n=0), "n and k"),
                                      (dict(k=0), "n and k"), (dict(k_second=-1), "k_second"), (dict(x=None), "NULL"), (dict(w=None), "NULL"),
                                      (dict(y=None), "NULL"), (dict(x_stride=5), "stride"), (dict(w_stride=5), "stride"), (dict(y_stride=4), "stride"),
                                      (dict(k_second=2), "go together"), (dict(x_second=P), "go together"),
                                      (dict(residual=P, residual_stride=4), "stride"), (dict(pre=P, pre_stride=4), "stride"),
                                      (dict(bias=P + 2), "aligned"), (dict(rows=1 << 30), "rows")])
def test_linear(bad, word):
    a = layer(**bad)
    refused(lib().massive_linear(ctypes.byref(a), None), word)


def grads(**more):
    a = dict(dy=P, x=P, w=P, dx=P, dw=P, dbias=P, rows=4, dy_stride=5, x_stride=6, w_stride=6, dx_stride=6, dw_stride=6, n=5, k=6, type=0, act=0)
    return operators._LinearGrads(**{**a, **more})


@pytest.mark.parametrize("bad,word", [(dict(type=3), "type"), (dict(act=9), "act"), (dict(dy=None), "NULL"), (dict(act=1), "pre"), (dict(w=None), "w is"),
                                      (dict(x=None), "x is"), (dict(dy_stride=4), "stride"), (dict(dw_stride=5), "stride"), (dict(dx_stride=5), "stride"),
                                      (dict(dx_second=P), "second"), (dict(dw=P + 1), "aligned"), (dict(act=2, pre=P, pre_stride=4), "stride")])
def test_linear_backward(bad, word):
    a = grads(**bad)
    refused(lib().massive_linear_backward(ctypes.byref(a), P, 1 << 40, None), word)


def test_linear_workspace():
    a, size = grads(), ctypes.c_int64()
    assert lib().massive_linear_workspace(ctypes.byref(a), ctypes.byref(size)) == OK and size.value > 0
    refused(lib().massive_linear_backward(ctypes.byref(a), P, size.value - 1, None), "workspace", ECAPACITY)
    refused(lib().massive_linear_backward(ctypes.byref(a), None, size.value, None), "workspace", ECAPACITY)
    refused(lib().massive_linear_backward(ctypes.byref(a), P + 8, size.value, None), "aligned")
    refused(lib().massive_linear_workspace(ctypes.byref(a), None), "NULL")
    only_dx = grads(dw=None, dbias=None)
    assert lib().massive_linear_workspace(ctypes.byref(only_dx), ctypes.byref(size)) == OK and size.value == 0
    nothing = grads(dx=None, dw=None, dbias=None)
    assert lib().massive_linear_backward(ctypes.byref(nothing), None, 0, None) == OK
    assert lib().massive_linear(ctypes.byref(layer(rows=0, x=None, y=None)), None) == OK
    refused(lib().massive_linear(None, None), "NULL")
    refused(lib().massive_linear_backward(None, None, 0, None), "NULL")


def tensor(**more):
    return operators._AdamwTensor(**{**dict(param=P, grad=P, m=P, v=P, n=10), **more})


def step(**more):
    a = dict(lr=1e-3, beta_first=0.9, beta_second=0.99, eps=1e-8, weight_decay=0.0, t=1, state_bits=32, param_type=0, grad_type=0)
    return operators._AdamwArgs(**{**a, **more})


@pytest.mark.parametrize("args,word", [(dict(state_bits=16), "state_bits"), (dict(param_type=2), "param_type"), (dict(t=0), "t counts"), (dict(lr=-1.0), "lr"),
                                       (dict(lr=float("nan")), "lr"), (dict(eps=float("inf")), "lr"), (dict(beta_first=1.0), "betas"),
                                       (dict(beta_second=-0.5), "betas"), (dict(reserved=3), "reserved"), (dict(state_bits=8), "scales")])
def test_adamw_args(args, word):
    t, a = tensor(), step(**args)
    refused(lib().massive_adamw(ctypes.byref(t), 1, ctypes.byref(a), None), word)


@pytest.mark.parametrize("bad,word", [(dict(param=None), "NULL"), (dict(grad=None), "NULL"), (dict(m=None), "NULL"), (dict(n=-1), "n must"),
                                      (dict(m_scale=P, v_scale=P), "scales"), (dict(m_scale=P), "scales"), (dict(param=P + 2), "aligned"), (dict(copy=P + 1), "aligned")])
def test_adamw_tensors(bad, word):
    t, a = tensor(**bad), step()
    refused(lib().massive_adamw(ctypes.byref(t), 1, ctypes.byref(a), None), word)
    refused(lib().massive_adamw(None, 1, ctypes.byref(a), None), "NULL")
    refused(lib().massive_adamw(ctypes.byref(t), 1, None, None), "NULL")
    empty = tensor(n=0)
    assert lib().massive_adamw(ctypes.byref(empty), 1, ctypes.byref(a), None) == OK
    assert lib().massive_adamw(None, 0, ctypes.byref(a), None) == OK


def test_adamw_states():
    call = lib().massive_adamw_states
    refused(call(P, P, P, P, -1, P, P, None), "negative")
    refused(call(P, None, P, P, 1, P, P, None), "NULL")
    refused(call(P, P, P + 2, P, 1, P, P, None), "aligned")
    assert call(None, None, None, None, 0, None, None, None) == OK


def test_struct_layouts_match_the_binding(tmp_path):
    """Every field of the operators' structs, as a C99 compiler sees the header."""
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("needs gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"massive_row_format": operators._Format, "massive_block": operators._Block, "massive_linear_args": operators._LinearArgs,
               "massive_linear_grads": operators._LinearGrads, "massive_adamw_tensor": operators._AdamwTensor,
               "massive_adamw_args": operators._AdamwArgs}
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "massive.h"', "int main(void) {"]
    want = []
    for name, s in structs.items():
        for f, t in s._fields_:
            lines.append('printf("%%zu %%zu\\n", offsetof(%s, %s), sizeof(((%s*)0)->%s));' % (name, f, name, f))
            want.append((getattr(s, f).offset, ctypes.sizeof(t)))
        lines.append('printf("%%zu 0\\n", sizeof(%s));' % name)
        want.append((ctypes.sizeof(s), 0))
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    assert [tuple(int(v) for v in line.split()) for line in out.splitlines()] == want
    assert operators._ADAMW_ROW.itemsize == ctypes.sizeof(operators._AdamwTensor)
    assert all(operators._ADAMW_ROW.fields[f][1] == getattr(operators._AdamwTensor, f).offset for f in operators._ADAMW_ROW.names)


def test_constants_match_the_header():
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "massive.h")).read()
    defs = dict(re.findall(r"#define (MASSIVE_\w+) (\d+)", text))
    assert [int(defs["MASSIVE_" + n]) for n in ("F32", "BF16", "PACKED")] == [operators.F32, operators.BF16, operators.PACKED]
    assert {k: int(defs["MASSIVE_ACT_" + k.upper()]) for k in operators.ACTIVATIONS} == operators.ACTIVATIONS


def test_tensors_on_the_cpu_are_refused():
    import torch
    x = torch.zeros(3, 16)
    for bad in (lambda: operators.pack_rows(x, RowFormat(16)), lambda: operators.linear(x, torch.zeros(2, 16)), lambda: operators.AdamW([x]),
                lambda: operators.block_mean(x, torch.zeros(2, dtype=torch.int32), torch.zeros(0, dtype=torch.int32))):
        with pytest.raises(ValueError, match="device"):
            bad()
