"""What dropout, the norm and the gated layer refuse, before any device call (no GPU needed)."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2410_22697_amd import massive, operators
from paper_2410_22697_amd.massive import ECAPACITY, EINVAL, OK

pytestmark = pytest.mark.skipif(not os.path.exists(massive.LIB_PATH), reason="libmassive.so not built")
P = 4096  # an address that is aligned and never followed: every call here is refused, or has nothing to do


def lib():
    return operators._load()


def refused(rc, word, code=EINVAL):
    message = lib().massive_last_error(None).decode()
    assert rc == code and word in message, (rc, message)


def drop(**more):
    a = dict(x=P, y=P, rows=4, x_stride=6, y_stride=6, p=0.5, d=6, type=0)
    return operators._DropoutArgs(**{**a, **more})


@pytest.mark.parametrize("bad,word", [(dict(type=2), "type"), (dict(rows=-1), "rows"), (dict(rows=1 << 30), "rows"), (dict(d=0), "d must"),
                                      (dict(d=(1 << 20) + 1), "d must"), (dict(p=-0.1), "p must"), (dict(p=1.1), "p must"), (dict(p=float("nan")), "p must"),
                                      (dict(x=None), "NULL"), (dict(y=None), "NULL"), (dict(x_stride=5), "stride"), (dict(y_stride=5), "stride"),
                                      (dict(residual=P, residual_stride=5), "stride"), (dict(x=P + 2), "aligned"), (dict(y=P + 1, type=1), "aligned"),
                                      (dict(seed_at=P + 4), "aligned")])
def test_dropout(bad, word):
    a = drop(**bad)
    refused(lib().massive_dropout(ctypes.byref(a), None), word)


def norm(**more):
    a = dict(x=P, y=P, rows=4, x_stride=6, y_stride=6, eps=1e-6, d=6, type=0)
    return operators._NormArgs(**{**a, **more})


FMT = operators._Format(6, 8, 0, 0, 0)


@pytest.mark.parametrize("bad,word", [(dict(type=2), "type"), (dict(rows=-1), "rows"), (dict(d=0), "d must"), (dict(d=(1 << 20) + 1), "d must"),
                                      (dict(eps=-1e-9), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=1e39), "eps"), (dict(x=None), "NULL"),
                                      (dict(y=None), "NULL"), (dict(x_stride=5), "stride"), (dict(y_stride=5), "stride"),
                                      (dict(residual=P, residual_stride=5), "stride"), (dict(sum=P, sum_stride=5), "stride"),
                                      (dict(weight=P + 2), "aligned"), (dict(slots=P), "slots"), (dict(fmt=ctypes.pointer(FMT), d=7, x_stride=7), "format"),
                                      (dict(fmt=ctypes.pointer(FMT), table_rows=-1), "table_rows"), (dict(fmt=ctypes.pointer(FMT), table_rows=4, y=P + 2), "table"),
                                      (dict(fmt=ctypes.pointer(FMT), table_rows=4, slots=P + 2), "slots"),
                                      (dict(fmt=ctypes.pointer(operators._Format(6, 3, 0, 0, 0))), "bits")])
def test_norm(bad, word):
    a = norm(**bad)
    refused(lib().massive_rms_norm(ctypes.byref(a), None), word)


def norm_grads(**more):
    a = dict(dy=P, s=P, weight=P, dx=P, dweight=P, rows=4, dy_stride=6, s_stride=6, dx_stride=6, eps=1e-6, d=6, type=0)
    return operators._NormGrads(**{**a, **more})


@pytest.mark.parametrize("bad,word", [(dict(type=2), "type"), (dict(rows=-1), "rows"), (dict(d=0), "d must"), (dict(dy=None), "NULL"), (dict(s=None), "NULL"),
                                      (dict(dy_stride=5), "stride"), (dict(s_stride=5), "stride"), (dict(dx_stride=5), "stride"),
                                      (dict(ds=P, ds_stride=5), "stride"), (dict(eps=-1.0), "eps"), (dict(dweight=P + 1), "aligned")])
def test_norm_backward(bad, word):
    a = norm_grads(**bad)
    refused(lib().massive_rms_norm_backward(ctypes.byref(a), P, 1 << 40, None), word)


def test_workspaces_and_calls_with_nothing_to_do():
    size = ctypes.c_int64()
    a = norm_grads()
    assert lib().massive_rms_norm_workspace(ctypes.byref(a), ctypes.byref(size)) == OK and size.value > 0
    refused(lib().massive_rms_norm_backward(ctypes.byref(a), P, size.value - 1, None), "workspace", ECAPACITY)
    refused(lib().massive_rms_norm_backward(ctypes.byref(a), None, size.value, None), "workspace", ECAPACITY)
    refused(lib().massive_rms_norm_backward(ctypes.byref(a), P + 8, size.value, None), "aligned")
    refused(lib().massive_rms_norm_workspace(ctypes.byref(a), None), "NULL")
    none = norm_grads(dx=None, dweight=None)
    assert lib().massive_rms_norm_workspace(ctypes.byref(none), ctypes.byref(size)) == OK and size.value == 0
    assert lib().massive_rms_norm_backward(ctypes.byref(none), None, 0, None) == OK
    assert lib().massive_rms_norm_backward(ctypes.byref(norm_grads(rows=0, dweight=None)), None, 0, None) == OK
    assert lib().massive_dropout(ctypes.byref(drop(rows=0, x=None, y=None)), None) == OK
    assert lib().massive_rms_norm(ctypes.byref(norm(rows=0, x=None, y=None)), None) == OK
    for call in (lib().massive_dropout, lib().massive_rms_norm):
        refused(call(None, None), "NULL")
    refused(lib().massive_rms_norm_backward(None, None, 0, None), "NULL")


def layer(**more):
    a = dict(x=P, w=P, y=P, rows=4, x_stride=6, w_stride=6, y_stride=5, n=5, k=6, k_second=0, type=0, act=3)
    return operators._GatedArgs(**{**a, **more})


@pytest.mark.parametrize("bad,word", [(dict(type=2), "type"), (dict(act=4), "act"), (dict(act=-1), "act"), (dict(rows=-1), "rows"), (dict(n=0), "n must"),
                                      (dict(n=(1 << 19) + 1), "n must"), (dict(k=0), "n must"), (dict(k_second=-1), "k_second"), (dict(x=None), "NULL"),
                                      (dict(w=None), "NULL"), (dict(y=None), "NULL"), (dict(x_stride=5), "stride"), (dict(w_stride=5), "stride"),
                                      (dict(y_stride=4), "stride"), (dict(k_second=2), "go together"), (dict(x_second=P), "go together"),
                                      (dict(pre=P, pre_stride=9), "stride"), (dict(bias=P + 2), "aligned"), (dict(rows=1 << 30), "rows")])
def test_gated(bad, word):
    a = layer(**bad)
    refused(lib().massive_gated(ctypes.byref(a), None), word)


def gated_grads(**more):
    a = dict(dy=P, pre=P, x=P, w=P, dx=P, dw=P, dbias=P, rows=4, dy_stride=5, pre_stride=10, x_stride=6, w_stride=6, dx_stride=6, dw_stride=6, n=5, k=6,
             type=0, act=3)
    return operators._GatedGrads(**{**a, **more})


@pytest.mark.parametrize("bad,word", [(dict(type=3), "type"), (dict(act=9), "act"), (dict(dy=None), "NULL"), (dict(pre=None), "pre"), (dict(w=None), "w is"),
                                      (dict(x=None), "x is"), (dict(dy_stride=4), "stride"), (dict(pre_stride=9), "stride"), (dict(dw_stride=5), "stride"),
                                      (dict(dx_stride=5), "stride"), (dict(dx_second=P), "second"), (dict(dw=P + 1), "aligned"), (dict(n=0), "n must")])
def test_gated_backward(bad, word):
    a = gated_grads(**bad)
    refused(lib().massive_gated_backward(ctypes.byref(a), P, 1 << 40, None), word)


def test_gated_workspace():
    a, size = gated_grads(), ctypes.c_int64()
    assert lib().massive_gated_workspace(ctypes.byref(a), ctypes.byref(size)) == OK and size.value > 0
    refused(lib().massive_gated_backward(ctypes.byref(a), P, size.value - 1, None), "workspace", ECAPACITY)
    refused(lib().massive_gated_backward(ctypes.byref(a), None, size.value, None), "workspace", ECAPACITY)
    refused(lib().massive_gated_backward(ctypes.byref(a), P + 8, size.value, None), "aligned")
    refused(lib().massive_gated_workspace(ctypes.byref(a), None), "NULL")
    refused(lib().massive_gated_workspace(None, ctypes.byref(size)), "NULL")
    assert lib().massive_gated_backward(ctypes.byref(gated_grads(dx=None, dw=None, dbias=None)), None, 0, None) == OK
    assert lib().massive_gated(ctypes.byref(layer(rows=0, x=None, y=None)), None) == OK
    refused(lib().massive_gated(None, None), "NULL")
    refused(lib().massive_gated_backward(None, None, 0, None), "NULL")


def test_struct_layouts_match_the_binding(tmp_path):
    """Every field of the structs, as a C99 compiler sees the header."""
    if shutil.which("gcc") is None:
        pytest.skip("needs gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"massive_dropout_args": operators._DropoutArgs, "massive_norm_args": operators._NormArgs, "massive_norm_grads": operators._NormGrads,
               "massive_gated_args": operators._GatedArgs, "massive_gated_grads": operators._GatedGrads}
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "massive.h"', "int main(void) {"]
    want = []
    for name, s in structs.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(ctypes.sizeof(s))
        for field, _ in s._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, field))
            want.append(getattr(s, field).offset)
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0;", "}", ""]))
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)])
    assert [int(v) for v in subprocess.check_output([str(exe)]).split()] == want


X = torch.randn(6, 16)


@pytest.mark.parametrize("call,word", [
    (lambda: operators.dropout(X, 0.5, 1), "device"), (lambda: operators.dropout(X[0], 0.5, 1), "2-d"),
    (lambda: operators.dropout(X.double(), 0.5, 1), "float64"), (lambda: operators.dropout(X, 0.5, 2 ** 64), "64 bits"),
    (lambda: operators.dropout(X, 0.5, 1.5), "whole number"), (lambda: operators.dropout(X, 0.5, 1, draw=-1), "draw"),
    (lambda: operators.dropout(X, 0.5, 1, draw=2 ** 32), "draw"), (lambda: operators.dropout(X, 0.5, torch.zeros(2, dtype=torch.int64)), "one int64"),
    (lambda: operators.dropout(X, 0.5, torch.zeros(1)), "one int64"), (lambda: operators.dropout(X.t(), 0.5, 1), "contiguous rows"),
    (lambda: operators.dropout_backward(X.expand(1, 6, 16)[0].expand(6, 16)[:1].expand(6, 16), 0.5, 1), "overlap"),
    (lambda: operators.gated(X, torch.randn(10, 16)), "device"),
    (lambda: operators.gated(X, torch.randn(9, 16)), "two for each"), (lambda: operators.gated(X, torch.randn(10, 15)), "shape"),
    (lambda: operators.gated(X, torch.randn(10, 16), act="tanh"), "act must"), (lambda: operators.gated_backward(X, X, torch.randn(32, 16), X), "device"),
    (lambda: operators.rms_norm(X), "device"), (lambda: operators.rms_norm(X[0]), "2-d"), (lambda: operators.rms_norm_backward(X, X), "device")])
def test_the_binding_refuses(call, word):
    with pytest.raises(ValueError, match=word):
        call()


def test_tangents_are_refused():
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(X, torch.ones_like(X))
        for bad in (lambda: operators.dropout(dual, 0.5, 1), lambda: operators.dropout(X, 0.5, 1, residual=dual), lambda: operators.rms_norm(dual),
                    lambda: operators.rms_norm(X, residual=dual), lambda: operators.rms_norm_backward(dual, X), lambda: operators.dropout_backward(dual, 0.5, 1),
                    lambda: operators.gated(dual, X), lambda: operators.gated_backward(X, X, X, dual)):
            with pytest.raises(ValueError, match="tangent"):
                bad()
