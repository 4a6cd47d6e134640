"""The form that each size of the gated layer's exact tests takes (csrc/gated_rules.hpp, built with g++; no GPU needed), and
that together they take every form."""
import os
import shutil
import subprocess

import pytest

from gated_sizes import FORWARD, GRADIENTS

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    exe = str(tmp_path_factory.mktemp("forms") / "gated_forms")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", os.path.join(HERE, "native", "gated_forms.cpp"), "-o", exe])
    lines = ["%s %d %s" % (what, case[0] == "bf16", " ".join(map(str, case[1:-1]))) for what, cases in (("f", FORWARD), ("b", GRADIENTS)) for case in cases]
    out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=60)
    assert out.returncode == 0
    return out.stdout.splitlines()


def test_each_size_takes_its_form(forms):
    want = [case[-1] for case in FORWARD + GRADIENTS]
    assert forms == want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_form_is_taken(dtype):
    forward = {case[-1] for case in FORWARD if case[0] == dtype}
    assert forward == {"few"} | {"%s %s" % (w, d) for w in ("wide", "narrow") for d in ("direct", "registers")}
    back = [case[-1].split() for case in GRADIENTS if case[0] == dtype]
    assert {b[0] for b in back} == {"made", "sums", "dz"}

    def after(word, b):
        return b[b.index(word) + 1:] if word in b else None

    dw = [(b[0], *w[:2], int(w[3]), int(w[5]), int(w[7]), int(w[9])) for b in back for w in (after("dw", b),) if w]
    assert {(how, width, way) for how, width, way, *_ in dw} == {("made", w, "direct") for w in ("narrow", "wide")} | \
        {("dz", w, d) for w in ("narrow", "wide") for d in ("direct", "registers")} | {("sums", "wide", "registers")}
    # the loop of steps that follow each other: an even and an odd number of them, more than it begins and ends with, and
    # last steps that have all rows and not
    for width in ("narrow", "wide"):
        steps = [s for how, w, _, _, s, _, _ in dw if how == "made" and w == width and s >= 12]
        assert steps and (width == "narrow" or {s % 2 for s in steps} == {0, 1})
    assert {rest == 0 for how, _, _, _, s, rest, _ in dw if how == "made" and s >= 12} == {True, False}
    assert {parts > 1 for _, _, _, parts, _, _, _ in dw} == {True, False}
    assert {ways for *_, parts, _, _, ways in dw if parts > 2} == {1, 4, 16}
    dx = [(*w[:2], int(w[3]) > 1, int(w[5])) for b in back for w in (after("dx", b),) if w]
    assert {(width, way, parts) for width, way, parts, _ in dx} == {(w, d, p) for w in ("narrow", "wide") for d in ("direct", "registers")
                                                                   for p in (False, True) if not (w == "wide" and p)}
    assert {ways for _, _, parts, ways in dx if parts} >= {4, 16}
