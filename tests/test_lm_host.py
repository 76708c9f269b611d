"""CPU tests of the language-model operators' host side: refusals before any
device work, the structures' layout, and the timed cases' plain forms against
their definitions in 64 bits.  No kernel runs here."""
import ctypes
import os
import shutil
import subprocess
import sys

import pytest
import torch

from conftest import ROOT, cuda_available
from paper_1904_00962_gb300 import binding as B
from paper_1904_00962_gb300 import build as build_mod


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return B.load()


def _refused(call, status=B.LAMB_ERR_INVALID_ARG, word=""):
    with pytest.raises(B.LambError) as e:
        call()
    assert e.value.status == status
    assert word in str(e.value)


@pytest.mark.parametrize("args,word", [
    ((0, 64, 10, 0), "vocab"), ((-5, 64, 10, 0), "vocab"),
    ((2 ** 31, 64, 10, 0), "vocab"), ((10, 0, 10, 0), "width"),
    ((10, 2 ** 21, 10, 0), "width"), ((10, 64, 0, 0), "max_tokens"),
    ((10, 64, 2 ** 25, 0), "max_tokens"), ((10, 64, 10, -1), "device"),
    ((2 ** 30, 64, 2 ** 24, 0), "max_tokens times vocab")])
def test_vocab_create_refuses(lib, args, word):
    _refused(lambda: B.lamb_vocab_create(*args), word=word)


def test_vocab_calls_refuse_a_null_plan(lib):
    P = 1 << 20
    for call in (
            lambda: B.lamb_vocab_embed(0, P, 0, 8, P, 1, 1.0, P, 0, 8, 0),
            lambda: B.lamb_vocab_embed_grad(0, P, 0, 8, P, 1, 1.0, P, 0, 8, 0,
                                            0),
            lambda: B.lamb_vocab_loss(0, P, 8, P, 8, P, 1, 0, P, 0),
            lambda: B.lamb_vocab_loss_grad(0, P, 8, P, 8, P, 1, 0, 0, P, P, 8,
                                           P, 0, 8, 0, 0),
            lambda: B.lamb_vocab_query(0)):
        _refused(call, word="plan")
    B.lamb_vocab_destroy(0)      # a no-op


@pytest.mark.parametrize("kw,status,word", [
    (dict(rows=[], cols=[]), B.LAMB_ERR_INVALID_ARG, "n_matrices"),
    (dict(rows=[-1], cols=[4]), B.LAMB_ERR_INVALID_ARG, "sides"),
    (dict(rows=[4], cols=[2 ** 21]), B.LAMB_ERR_INVALID_ARG, "sides"),
    (dict(rows=[2 ** 16], cols=[2 ** 16]), B.LAMB_ERR_INVALID_ARG, "shorter"),
    (dict(rows=[2 ** 15] * 65, cols=[2 ** 15] * 65), B.LAMB_ERR_INVALID_ARG,
     "2^36"),
    (dict(rows=[4], cols=[4], grad_dtype=7), B.LAMB_ERR_UNSUPPORTED_DTYPE,
     "grad_dtype"),
    (dict(rows=[4], cols=[4], copy_dtype=B.LAMB_F32),
     B.LAMB_ERR_UNSUPPORTED_DTYPE, "copy_dtype"),
    (dict(rows=[4], cols=[4], device=-1), B.LAMB_ERR_INVALID_ARG, "device")])
def test_muon_create_refuses(lib, kw, status, word):
    _refused(lambda: B.lamb_muon_create(**kw), status, word)


def test_muon_calls_refuse_a_null_plan(lib):
    h = B.make_muon_hyper()
    for call in (lambda: B.lamb_muon_bind(0, [1], [1], [1]),
                 lambda: B.lamb_muon_bind_direction(0, [1], [1]),
                 lambda: B.lamb_muon_step(0, h, 1 << 20),
                 lambda: B.lamb_muon_direction(0, h),
                 lambda: B.lamb_muon_query(0)):
        _refused(call, word="plan")
    B.lamb_muon_destroy(0)       # a no-op


@pytest.mark.skipif(cuda_available(), reason="checks the no-GPU error path")
def test_create_without_a_gpu_reports_it(lib):
    for call in (lambda: B.lamb_vocab_create(10, 64, 10),
                 lambda: B.lamb_muon_create([4], [4])):
        with pytest.raises(B.LambError) as e:
            call()
        assert e.value.status in (B.LAMB_ERR_CUDA, B.LAMB_ERR_OOM)


def test_muon_hyper_fields(lib):
    h = B.make_muon_hyper(momentum=0.9, scale="rms", steps=7, nesterov=False,
                          coefficients=(1.0, 2.0, 3.0), update_scale=0.5)
    assert (h.momentum, h.a, h.b, h.c, h.update_scale) == (0.9, 1, 2, 3, 0.5)
    assert (h.steps, h.scale_kind, h.flags) == (7, B.LAMB_MUON_SCALE_RMS, 0)
    assert B.make_muon_hyper().flags == B.LAMB_MUON_FLAG_NESTEROV
    with pytest.raises(KeyError):
        B.make_muon_hyper(scale="other")


def test_muon_hyper_layout(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not available")
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "lamb.h"',
             'int main(void){',
             'printf("size %zu\\n", sizeof(lamb_muon_hyper_t));']
    for f, _ in B.lamb_muon_hyper_t._fields_:
        lines.append(f'printf("{f} %zu\\n", offsetof(lamb_muon_hyper_t, {f}));')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    exe = tmp_path / "layout"
    res = subprocess.run([gcc, "-std=c99", "-Wall", "-Werror", "-I",
                          os.path.join(ROOT, "include"), "-I",
                          "/usr/local/cuda/include", str(src), "-o", str(exe)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    out = dict(l.split() for l in subprocess.run(
        [str(exe)], capture_output=True, text=True).stdout.splitlines())
    assert int(out.pop("size")) == ctypes.sizeof(B.lamb_muon_hyper_t)
    for f, v in out.items():
        assert int(v) == getattr(B.lamb_muon_hyper_t, f).offset, f


@pytest.fixture(scope="module")
def cases():
    if ROOT not in sys.path:
        sys.path.insert(0, ROOT)
    from perf import operators
    device, operators.DEV = operators.DEV, "cpu"
    yield operators
    operators.DEV = device


@pytest.mark.parametrize("case,bound", [
    (dict(op="lookup", tokens=50, vocab=40, width=9, table="f32", out="f32",
          masked=0.2, padded=0.2), 1e-6),
    (dict(op="lookup_grad", tokens=90, vocab=40, width=9, grad="f32",
          table="f32", accumulate=True, masked=0.2, padded=0.2), 1e-6),
    (dict(op="head", tokens=30, vocab=70, width=24, train=True, ignored=0.3),
     4e-3),
    (dict(op="direction", shapes="1*12x30,2*30x12"), 4e-3),
    (dict(op="step", shapes="1*12x30"), 4e-3)])
def test_plain_forms_are_the_definitions(cases, case, bound):
    """The timed plain forms against 64 bits, written apart (bf16 results are
    within 2^-8)."""
    got = cases.run(cases.prepare(case, 3))
    want = cases.exact(case, 3)
    if not isinstance(want, dict):
        got, want = {"": got}, {"": want}
    for k, w in want.items():
        err = float((got[k].double() - w).norm() / w.norm())
        assert err < bound, (k, err)


def test_timed_cases(cases):
    listed = cases.listed()
    assert 4 <= len(listed) <= 12
    assert len({c["name"] for c in listed}) == len(listed)
    import random
    drawn = [cases.draw(random.Random(s)) for s in range(40)]
    most = max(cases.work(c)["flops"] for c in listed)
    for c in listed + drawn:
        w = cases.work(c)
        assert w["bytes"] > 0 and w["flops"] > 0
        assert w["flops"] <= most
