"""The binding's two ways to the library, its C part and its Python part, hand over the same arguments (CPU): both run against a library that
writes down what it is called with."""
import ctypes
import importlib.util
import itertools
import os
import re
import subprocess
import sysconfig

import pytest
import torch

import paper_2310_12670_amd as reft
from paper_2310_12670_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F8 = torch.float8_e4m3fn, torch.float8_e5m2
NAMES = ["reft_heads_forward", "reft_heads_backward", "reft_gate_forward", "reft_gate_backward", "reft_transpose"]
REST = ["reft_dropout", "reft_norm_forward", "reft_norm_backward", "reft_quantize", "reft_product"]


def stub(names):
    """A C file with those functions of include/reft.h, each of which appends its arguments to a text."""
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "reft.h")).read(), flags=re.S)
    out = ['#include "%s"' % os.path.join(ROOT, "include", "reft.h"), "#include <stdio.h>", "#include <stdarg.h>",
           "static char said[1 << 16]; static int at;",
           "const char *stub_said(void) { return said; }", "void stub_clear(void) { at = 0; said[0] = 0; }",
           "int hipGetDevice(int *d) { *d = 0; return 0; }",
           "static void tell(const char *f, ...) { va_list v; va_start(v, f); at += vsnprintf(said + at, sizeof said - at, f, v); va_end(v); }",
           'static void heads(const char *n, const reft_heads *h) { if (h) tell(" %s=(%p %llu %llu)", n, h->p, (unsigned long long)h->row, '
           '(unsigned long long)h->head); else tell(" %s=none", n); }',
           'static void eight(const char *n, const reft_eight *e) { if (e && e->q) tell(" %s=(%p %llu %p %llu)", n, e->q, (unsigned long long)e->ld, '
           'e->scales, (unsigned long long)e->ld_s); else tell(" %s=none", n); }']
    for name in names:
        args = re.search(r"int %s\(([^;]*)\);" % name, header).group(1)
        body = []
        for arg in (" ".join(a.split()) for a in args.split(",")):
            kind, var = re.match(r"(.*?[ *])(\w+)$", arg).groups()
            if "reft_heads" in kind:
                body.append('heads("%s", %s);' % (var, var))
            elif "reft_eight" in kind:
                body.append('eight("%s", %s);' % (var, var))
            elif "*" in kind or "reft_stream" in kind:
                body.append('tell(" %s=%%p", (void *)%s);' % (var, var))
            elif "double" in kind:
                body.append('tell(" %s=%%.17g", %s);' % (var, var))
            elif "uint64_t" in kind:
                body.append('tell(" %s=%%llu", (unsigned long long)%s);' % (var, var))
            else:
                body.append('tell(" %s=%%d", %s);' % (var, var))
        out.append("int %s(%s) { %s return 0; }" % (name, args, " ".join(body)))
    return "\n".join(out)


@pytest.fixture(scope="module")
def both(tmp_path_factory):
    """(the C part on the stub, the stub)"""
    d = tmp_path_factory.mktemp("marshal")
    (d / "stub.c").write_text(stub(NAMES + REST))
    # a name of its own: one that is loaded already would stand for it
    subprocess.run(["gcc", "-O1", "-w", "-fPIC", "-shared", "-o", str(d / "libstub.so"), str(d / "stub.c")], check=True)
    out = str(d / ("_marshal" + sysconfig.get_config_var("EXT_SUFFIX")))
    subprocess.run(["gcc", "-O2", "-std=c11", "-Wall", "-Wextra", "-Wno-unused-parameter", "-Wno-missing-field-initializers", "-Werror", "-fPIC",
                    "-shared", "-I", sysconfig.get_paths()["include"], "-o", out, os.path.join(build.CSRC, "reft_marshal.c"), "-L", str(d),
                    "-l:libstub.so", "-Wl,-rpath,$ORIGIN"], check=True)
    spec = importlib.util.spec_from_file_location("_marshal", out)
    part = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(part)
    for t, code in ((torch.float32, 0), (torch.bfloat16, 1), (torch.float16, 2), (F8[0], 3), (F8[1], 4), (torch.int64, 5)):
        part.know(t, code)
    lib = ctypes.CDLL(str(d / "libstub.so"))
    lib.stub_said.restype = ctypes.c_char_p
    real = reft.binding._load()
    for name in NAMES + REST:
        getattr(lib, name).argtypes = getattr(real, name).argtypes
    return part, lib


class OnTheGpu:
    """A tensor that says it is on GPU 0."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


def gpu(*shape, dtype=torch.float32):
    if dtype in F8:
        return OnTheGpu(torch.zeros(*shape, dtype=torch.uint8).view(dtype))
    return OnTheGpu(torch.zeros(*shape, dtype=dtype))


def eight(rows, cols, dtype=F8[0]):
    return gpu(rows, cols, dtype=dtype), gpu(-(-cols // 512), rows, 4, dtype=torch.uint8)


class NoPart:
    """In place of the C part: it takes no call, and stays where it is."""

    def know(self, *_):
        pass

    def __getattr__(self, name):
        return lambda *args: None


class Only:
    """The C part, which has to take every call."""

    def __init__(self, part):
        self.part = part

    def know(self, *args):
        self.part.know(*args)

    def __getattr__(self, name):
        def call(*args):
            rc = getattr(self.part, name)(*args)
            assert rc is not None, name + " left the call to the Python part"
            return rc
        return call


def heads_calls():
    for dtype, with_k, by_head, wide_weight in itertools.product((torch.float32, torch.bfloat16), (True, False), (True, False), (True, False)):
        def room(h, dtype=dtype, by_head=by_head):
            return OnTheGpu(torch.zeros(h, 5, 32, dtype=dtype).transpose(0, 1)) if by_head else gpu(5, h, 32, dtype=dtype)
        q, qo, dq = room(6), room(6), room(6)
        k, ko, dk = (room(2), room(2), room(2)) if with_k else (None, None, None)
        w = gpu(32, dtype=torch.float32 if wide_weight else dtype), gpu(32, dtype=torch.float32 if wide_weight else dtype)
        at = gpu(5, dtype=torch.int64), gpu(12)
        yield lambda q=q, k=k, w=w, at=at, qo=qo, ko=ko: reft.reft_heads_forward(q, k, *w, *at, 1e-5, qo, ko, adjacent=by_head, stream=77)
        yield lambda q=q, k=k, w=w, at=at, qo=qo, ko=ko: reft.reft_heads_forward(q, k, None, w[1], *at, 1e-5, qo, ko)
        for some in range(4):
            kw = dict(dq=dq if some & 1 else None, dq_weight=gpu(32) if some & 2 else None, workspace=gpu(4096, dtype=torch.uint8))
            if with_k:
                kw.update(dk=dk if some != 1 else None, dk_weight=gpu(32) if some == 3 else None)
            yield lambda q=q, k=k, w=w, at=at, qo=qo, ko=ko, kw=kw: reft.reft_heads_backward(qo, ko, q, k, *w, *at, 1e-6, adjacent=True, stream=3, **kw)


def gate_calls():
    def call(fn, *args, **kw):
        return lambda: fn(*args, **kw)
    for dtype, gated, kept in itertools.product((torch.float16, torch.float32), (True, False), F8):
        r, c = 9, 640
        g, u, y = gpu(r, c, dtype=dtype), gpu(r, c, dtype=dtype) if gated else None, gpu(r, c, dtype=dtype)
        for i, act in enumerate(("silu", "gelu", "gelu_tanh", "relu2", 2)):
            yield call(reft.reft_gate_forward, g, u, act, y=y if i & 1 else None, y8=eight(r, c, F8[i & 1]) if i & 2 else None,
                       g8=eight(r, c, kept) if i != 3 else None, u8=eight(r, c, kept) if gated and i else None, stream=5)
        for i in range(32):
            outs = dict(dg=gpu(r, c, dtype=dtype) if i & 1 else None, dg8=eight(r, c) if i & 2 else None, dg8_t=eight(c, r) if i & 4 else None,
                        y8_t=eight(c, r, F8[1]) if i & 8 else None)
            if gated:
                outs.update(du=gpu(r, c, dtype=dtype) if i & 16 else None, du8=eight(r, c) if i & 1 else None, du8_t=eight(c, r) if i & 2 else None)
            yield call(reft.reft_gate_backward, y, eight(r, c, kept), eight(r, c, kept) if gated else None, "gelu", stream=9, **outs)
    for a, b in itertools.product(F8, F8):
        yield call(reft.reft_transpose, *eight(700, 33, a), *eight(33, 700, b), stream=8)


@pytest.mark.parametrize("calls", [heads_calls, gate_calls])
def test_both_parts_hand_over_the_same(both, monkeypatch, calls):
    part, lib = both
    monkeypatch.setattr(reft.binding, "_load", lambda: lib)
    monkeypatch.setattr(reft.binding, "_seen", lambda t: True)
    count = 0
    for call in calls():
        said = []
        for way in (Only(part), NoPart()):
            monkeypatch.setattr(reft.binding, "_marshal", way)
            lib.stub_clear()
            call()
            said.append(lib.stub_said().decode())
        assert said[0] and said[0] == said[1]
        count += 1
    assert count > 40
