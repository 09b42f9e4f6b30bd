"""What the operators inside the sublayers refuse, before anything reaches the GPU (CPU tensors serve as operands), and what they launch at
the ends of their ranges."""
import ctypes

import pytest
import torch

import paper_2310_12670_amd as reft
from test_step_launches import ADDRESS, RUNTIME, Library  # noqa: F401

E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2


def pair(rows, cols, dtype=E4):
    return torch.zeros(rows, cols, dtype=torch.uint8).view(dtype), torch.zeros(-(-cols // 512), rows, 4, dtype=torch.uint8)


def refused(code, fn, *args, **kw):
    with pytest.raises(reft.ReftError) as e:
        fn(*args, **kw)
    assert e.value.code == code and len(e.value.message) > 10
    return e.value.message


EINVAL, ESIZE = reft.REFT_EINVAL, reft.REFT_ESIZE


def test_heads_forward():
    x, k, w = torch.zeros(4, 3, 16), torch.zeros(4, 2, 16), torch.ones(16)
    at, f = torch.zeros(4, dtype=torch.int64), torch.ones(8)
    y, yk = torch.zeros_like(x), torch.zeros_like(k)
    call = reft.reft_heads_forward
    assert "cpu" in refused(EINVAL, call, x, k, w, w, at, f, 1e-5, y, yk)                       # right but for the memory
    assert "cpu" in refused(EINVAL, call, x, None, None, None, None, None, 0.0, y)
    refused(EINVAL, call, x, k, w, w, at, f, 1e-5, y)                                           # k without k_out
    refused(EINVAL, call, x, None, w, w, at, f, 1e-5, y, yk)
    refused(EINVAL, call, x, k.half(), w, w, at, f, 1e-5, y, yk)
    refused(EINVAL, call, x, torch.zeros(5, 2, 16), w, w, at, f, 1e-5, y, torch.zeros(5, 2, 16))
    refused(EINVAL, call, x, torch.zeros(4, 2, 15), w, w, at, f, 1e-5, y, yk)
    refused(EINVAL, call, x[0], None, w, w, at, f, 1e-5, y)
    refused(EINVAL, call, x.double(), None, w, w, at, f, 1e-5, y.double())
    refused(EINVAL, call, x, None, w.half(), None, at, f, 1e-5, y)
    refused(EINVAL, call, x.half(), k.half(), w, w.half(), at, f, 1e-5, y.half(), yk.half())    # weights of two types
    refused(EINVAL, call, x, None, torch.ones(15), None, at, f, 1e-5, y)
    refused(EINVAL, call, x, None, w, None, at.to(torch.int32), f, 1e-5, y)
    refused(EINVAL, call, x, None, w, None, at[:3], f, 1e-5, y)
    refused(EINVAL, call, x, None, w, None, torch.zeros(8, dtype=torch.int64)[::2], f, 1e-5, y)
    refused(EINVAL, call, x, None, w, None, None, f, 1e-5, y)
    refused(EINVAL, call, x, None, w, None, at, f.double(), 1e-5, y)
    refused(ESIZE, call, x, None, w, None, at, torch.ones(9), 1e-5, y)
    refused(EINVAL, call, x, None, w, None, at, f, -1.0, y)
    refused(EINVAL, call, x, None, w, None, at, f, float("nan"), y)
    refused(EINVAL, call, x.transpose(1, 2), None, torch.ones(3), None, at, torch.ones(1), 1e-5, torch.zeros(4, 16, 3))
    refused(ESIZE, call, torch.zeros(1, 1, 513), None, None, None, None, None, 1e-5, torch.zeros(1, 1, 513))
    refused(ESIZE, call, torch.zeros(1, 1, 0), None, None, None, None, None, 1e-5, torch.zeros(1, 1, 0))
    refused(ESIZE, call, torch.zeros(1, 0, 8), None, None, None, None, None, 1e-5, torch.zeros(1, 0, 8))
    for wrong in (7, [1.0], "x"):
        refused(EINVAL, call, wrong, None, None, None, None, None, 1e-5, y)
        refused(EINVAL, call, x, None, None, None, None, None, 1e-5, wrong)
        refused(EINVAL, call, x, None, wrong, None, None, None, 1e-5, y)
    call(torch.zeros(0, 3, 16), None, None, None, torch.zeros(0, dtype=torch.int64), torch.zeros(0), 1e-5, torch.zeros(0, 3, 16))


@pytest.mark.parametrize("shape,strides", [((4, 3, 16), (48, 15, 1)), ((4, 3, 16), (47, 16, 1)), ((4, 3, 16), (16, 63, 1)), ((4, 3, 16), (16, 16, 1)),
                                           ((4, 3, 16), (0, 16, 1)), ((4, 3, 16), (64, 0, 1)), ((4, 1, 16), (15, 16, 1)), ((1, 3, 16), (0, 8, 1))])
def test_results_that_overlap_themselves(shape, strides):
    """Elements that share a place: the last to be written would be a matter of timing."""
    out = torch.zeros(1000).as_strided(shape, strides)
    x = torch.zeros(shape)
    assert "overlap" in refused(ESIZE, reft.reft_heads_forward, x, None, None, None, None, None, 1e-5, out)
    assert "overlap" in refused(ESIZE, reft.reft_heads_backward, x, None, x, None, None, None, None, None, 1e-5, dq=out)
    assert "cpu" in refused(EINVAL, reft.reft_heads_forward, out, None, None, None, None, None, 1e-5, x)      # inputs may


@pytest.mark.parametrize("shape,strides", [((4, 3, 16), (48, 16, 1)), ((4, 3, 16), (16, 64, 1)), ((4, 3, 16), (100, 20, 1)), ((1, 3, 16), (0, 16, 1)),
                                           ((4, 1, 16), (16, 0, 1)), ((1, 1, 16), (0, 0, 1)), ((4, 3, 1), (3, 1, 7))])
def test_results_apart(shape, strides):
    out = torch.zeros(1000).as_strided(shape, strides)
    assert "cpu" in refused(EINVAL, reft.reft_heads_forward, torch.zeros(shape), None, None, None, None, None, 1e-5, out)


def test_heads_backward():
    x, k, w = torch.zeros(4, 3, 16), torch.zeros(4, 2, 16), torch.ones(16)
    at, f = torch.zeros(4, dtype=torch.int64), torch.ones(8)
    call = reft.reft_heads_backward
    need = reft.reft_heads_backward_workspace(4, 3, 2, 16)
    assert need > 0 and reft.reft_heads_backward_workspace(0, 3, 2, 16) == 0
    room = torch.zeros(need + 16, dtype=torch.uint8)
    args = (x, k, x, k, w, w, at, f, 1e-5)
    full = dict(dq=x, dk=k, dq_weight=w, dk_weight=w)
    assert "cpu" in refused(EINVAL, call, *args, **full, workspace=room[:need])
    refused(EINVAL, call, *args)                                                                # no output
    assert "workspace" in refused(EINVAL, call, *args, **full)
    assert "16 bytes" in refused(EINVAL, call, *args, dq_weight=w, workspace=room[8:])
    assert "too small" in refused(ESIZE, call, *args, dk_weight=w, workspace=room[:need - 1])
    assert "contiguous" in refused(EINVAL, call, *args, dk_weight=w, workspace=torch.zeros(2 * need, dtype=torch.uint8)[::2])
    assert "cpu" in refused(EINVAL, call, *args, dq=x)                                          # no sums: no workspace
    refused(EINVAL, call, x, None, x, k, w, w, at, f, 1e-5, dq=x)
    for kw in (dict(dk=k), dict(dk_weight=w)):
        refused(EINVAL, call, x, None, x, None, w, None, at, f, 1e-5, dq=x, workspace=room, **kw)
    refused(EINVAL, call, *args, dq=x.half())
    refused(EINVAL, call, *args, dq=k)
    refused(EINVAL, call, *args, dq_weight=w.half(), workspace=room)
    refused(EINVAL, call, x.half(), k, x, k, w, w, at, f, 1e-5, dq=x)
    refused(ESIZE, call, *args[:7], torch.ones(9), 1e-5, dq=x)
    # the workspace says no more than the call asks for, and grows no further than the chip's blocks
    assert reft.reft_heads_backward_workspace(1 << 20, 64, 8, 128) <= 512 * 2 * 128 * 4


def test_gate_forward():
    g, u = torch.zeros(4, 8), torch.zeros(4, 8)
    call = reft.reft_gate_forward
    assert "cpu" in refused(EINVAL, call, g, u, "silu", y=g, y8=pair(4, 8), g8=pair(4, 8), u8=pair(4, 8))
    assert "cpu" in refused(EINVAL, call, g, u, reft.REFT_RELU2, g8=pair(4, 8, E5), y8=pair(4, 8))
    for act in ("relu", "", None, 1.5, -1, 4, ["silu"]):
        refused(EINVAL, call, g, u, act, y=g)
    refused(EINVAL, call, g, u, "silu")                                                         # no output
    refused(EINVAL, call, g, None, "silu", u8=pair(4, 8))                                       # u8 without u
    refused(EINVAL, call, g, u, "silu", g8=pair(4, 8), u8=pair(4, 8, E5))                       # two formats
    refused(EINVAL, call, g, u.half(), "silu", y=g)
    refused(EINVAL, call, g, torch.zeros(4, 9), "silu", y=g)
    refused(EINVAL, call, g, u, "silu", y=g.half())
    refused(EINVAL, call, g, u, "silu", y8=pair(8, 4))
    refused(EINVAL, call, g, u, "silu", y8=pair(4, 8)[0])
    refused(EINVAL, call, g, u, "silu", y8=(pair(4, 8)[0], None))
    refused(EINVAL, call, g, u, "silu", y8=(pair(4, 8)[0], torch.zeros(1, 5, 4, dtype=torch.uint8)))
    refused(EINVAL, call, g, u, "silu", y8=(g, pair(4, 8)[1]))
    refused(EINVAL, call, g.t(), None, "silu", y=torch.zeros(8, 4))
    refused(EINVAL, call, g.to(torch.int32), None, "silu", y=g.to(torch.int32))
    call(torch.zeros(0, 8), None, "gelu", y=torch.zeros(0, 8))
    call(torch.zeros(4, 0), None, "gelu", y=torch.zeros(4, 0))
    lib, a = reft.binding._load(), g.data_ptr()
    f = lambda at=a, ld=8, rows=4, cols=8, dtype=0, act=0, y=a, ld_y=8: lib.reft_gate_forward(   # noqa: E731
        at, ld, None, 0, rows, cols, dtype, act, y, ld_y, None, -1, None, None, -1, reft.binding._CHECK_ONLY)
    assert f() == reft.REFT_OK and f(ld=7) == ESIZE and f(ld_y=7) == ESIZE and f(at=a + 1) == EINVAL and f(y=a + 2) == EINVAL
    assert f(dtype=3) == EINVAL and f(act=4) == EINVAL and f(at=None) == EINVAL and f(rows=2 ** 31) == ESIZE
    e = reft.binding._Eight(a, 8, a, 4)
    h = lambda e=e, fmt=3: lib.reft_gate_forward(a, 8, None, 0, 4, 8, 0, 0, None, 0, ctypes.byref(e), fmt, None, None, -1,   # noqa: E731
                                                 reft.binding._CHECK_ONLY)
    assert h() == reft.REFT_OK and h(fmt=1) == EINVAL
    assert h(reft.binding._Eight(a, 7, a, 4)) == ESIZE and h(reft.binding._Eight(a, 8, a, 3)) == ESIZE and h(reft.binding._Eight(a, 8, None, 4)) == EINVAL


def test_gate_backward():
    dy = torch.zeros(4, 8)
    g8, u8 = pair(4, 8), pair(4, 8)
    call = reft.reft_gate_backward
    assert "cpu" in refused(EINVAL, call, dy, g8, u8, "silu", dg=dy, du=torch.zeros(4, 8), dg8=pair(4, 8, E5), du8=pair(4, 8, E5), dg8_t=pair(8, 4, E5),
                            du8_t=pair(8, 4, E5), y8_t=pair(8, 4))
    refused(EINVAL, call, dy, g8, u8, "silu")
    refused(EINVAL, call, dy, None, u8, "silu", dg=dy)
    refused(EINVAL, call, dy, g8, pair(4, 8, E5), "silu", dg=dy)
    for kw in (dict(du=dy), dict(du8=pair(4, 8)), dict(du8_t=pair(8, 4))):
        refused(EINVAL, call, dy, g8, None, "silu", **kw)
    refused(EINVAL, call, dy, g8, u8, "silu", dg8=pair(4, 8), du8=pair(4, 8, E5))
    refused(EINVAL, call, dy, g8, u8, "silu", dg8_t=pair(4, 8))
    refused(EINVAL, call, dy, pair(4, 9), u8, "silu", dg=dy)
    refused(EINVAL, call, dy, g8, u8, "tanh", dg=dy)
    refused(EINVAL, call, dy, g8, u8, "silu", dg=dy.half())
    call(torch.zeros(0, 8), pair(0, 8), None, "silu", dg=torch.zeros(0, 8))


def test_transpose():
    call = reft.reft_transpose
    assert "cpu" in refused(EINVAL, call, *pair(4, 8), *pair(8, 4, E5))
    refused(EINVAL, call, *pair(4, 8), *pair(4, 8))
    refused(EINVAL, call, *pair(4, 8), pair(8, 4)[0], pair(4, 8)[1])
    refused(EINVAL, call, pair(4, 8)[0], None, *pair(8, 4))
    refused(EINVAL, call, pair(4, 8)[0].float(), pair(4, 8)[1], *pair(8, 4))
    refused(EINVAL, call, *pair(4, 8), 5, pair(8, 4)[1])
    call(*pair(0, 8), *pair(8, 0))


# ---- what is launched (no GPU: see test_step_launches) -----------------------------------------------------------------
@pytest.fixture(scope="module")
def inside(tmp_path_factory):
    import os
    import subprocess
    d = tmp_path_factory.mktemp("inside_launches")
    (d / "runtime.cpp").write_text(RUNTIME)
    objs = [str(d / "runtime.o")]
    subprocess.run(["g++", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-O1", "-std=c++17", "-fPIC", "-w", "-c", "-o", objs[0],
                    str(d / "runtime.cpp")], check=True)
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_12670_amd", "csrc")
    for name in ("reft_step", "reft_product", "reft_heads", "reft_gate"):
        objs.append(str(d / (name + ".o")))
        subprocess.run(["hipcc", "--offload-host-only", "--offload-arch=gfx950", "-fuse-cuid=none", "-O1", "-std=c++17", "-fPIC", "-w", "-c",
                        "-o", objs[-1], os.path.join(csrc, name + ".hip")], check=True)
    so = str(d / "lib.so")
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-Wl,-z,muldefs", "-o", so, *objs], check=True)
    lib = Library(so)
    real = reft.binding._load()
    for name in ("reft_heads_forward", "reft_heads_backward", "reft_heads_backward_workspace", "reft_gate_forward", "reft_gate_backward",
                 "reft_transpose"):
        getattr(lib.lib, name).argtypes, getattr(lib.lib, name).restype = getattr(real, name).argtypes, getattr(real, name).restype
    return lib


def heads(lib, rows, q, k, cols, dtype=reft.REFT_BF16, back=False, adjacent=0):
    H = reft.binding._Heads
    x, y = ctypes.byref(H(ADDRESS, (q + k) * cols, cols)), (ctypes.byref(H(ADDRESS, (q + k) * cols, cols)) if k else None)
    if not back:
        return lib.lib.reft_heads_forward(x, q, y, k, None, None, ADDRESS, ADDRESS, cols // 2, adjacent, rows, cols, dtype, dtype, 1e-5, x, y, None)
    need = lib.lib.reft_heads_backward_workspace(rows, q, k, cols)
    return lib.lib.reft_heads_backward(x, y, x, q, y, k, None, None, ADDRESS, ADDRESS, cols // 2, adjacent, rows, cols, dtype, dtype, 1e-5, x, y, ADDRESS,
                                       ADDRESS if k else None, ADDRESS, need, None)


@pytest.mark.parametrize("rows", [1, 2, 5, 100, 1001, 4096, 16384, 1 << 20, (1 << 31) - 1])
@pytest.mark.parametrize("q,k", [(1, 0), (1, 1), (9, 3), (64, 8), (65535, 65535)])
@pytest.mark.parametrize("cols", [1, 64, 80, 128, 200, 512])
def test_heads_are_launched_at_every_size(inside, rows, q, k, cols):
    """The grid fits, and the gradients' parts fit the workspace that is asked for."""
    inside.launches()
    assert heads(inside, rows, q, k, cols) == reft.REFT_OK
    ((name, grid, block),) = inside.launches()
    assert "k_heads_forward" in name and block[0] == 256
    assert heads(inside, rows, q, k, cols, back=True) == reft.REFT_OK
    (first, grid, _), (second, _, _) = inside.launches()
    assert "k_heads_backward" in first and "k_heads_weights" in second
    assert inside.lib.reft_heads_backward_workspace(rows, q, k, cols) == grid[0] * 2 * cols * 4 and 1 <= grid[0] <= 512


def test_limits_of_heads(inside):
    assert heads(inside, 1 << 31, 1, 0, 8) == ESIZE and heads(inside, 1, 65536, 0, 8) == ESIZE and heads(inside, 1, 1, 65536, 8) == ESIZE
    assert heads(inside, 1, 1, 0, 513) == ESIZE and heads(inside, 1, 1, 0, 512) == reft.REFT_OK
    inside.launches()


def eight(cols, rows):
    return ctypes.byref(reft.binding._Eight(ADDRESS, cols, ADDRESS, rows))


def test_limits_of_the_gate(inside):
    def forward(rows, cols):
        rc = inside.lib.reft_gate_forward(ADDRESS, cols, None, 0, rows, cols, 0, 0, ADDRESS, cols, None, -1, None, None, -1, None)
        assert (rc == reft.REFT_OK) == (len(inside.launches()) == 1)
        return rc

    def backward(rows, cols):
        rc = inside.lib.reft_gate_backward(ADDRESS, cols, eight(cols, rows), None, 3, rows, cols, 0, 0, ADDRESS, cols, None, 0, None, None, None, None,
                                           -1, eight(rows, cols), 3, None)
        assert (rc == reft.REFT_OK) == (len(inside.launches()) == 1)
        return rc

    def transpose(rows, cols):
        rc = inside.lib.reft_transpose(eight(cols, rows), 3, rows, cols, eight(rows, cols), 3, None)
        assert (rc == reft.REFT_OK) == (len(inside.launches()) == 1)
        return rc
    inside.launches()
    # 2^26 - 4 waves of 512 columns
    assert forward((1 << 26) - 4, 512) == reft.REFT_OK and forward((1 << 26) - 3, 512) == ESIZE
    assert forward(15, (1 << 31) - 1) == reft.REFT_OK and forward(1, 1 << 31) == ESIZE and forward(1 << 31, 1) == ESIZE
    for f in (backward, transpose):
        # 2^23 - 1 tiles
        assert f(128, 128 * 0x7FFFFF) == reft.REFT_OK and f(129, 128 * 0x7FFFFF) == ESIZE and f(128, 128 * 0x7FFFFF + 1) == ESIZE
        assert f(128 * 0x7FFFFF, 128) == reft.REFT_OK and f(128 * 0x7FFFFF + 1, 128) == ESIZE
        assert f(1 << 31, 1) == ESIZE and f(1, 1 << 31) == ESIZE


# ---- memory that the current GPU does not see -------------------------------------------------------------------------------
def test_another_gpus_memory_is_refused():
    from test_step_operands import Elsewhere
    far = lambda t: Elsewhere(t)                                                         # noqa: E731
    x, w, e = torch.zeros(4, 3, 16), torch.ones(16), pair(4, 48)
    at, f = torch.zeros(4, dtype=torch.int64), torch.ones(8)
    flat = torch.zeros(4, 48)
    away = lambda p: (far(p[0]), far(p[1]))                                                # noqa: E731
    calls = [lambda: reft.reft_heads_forward(far(x), None, far(w), None, far(at), far(f), 1e-5, far(x)),
             lambda: reft.reft_heads_backward(far(x), None, far(x), None, None, None, far(at), far(f), 1e-5, dq=far(x)),
             lambda: reft.reft_gate_forward(far(flat), None, "silu", y8=away(e)),
             lambda: reft.reft_gate_backward(far(flat), away(e), None, "silu", dg=far(flat)),
             lambda: reft.reft_transpose(*away(e), *away(pair(48, 4)))]
    for call in calls:
        for _ in range(2):
            assert "cuda:77" in refused(EINVAL, call)
