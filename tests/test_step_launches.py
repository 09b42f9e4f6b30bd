"""What the training step's operators launch, without a GPU: the host code of ``reft_step.hip`` and ``reft_product.hip`` as it is, on a
HIP runtime that runs nothing, notes every kernel and its grid, and refuses the grids that HIP refuses."""
import ctypes
import os
import subprocess

import pytest

import paper_2310_12670_amd as reft

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2310_12670_amd", "csrc")

RUNTIME = r"""
#include <hip/hip_runtime_api.h>
#include <cstdarg>
#include <map>
#include <string>
#include <vector>

struct Launch { std::string name; dim3 grid, block; };
static std::map<const void *, std::string> names;
static std::vector<Launch> launches;
static Launch pushed;

extern "C" {
uint64_t sim_launches() { return launches.size(); }
void sim_clear() { launches.clear(); }
const char *sim_name(uint64_t i) { return launches[i].name.c_str(); }
void sim_grid(uint64_t i, uint32_t *out)
{
    const Launch &l = launches[i];
    const uint32_t v[6] = {l.grid.x, l.grid.y, l.grid.z, l.block.x, l.block.y, l.block.z};
    for (int k = 0; k < 6; ++k) out[k] = v[k];
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) { pushed.grid = grid, pushed.block = block; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, hipStream_t *s)
{
    *grid = pushed.grid, *block = pushed.block, *shared = 0, *s = nullptr;
    return hipSuccess;
}
static hipError_t last;
hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **, size_t, hipStream_t)
{
    const uint64_t most = 0xffffffffu;
    if (!grid.x || !grid.y || !grid.z || (uint64_t)grid.x * block.x > most || (uint64_t)grid.y * block.y > most || grid.y > 65535 ||
        grid.z > 65535 || block.x * block.y * block.z > 1024)
        return last = hipErrorInvalidConfiguration;
    launches.push_back(Launch{names[f], grid, block});
    return hipSuccess;
}
hipError_t hipGetLastError() { const hipError_t e = last; last = hipSuccess; return e; }
const char *hipGetErrorString(hipError_t) { return "refused"; }
void **__hipRegisterFatBinary(const void *) { return nullptr; }
void __hipRegisterFunction(void **, const void *f, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names[f] = name; }
void __hipUnregisterFatBinary(void **) {}
char __hip_fatbin[1];
}
namespace reft { int fail(int code, const char *, ...) { return code; } }
"""

ADDRESS = 1 << 40                                            # on everything that matters; never read
E4M3, BF16, F32 = reft.REFT_E4M3, reft.REFT_BF16, reft.REFT_F32


class Library:
    def __init__(self, so):
        self.lib = ctypes.CDLL(so)
        self.lib.sim_launches.restype = self.lib.reft_product_workspace.restype = ctypes.c_uint64
        self.lib.sim_name.restype = ctypes.c_char_p
        u64, i, p = ctypes.c_uint64, ctypes.c_int, ctypes.c_void_p
        self.lib.sim_name.argtypes = [u64]
        self.lib.sim_grid.argtypes = [u64, p]
        self.lib.reft_product_workspace.argtypes = [u64, u64, u64]
        self.lib.reft_product.argtypes = [p, u64, i, p, u64, p, u64, i, p, u64, i, u64, u64, u64, p, u64, i, p, u64, p]
        self.lib.reft_quantize.argtypes = [p, u64, u64, u64, i, i, i, p, u64, p, u64, p, u64, p, u64, p]

    def launches(self):
        """(kernel, grid, block) of what was launched since the last look."""
        out = []
        for n in range(self.lib.sim_launches()):
            v = (ctypes.c_uint32 * 6)()
            self.lib.sim_grid(n, v)
            out.append((self.lib.sim_name(n).decode(), tuple(v[:3]), tuple(v[3:])))
        self.lib.sim_clear()
        return out

    def product(self, M, N, K, out=BF16, ld=None, lead=0, blocks=0):
        ld = ld or -(-K // 16) * 16
        need = self.lib.reft_product_workspace(M, N, K)
        rc = self.lib.reft_product(ADDRESS + lead, ld, E4M3, ADDRESS, M, ADDRESS, ld, E4M3, ADDRESS, -(-N // 128) if blocks else N, blocks,
                                   M, N, K, ADDRESS, N, out, ADDRESS, need, None)
        return rc, self.launches()


@pytest.fixture(scope="module")
def step(tmp_path_factory):
    d = tmp_path_factory.mktemp("step_launches")
    (d / "runtime.cpp").write_text(RUNTIME)
    objs = [str(d / "runtime.o")]
    subprocess.run(["g++", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-O1", "-std=c++17", "-fPIC", "-w", "-c", "-o", objs[0],
                    str(d / "runtime.cpp")], check=True)
    for name in ("reft_step", "reft_product"):
        objs.append(str(d / (name + ".o")))
        subprocess.run(["hipcc", "--offload-host-only", "--offload-arch=gfx950", "-fuse-cuid=none", "-O1", "-std=c++17", "-fPIC", "-w", "-c",
                        "-o", objs[-1], os.path.join(CSRC, name + ".hip")], check=True)
    so = str(d / "lib.so")
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-Wl,-z,muldefs", "-o", so, *objs], check=True)
    return Library(so)


# ---- the order of a product's sums ----------------------------------------------------------------------------------
@pytest.mark.parametrize("M,N,K", [(40, 300, 4097), (64, 512, 2048), (130, 300, 4097), (200, 300, 9001), (128, 4096, 11008), (512, 4096, 11008),
                                   (1001, 770, 5128), (300, 700, 896), (4000, 4000, 4000), (100, 40, 20)])
@pytest.mark.parametrize("out", [F32, BF16])
def test_parts_of_K_go_by_sizes_alone(step, M, N, K, out):
    """As many parts wherever the rows lie and however far apart: at 16 bytes, one byte on, in rows of an odd or a very large length."""
    cuts = set()
    for kw in ({}, dict(lead=1), dict(ld=K + K % 2 + 1), dict(ld=1 << 24)):
        rc, kernels = step.product(M, N, K, out, **kw)
        assert rc == reft.REFT_OK
        (first, grid, _), rest = kernels[0], kernels[1:]
        parts = grid[2] if "k_product_any" in first else grid[1]
        assert ("k_product_any" in first) == bool(kw)
        assert [("k_add_parts" in name) for name, _, _ in rest] == [True] * (parts > 1)
        cuts.add(parts)
    assert len(cuts) == 1
    need = step.lib.reft_product_workspace(M, N, K)
    assert need == (M * N * 4 * cuts.pop() if need else 0)


# ---- sizes that the header allows are launched ------------------------------------------------------------------------
ONE_COLUMN = [(1 << 26) - n for n in (1, 2, 3, 4, 5)]


@pytest.mark.parametrize("rows", [1, 5, 1 << 20] + ONE_COLUMN)
@pytest.mark.parametrize("blocks", [0, 1])
def test_quantize_takes_its_most_rows(step, rows, blocks):
    """One row more a block than a grid has room for would make 2^32 threads, which HIP refuses."""
    tall = -(-rows // 128) if blocks else rows
    assert step.lib.reft_quantize(ADDRESS, 1, rows, 1, F32, E4M3, blocks, ADDRESS, 1, ADDRESS, tall, None, 0, None, 0, None) == reft.REFT_OK
    ((name, grid, block),) = step.launches()
    each = 4 if "k_quantize_rows" in name else 128
    assert grid[0] == -(-rows // each)
    assert ("k_quantize_rows" in name) == (not blocks and rows <= (1 << 26) - 4)


@pytest.mark.parametrize("N", [1, 300, 1 << 20] + [(1 << 26) - n for n in (1, 15, 16, 17)] + [1 << 26, (1 << 26) + 1, 1 << 30])
@pytest.mark.parametrize("M", [1, 16])
@pytest.mark.parametrize("lead", [0, 1])
def test_product_of_few_rows_takes_its_most_columns(step, M, N, lead):
    rc, kernels = step.product(M, N, 16, lead=lead)
    assert rc == reft.REFT_OK
    ((name, grid, block),) = kernels
    few = "k_product_few" in name
    assert few == (N <= (1 << 26) - 16) and grid[0] == -(-N // (16 if few else 128))


# ---- the limits that include/reft.h states: the last size on this side, the first on the other --------------------------------
def test_limits_of_dropout(step):
    def dropout(rows, cols):
        f = step.lib.reft_dropout
        u64 = ctypes.c_uint64
        f.argtypes = [ctypes.c_void_p, u64, ctypes.c_void_p, u64, u64, u64, ctypes.c_int, ctypes.c_double, u64, u64, ctypes.c_void_p]
        rc = f(ADDRESS, cols, ADDRESS, cols, rows, cols, F32, 0.1, 1, 1, None)
        assert (rc == reft.REFT_OK) == (len(step.launches()) == 1)
        return rc
    assert dropout((1 << 31) - 1, 1) == reft.REFT_OK and dropout(1 << 31, 1) == reft.REFT_ESIZE
    assert dropout(1, (1 << 31) - 1) == reft.REFT_OK and dropout(1, 1 << 31) == reft.REFT_ESIZE
    # 2^34 - 1024 groups of eight columns: 0xffffff blocks of 1024
    assert dropout(1024, 8 * 0xFFFFFF) == reft.REFT_OK and dropout(1025, 8 * 0xFFFFFF) == reft.REFT_ESIZE
    assert dropout((1 << 30) - 64, 16 * 8) == reft.REFT_OK and dropout((1 << 30) - 63, 16 * 8) == reft.REFT_ESIZE


@pytest.mark.parametrize("blocks", [0, 1])
def test_limits_of_quantize(step, blocks):
    def quantize(rows, cols):
        tall = -(-rows // 128) if blocks else rows
        rc = step.lib.reft_quantize(ADDRESS, cols, rows, cols, F32, E4M3, blocks, ADDRESS, cols, ADDRESS, tall, None, 0, None, 0, None)
        assert (rc == reft.REFT_OK) == (len(step.launches()) == 1)
        return rc
    assert quantize((1 << 26) - 1, 31 * 128) == reft.REFT_OK and quantize((1 << 26) - 1, 32 * 128) == reft.REFT_ESIZE
    assert quantize(1 << 26, 1) == reft.REFT_ESIZE
    assert quantize(256 * 128, 128 * 65535) == reft.REFT_OK and quantize(256 * 128 + 1, 128 * 65535) == reft.REFT_ESIZE
    assert quantize(1, 128 * 65535 + 1) == reft.REFT_ESIZE


def test_limits_of_the_product(step):
    last = 128 * 0xFFFFFF
    assert step.product(64, last, 16)[0] == reft.REFT_OK and step.product(64, last + 1, 16)[0] == reft.REFT_ESIZE
    assert step.product(1, last, 16, lead=1)[0] == reft.REFT_OK
    assert step.product(65, 1 << 30, 16)[0] == reft.REFT_ESIZE and step.product(65, (1 << 30) - 128, 16)[0] == reft.REFT_OK
    assert step.product(128 * 65535, 128 * 128, 16)[0] == reft.REFT_OK and step.product(128 * 65535, 128 * 129, 16)[0] == reft.REFT_ESIZE
    assert step.product(128 * 65535 + 1, 1, 16)[0] == reft.REFT_ESIZE
    assert step.product(1, 1, (1 << 31) - 1)[0] == reft.REFT_OK and step.product(1, 1, 1 << 31)[0] == reft.REFT_ESIZE
