"""How a product is cut when the device does not tell how many clusters it runs, against a CUDA
runtime that refuses the question: an error, not another plan than the next call's."""
import os
import shutil
import subprocess
import sys
import textwrap

import pytest

from paper_2608_01127_gb300 import _build

RUNTIME = r"""
#include <cuda.h>
#include <cuda_runtime_api.h>
static int refuse = 0, asked = 0, none_from = 9, grid = 0, cluster = 0;
static cudaError_t last = cudaSuccess;
static CUresult encode(...) { return CUDA_SUCCESS; }
extern "C" {
void fake(int refuse_, int none_from_) { refuse = refuse_; none_from = none_from_; }
int fake_grid() { int n = grid; grid = 0; return n; }
int fake_cluster() { return cluster; }
int fake_asked() { int n = asked; asked = 0; return n; }
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaSetDevice(int) { return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, enum cudaDeviceAttr, int) { *v = 152; return cudaSuccess; }
cudaError_t cudaGetSymbolAddress(void** p, const void*) { *p = (void*)0x100000; return cudaSuccess; }
cudaError_t cudaGetDriverEntryPointByVersion(const char*, void** p, unsigned, unsigned long long,
                                             enum cudaDriverEntryPointQueryResult* r) {
  *p = (void*)encode;
  *r = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void*, enum cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t* c) {
  ++asked;
  if (refuse) return last = cudaErrorMemoryAllocation;
  int r = 1;
  for (unsigned i = 0; i < c->numAttrs; ++i)
    if (c->attrs[i].id == cudaLaunchAttributeClusterDimension) r = c->attrs[i].val.clusterDim.x;
  *n = r >= none_from ? 0 : 152 / r - (r > 2) * 4;
  return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void*, void**) {
  grid = c->gridDim.x;
  cluster = 1;
  for (unsigned i = 0; i < c->numAttrs; ++i)
    if (c->attrs[i].id == cudaLaunchAttributeClusterDimension) cluster = c->attrs[i].val.clusterDim.x;
  return last;
}
cudaError_t cudaGetLastError() { cudaError_t e = last; last = cudaSuccess; return e; }
}
"""

CALLS = """
    import ctypes
    fake, lib = ctypes.CDLL({fake!r}), ctypes.CDLL({lib!r})
    lib.mw_last_error.restype = ctypes.c_char_p
    P = ctypes.c_void_p(0x10000)
    for refuse in {refusals}:
        fake.fake(refuse, {none_from})
        for M, N, K, T in ((8, 2560, 10240, 0), (64, 7680, 2560, 0), (301, 1152, 1152, 0), (2304, 768, 14080, 1)):
            code = lib.mw_scaled_matmul(P, P, 0, T, P, P, 0, T, P, M, N, K, 1, None)
            print(refuse, code, fake.fake_grid(), fake.fake_cluster(), fake.fake_asked(), lib.mw_last_error().decode())
"""


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    lib = _build.build()
    folder = tmp_path_factory.mktemp("runtime")
    source, fake = folder / "runtime.cpp", folder / "runtime.so"
    source.write_text(RUNTIME)
    cuda = os.path.dirname(os.path.dirname(_build._nvcc()))
    subprocess.run(["g++", "-shared", "-fPIC", "-I" + cuda + "/include", str(source), "-o", str(fake)],
                   check=True, capture_output=True)

    def run(refusals, none_from=9):
        code = textwrap.dedent(CALLS.format(fake=str(fake), lib=lib, refusals=refusals, none_from=none_from))
        r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True,
                           env={**os.environ, "LD_PRELOAD": str(fake)})
        assert r.returncode == 0, r.stderr[-2000:]
        return [line.split(maxsplit=5) for line in r.stdout.splitlines()]
    return run


def test_a_device_that_does_not_tell(runtime):
    good = runtime((0,))
    assert [line[1] for line in good] == ["0"] * 4
    lines = runtime((1, 0))
    for line in lines[:4]:
        assert line[1] == "3" and line[2] == "0" and "clusters" in line[5]
    # the call after it as if nothing had been
    assert [line[1:4] for line in lines[4:]] == [line[1:4] for line in good]


def test_it_is_asked_once(runtime):
    lines = runtime((0, 0))
    assert sum(int(line[4]) for line in lines[:4]) == 8 and sum(int(line[4]) for line in lines[4:]) == 0


def test_clusters_that_the_device_cannot_run(runtime):
    assert any(int(line[3]) >= 4 for line in runtime((0,)))
    lines = runtime((0,), none_from=4)
    assert [line[1] for line in lines] == ["0"] * 4 and all(int(line[3]) < 4 for line in lines)
