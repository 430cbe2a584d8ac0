"""A call whose first kernel could not be launched launches nothing behind it: no kernel reads a
workspace that was not written, no count grows over rows that were not.  On the CPU: the store's
and the tree attention's host code with a CUDA runtime whose n-th launch fails."""
import os
import subprocess

import pytest

from paper_2608_21541_gb300 import build as B

# a runtime that counts launches, of which the n-th fails
RUNTIME = r"""
#include <cuda_runtime.h>

int launches = 0, fails = 0;
cudaError_t last = cudaSuccess;
static cudaError_t launch() {
  if (++launches == fails) last = cudaErrorInvalidValue;
  return launches == fails ? cudaErrorInvalidValue : cudaSuccess;
}
extern "C" {
cudaError_t CUDARTAPI cudaLaunchKernel(const void*, dim3, dim3, void**, size_t, cudaStream_t) { return launch(); }
cudaError_t CUDARTAPI cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void**) { return launch(); }
cudaError_t CUDARTAPI cudaGetLastError() { const cudaError_t e = last; last = cudaSuccess; return e; }
cudaError_t CUDARTAPI __cudaLaunchKernel(cudaKernel_t, dim3, dim3, void**, size_t, cudaStream_t) { return launch(); }
cudaError_t CUDARTAPI __cudaGetKernel(cudaKernel_t*, const void*) { return cudaSuccess; }
unsigned CUDARTAPI __cudaPushCallConfiguration(dim3, dim3, size_t, CUstream_st*) { return 0; }
cudaError_t CUDARTAPI __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return cudaSuccess; }
void** CUDARTAPI __cudaRegisterFatBinary(void*) { static void* h; return &h; }
void CUDARTAPI __cudaRegisterFatBinaryEnd(void**) {}
void CUDARTAPI __cudaUnregisterFatBinary(void**) {}
void CUDARTAPI __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
void CUDARTAPI __cudaRegisterVar(void**, char*, char*, const char*, int, size_t, int, int) {}
char CUDARTAPI __cudaInitModule(void**) { return 0; }
}
"""

CALLS_IN_C = r"""
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include "internal.cuh"
#include "tree.cuh"

extern int launches, fails;
extern cudaError_t last;
namespace certkv {
void trace_begin(const char*, cudaStream_t) {}
void trace_end(cudaStream_t) {}
int tree_ctas() { return 152; }
int tree_mma_ctas(int) { return 304; }
__global__ void some_kernel(int) {}
bool launch_tree_tc(const TreeArgs&, int, cudaStream_t st) { return launch_kernel(true, some_kernel, 1, 32, 0, st, 1); }
bool launch_tree_mma(const TreeArgs&, int, cudaStream_t st) { return launch_kernel(true, some_kernel, 1, 32, 0, st, 1); }
}  // namespace certkv

int main(int argc, char** argv) {
  fails = atoi(argv[2]);
  const int units = atoi(argv[3]), tokens = atoi(argv[4]);
  void* fake = (void*)(1 << 20);
  certkv_store st = {units, CERTKV_STORE_FP8, 4, 64, fake, fake, 0, 0, (float*)fake, (float*)fake,
                     (int32_t*)fake, (int32_t*)fake, 0};
  certkv_rows r = {fake, 1 << 30, 1 << 30, 1 << 20, 128};
  int rc = -1;
  if (!strcmp(argv[1], "load")) {
    certkv_packed pk = {};
    pk.k = pk.v = (decltype(pk.k))fake;
    pk.offsets = (decltype(pk.offsets))fake;
    pk.real_counts = (decltype(pk.real_counts))fake;
    pk.capacity_slots = 9;
    rc = certkv_store_load(&pk, 1, 0, &st, fake, 1 << 30, 0);
  } else if (!strcmp(argv[1], "append")) {
    rc = certkv_store_append(1, 1, units, tokens, &r, &r, 0, 0, 0, &st, 0);
  } else {
    certkv_shape sh = {1, 1, units, units, 2, 128, 1};
    rc = certkv_tree_attn(&sh, tokens, &r, 0, 0, 0, &st, 0.f, &r, 0, fake, (size_t)1 << 40, 0);
  }
  printf("%d %d %d\n", rc, launches, (int)last);
}
"""


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    d = tmp_path_factory.mktemp("launch")
    csrc = os.path.join(os.path.dirname(B.__file__), "csrc")
    src, runtime, exe = d / "calls.cu", d / "runtime.cpp", d / "calls"
    src.write_text(CALLS_IN_C)
    runtime.write_text(RUNTIME)
    subprocess.run([B.NVCC, *B.ARCH, "-std=c++17", "--expt-relaxed-constexpr", "-cudart", "none",
                    "-I", csrc, "-I", B.INCLUDE, str(src), str(runtime), os.path.join(csrc, "store.cu"),
                    os.path.join(csrc, "tree.cu"), "-o", str(exe)], check=True)

    def run(what, fails, units=4, tokens=3):
        r = subprocess.run([str(exe), what, str(fails), str(units), str(tokens)],
                           capture_output=True, text=True, check=True)
        return tuple(int(x) for x in r.stdout.split())
    return run


# kernels of a call: load plan, load; rows, counts; (plan of many units,) split, merge
CALLS = [("load", {}, 2), ("append", {}, 2), ("append", dict(tokens=300), 2),
         ("tree", {}, 2), ("tree", dict(tokens=64), 2), ("tree", dict(units=300), 3),
         ("tree", dict(units=300, tokens=64), 3)]


@pytest.mark.parametrize("what,kw,kernels", CALLS)
def test_nothing_is_launched_behind_a_failure(call, what, kw, kernels):
    assert call(what, 0, **kw) == (0, kernels, 0)
    for n in range(1, kernels + 1):
        rc, launches, left = call(what, n, **kw)
        assert (rc, launches, left) == (5, n, 0), (n, rc, launches, left)
