"""As test_failed_launch.py, for pages, slot maps and gradients: nothing is launched behind a launch
that failed, so no list is read that was not written and no gradient of records that are not there."""
import os
import subprocess

import pytest

from paper_2608_21541_gb300 import build as B
from test_failed_launch import RUNTIME

MORE = r"""
extern "C" {
cudaError_t CUDARTAPI cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t CUDARTAPI cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t CUDARTAPI cudaMemsetAsync(void*, int, size_t, cudaStream_t) { return cudaSuccess; }
}
"""

CALLS_IN_C = r"""
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include "grad.cuh"
#include "internal.cuh"

extern int launches, fails;
extern cudaError_t last;
namespace certkv {
void trace_begin(const char*, cudaStream_t) {}
void trace_end(cudaStream_t) {}
int grad_ctas() { return 152; }
__global__ void some_kernel(int) {}
bool launch_grad_q(const GradArgs&, int, cudaStream_t st) { return launch_kernel(true, some_kernel, 1, 32, 0, st, 1); }
bool launch_grad_kv(const GradArgs&, int, cudaStream_t st) { return launch_kernel(true, some_kernel, 1, 32, 0, st, 1); }
}  // namespace certkv

int main(int argc, char** argv) {
  fails = atoi(argv[2]);
  const int units = atoi(argv[3]), pages = atoi(argv[4]), tokens = atoi(argv[5]), group = atoi(argv[6]);
  const bool slots = argv[7][0] == '1', drafts = argv[8][0] == '1';
  void* fake = (void*)(1 << 20);
  certkv_store st = {units, CERTKV_STORE_FP8, pages, 64, fake, fake, 0, 0, (float*)fake, (float*)fake,
                     (int32_t*)fake, (int32_t*)fake, 0};
  certkv_pages pg = {(int32_t*)fake, (int32_t*)fake, (int32_t*)fake};
  certkv_rows r = {fake, 1 << 30, 1 << 30, 1 << 20, 128};
  int rc = -1;
  if (!strcmp(argv[1], "list")) {
    rc = certkv_pages_list(&st, &pg, fake, 1 << 30, 0);
  } else if (!strcmp(argv[1], "reserve")) {
    rc = certkv_pages_reserve(1, 0, 0, &st, &pg, fake, 1 << 30, 0);
  } else if (!strcmp(argv[1], "map")) {
    rc = certkv_slot_map(1, tokens, 0, 0, 0, 0, &st, (int32_t*)fake, (int32_t*)fake, 0);
  } else {
    certkv_shape sh = {1, 1, units * group, units, 2, 128, 1};
    rc = certkv_tree_attn_grad(&sh, tokens, &r, drafts ? &r : 0, drafts ? &r : 0, 0, &st, 0.f, &r, (float*)fake, &r, 0,
                               &r, drafts ? &r : 0, drafts ? &r : 0, slots ? fake : 0, slots ? fake : 0, fake,
                               (size_t)1 << 40, 0);
  }
  printf("%d %d %d\n", rc, launches, (int)last);
}
"""


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    d = tmp_path_factory.mktemp("step")
    csrc = os.path.join(os.path.dirname(B.__file__), "csrc")
    src, runtime, exe = d / "calls.cu", d / "runtime.cpp", d / "calls"
    src.write_text(CALLS_IN_C)
    runtime.write_text(RUNTIME + MORE)
    subprocess.run([B.NVCC, *B.ARCH, "-std=c++17", "--expt-relaxed-constexpr", "-cudart", "none",
                    "-I", csrc, "-I", B.INCLUDE, str(src), str(runtime), os.path.join(csrc, "pages.cu"),
                    os.path.join(csrc, "grad.cu"), "-o", str(exe)], check=True)

    def run(what, fails, units=4, pages=4, tokens=3, group=2, slots=False, drafts=True):
        args = (what, fails, units, pages, tokens, group, int(slots), int(drafts))
        r = subprocess.run([str(exe), *map(str, args)], capture_output=True, text=True, check=True)
        return tuple(int(x) for x in r.stdout.split())
    return run


# kernels of a call: mark, sums, list; all by one block, or sums, back, out (and settle); one map;
# rows, (slots,) queries where they are not made with them, (fold of long segments,) drafts (and
# their chunks joined), or without drafts the merge
CALLS = [("list", {}, 3), ("reserve", {}, 1), ("reserve", dict(units=2000), 3),
         ("reserve", dict(pages=300), 4), ("map", {}, 1), ("map", dict(tokens=5000), 1),
         ("grad", {}, 3), ("grad", dict(drafts=False), 3), ("grad", dict(slots=True), 3),
         ("grad", dict(slots=True, tokens=64), 4), ("grad", dict(tokens=64, group=4, slots=True), 5),
         ("grad", dict(pages=40), 4), ("grad", dict(pages=40, drafts=False, slots=True, tokens=50), 5)]


@pytest.mark.parametrize("what,kw,kernels", CALLS)
def test_nothing_is_launched_behind_a_failure(call, what, kw, kernels):
    assert call(what, 0, **kw) == (0, kernels, 0)
    for n in range(1, kernels + 1):
        rc, launches, left = call(what, n, **kw)
        assert (rc, launches, left) == (5, n, 0), (n, rc, launches, left)
