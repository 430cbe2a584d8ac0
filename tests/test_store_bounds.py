"""Segments that do not lie in the packed cache are left out by certkv_store_load, whatever their
offset and length: the check itself on the CPU (csrc/store.cuh), and a load."""
import os
import subprocess

import pytest
import torch

from paper_2608_21541_gb300 import build as B
from paper_2608_21541_gb300 import certkv as ck

PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include "store.cuh"

int main(int argc, char** argv) {
  for (int i = 1; i + 2 < argc; i += 3)
    printf("%d", certkv::lies_in(atoll(argv[i]), atoll(argv[i + 1]), atoll(argv[i + 2])));
}
"""
TOP = 2 ** 63 - 1


def test_lies_in(tmp_path):
    src, exe = tmp_path / "lies.cu", tmp_path / "lies"
    src.write_text(PROGRAM)
    csrc = os.path.join(os.path.dirname(B.__file__), "csrc")
    subprocess.run([B.NVCC, *B.ARCH, "-std=c++17", "--expt-relaxed-constexpr", "-I", csrc, str(src),
                    "-o", str(exe)], check=True)
    cases = [(a, n, c) for a in (-TOP - 1, -1, 0, 1, 90, 100, 101, TOP - 5, TOP)
             for n in (0, 1, 10, 100, 101, 2 ** 31, 2 ** 31 - 1) for c in (1, 100, TOP)]
    got = subprocess.run([str(exe), *(str(x) for c in cases for x in c)], capture_output=True,
                         text=True, check=True).stdout
    assert [ch == "1" for ch in got] == [a >= 0 and a + n <= c for a, n, c in cases]


@pytest.mark.gpu
@pytest.mark.parametrize("offset,real", [(TOP, 5), (TOP - 4, 5), (TOP - 129, 130), (0, 2 ** 31 - 1),
                                         (TOP, 2 ** 31 - 1), (-TOP - 1, 5)])
@pytest.mark.parametrize("tail", [0, 1])
def test_a_segment_outside_is_left_out(offset, real, tail):
    rows = torch.ones((200, 128), dtype=torch.bfloat16, device="cuda")
    packed = ck.Packed(k=rows, v=rows, offsets=torch.tensor([0, offset, 150]).cuda(),
                       real_counts=torch.tensor([100, real, 50 - tail], dtype=torch.int32).cuda(),
                       positions=torch.zeros(200, dtype=torch.int32).cuda(), tail_slot=tail)
    st = ck.Store.empty(3, 3, "fp8", pool_pages=9)
    ck.certkv_store_load(packed, st)
    assert st.read_status() == ck.STATUS_STORE
    # pages are handed out in order: after a segment that wants more than the pool has, none
    last = 50 if real < 2 ** 31 - 1 else 0
    assert st.counts.tolist() == [100 + tail, 0, last]
