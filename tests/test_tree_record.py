"""What a split kernel of tree attention records for a row (csrc/tree.cuh), on the CPU: NaN when
any wait that the row's sum depends on ran out, the writer's own or another's."""
import os
import subprocess

from paper_2608_21541_gb300 import build as B

PROGRAM = r"""
#include <stdio.h>
#include "tree.cuh"

int main() {
  for (int i = 0; i < 4; ++i) {
    const float2 r = certkv::tree_record(i & 1, i & 2, 3.f, 0.5f);
    printf("%g %g\n", r.x, r.y);
  }
}
"""


def test_a_record_is_nan_when_any_part_of_it_is_missing(tmp_path):
    src, exe = tmp_path / "record.cu", tmp_path / "record"
    src.write_text(PROGRAM)
    csrc = os.path.join(os.path.dirname(B.__file__), "csrc")
    subprocess.run([B.NVCC, *B.ARCH, "-std=c++17", "--expt-relaxed-constexpr", "-I", csrc, str(src),
                    "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split("\n")
    assert got[1] == "3 0.5"  # ok, nobody gave up
    for line in (got[0], got[2], got[3]):
        assert line.split()[1].lstrip("-") == "nan"
