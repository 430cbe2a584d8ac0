"""The last waits of a block's roles, for the copies that each has on its way itself (csrc/follow.cuh),
on the CPU: with a flag of its own one whose copies never land does not shorten another's, as it would
with a flag that they share."""
import os
import re
import subprocess

import pytest

from paper_2608_21541_gb300 import build as B

CSRC = os.path.join(os.path.dirname(B.__file__), "csrc")
PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include "follow.cuh"

// one wait after the other, each until a role's copies have landed; past the limit they never do
int main(int argc, char** argv) {
  const uint32_t limit = atoi(argv[1]);
  bool shared = false;
  for (int r = 2; r < argc; ++r) {
    const uint32_t lands = atoi(argv[r]);
    for (int i = 0; i < 2; ++i) {
      bool own = false;
      bool& flag = i ? shared : own;
      uint32_t looks = 0;
      const bool there = certkv::look(limit, [&] { return looks++ >= lands; }, [&] { return flag; }, [&] { flag = true; });
      printf("%d %u ", there, looks);
    }
    printf("\n");
  }
}
"""


@pytest.fixture(scope="module")
def waits(tmp_path_factory):
    d = tmp_path_factory.mktemp("waits")
    src, exe = d / "waits.cu", d / "waits"
    src.write_text(PROGRAM)
    subprocess.run([B.NVCC, "-std=c++17", "--extended-lambda", "-I", CSRC, str(src), "-o", str(exe)],
                   check=True)

    def run(limit, *lands):
        out = subprocess.run([str(exe), str(limit), *map(str, lands)], capture_output=True, text=True,
                             check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return run


@pytest.mark.parametrize("lands", [0, 1, 255, 256, 257, 3000, 4999])
def test_a_wait_that_runs_out_does_not_shorten_another(waits, lands):
    first, second = waits(5000, 10 ** 6, lands)
    assert first == (0, 5000, 0, 5000)
    assert second[:2] == (1, lands + 1)
    assert second[2:] == ((1, lands + 1) if lands <= 255 else (0, 256))  # gone with copies on their way


def test_the_gradients_last_waits_have_flags_of_their_own():
    """Every wait for what is on its way at a role's end is of this kind, and no two roles of a block
    have the same flag."""
    for name, count in (("grad_q.cu", 2), ("grad_kv.cu", 2), ("grad_tc.cuh", 3)):
        text = open(os.path.join(CSRC, name)).read()
        assert len(re.findall(r"(?<!void )\bfinish\([^;]*\bown\b[^;]*\);", text)) == count, name
        assert not re.search(r"\bwait(_all)?\([^;]*\blast\b[^;]*\);", text), name
        if name != "grad_tc.cuh":
            flags = re.findall(r"GRAD_AT\(own\)( \+ \d+u)?", text)
            assert len(flags) == len(set(flags)) == 5, name
