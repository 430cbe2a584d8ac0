"""The last waits of a block's roles, for the copies that each has on its way itself (csrc/follow.cuh),
on the CPU: one whose copies never land does not shorten another's.  Beside it what a flag that the
waits share would have done."""
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

// looks until a role's copies have landed; past the limit they never do
int main(int argc, char** argv) {
  const uint32_t limit = atoi(argv[1]);
  int flag = 0;
  for (int r = 2; r < argc; ++r) {
    const uint32_t lands = atoi(argv[r]);
    uint32_t looks = 0;
    const bool own = certkv::outlast(limit, [&] { return looks++ >= lands; });
    bool shared = false, gave_up = false;
    for (uint32_t i = 0; i < limit && !shared && !gave_up; ++i) {
      shared = i >= lands;
      if (!shared && (i & 255u) == 255u && flag) gave_up = true;
    }
    if (!shared && !gave_up) flag = 1;
    printf("%d %u %d\n", own, looks, shared);
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
    assert first == (0, 5000, 0)
    assert second[:2] == (1, lands + 1)
    assert second[2] == (lands <= 255)  # with a flag between them the second would have gone early


def test_the_gradients_last_waits_take_no_flag():
    """Every wait for what is on its way at a role's end is of this kind."""
    for name, count in (("grad_q.cu", 2), ("grad_kv.cu", 2), ("grad_tc.cuh", 3)):
        text = open(os.path.join(CSRC, name)).read()
        assert len(re.findall(r"(?<!void )\bfinish\([^;]*\);", text)) == count, name
        assert not re.search(r"\bwait(_all)?\([^;]*\blast\b[^;]*\);", text), name
