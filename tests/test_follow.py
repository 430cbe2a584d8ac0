"""Following a warp that does not wait for its followers (csrc/follow.cuh), on the CPU: a walk of
n tiles whose leader is any number of tiles ahead, and stays so until the end.  Beside it what a
phase parity on a ring of eight barriers would have answered."""
import os
import subprocess

import pytest

from paper_2608_21541_gb300 import build as B

PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include "follow.cuh"

int main(int argc, char** argv) {
  const uint32_t n = atoi(argv[1]), lead = atoi(argv[2]), halt = atoi(argv[3]);
  // the leader has passed `lead` tiles before the follower looks for the first time, and one
  // more for every tile the follower takes, or whenever it finds the follower waiting; at `halt`
  // it stays
  uint32_t passed = lead < n ? lead : n, looks = 0, taken = 0;
  auto step = [&] { if (passed < n && passed < halt) ++passed; ++looks; };
  bool ok = true;
  for (uint32_t t = 0; t < n && ok; ++t, taken += ok) {
    ok = certkv::follow(t, 1000, [&] { return passed; }, [&] { return passed == halt && looks > 300; }, step);
    if (ok) step();
  }
  // the same with the parity of tile t's phase t / 8 of barrier t % 8: it reads as complete when
  // the last phase that completed has that parity
  uint32_t p = lead < n ? lead : n, by_parity = 0;
  for (uint32_t t = 0; t < n; ++t, ++by_parity) {
    bool there = false;
    for (int i = 0; i < 1000 && !there; ++i) {
      const uint32_t phases = (p + 7 - t % 8) / 8;  // completed, of barrier t % 8
      there = phases > 0 && ((phases - 1) & 1) == ((t / 8) & 1);
      if (!there && p < n) ++p;
    }
    if (!there) break;
    if (p < n) ++p;
  }
  printf("%u %u %u\n", taken, looks, by_parity);
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    d = tmp_path_factory.mktemp("follow")
    src, exe = d / "follow.cu", d / "follow"
    src.write_text(PROGRAM)
    subprocess.run([B.NVCC, "-std=c++17", "--extended-lambda", "-I",
                    os.path.join(os.path.dirname(B.__file__), "csrc"), str(src), "-o", str(exe)],
                   check=True)

    def run(n, lead, halt=1 << 30):
        r = subprocess.run([str(exe), str(n), str(lead), str(halt)], capture_output=True,
                           text=True, check=True)
        return [int(x) for x in r.stdout.split()]
    return run


@pytest.mark.parametrize("n", [1, 7, 8, 9, 40, 203])
@pytest.mark.parametrize("lead", [0, 1, 7, 8, 9, 15, 16, 17, 33, 500])
def test_every_tile_is_reached_however_far_behind(walk, n, lead):
    taken, looks, _ = walk(n, lead)
    assert taken == n and looks <= 2 * n


def test_a_parity_would_leave_a_late_follower_waiting(walk):
    assert walk(40, 0)[2] == 40 and walk(40, 7)[2] == 40
    assert walk(40, 9)[2] < 40 and walk(40, 15)[2] < 40


def test_a_leader_that_stays_is_given_up(walk):
    taken, looks, _ = walk(40, 0, halt=13)
    assert taken == 13 and 300 < looks < 350  # told to stop, before the limit
