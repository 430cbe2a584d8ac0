// follow.cuh — following a warp that does not wait for its followers.
//
// A phase parity tells only neighbouring phases of a barrier apart, so it can be waited on only
// by those that the barrier's owner waits for in turn: a follower eight tiles behind, on a ring
// of eight, would take a later phase for one that has not completed, and near the end of a walk
// wait for one that never comes.  A count that only grows has no such phase: however far behind,
// the follower finds its tile reached.
#pragma once

#include <stdint.h>

namespace certkv {

// Waits until `count()` says that tile t has been passed: true; false when `stop()` says so or
// after `limit` looks, with nothing else done about it (what only helps others may not stop
// them).  `idle()` between looks.
template <class Count, class Stop, class Idle>
__host__ __device__ inline bool follow(uint32_t t, uint32_t limit, Count count, Stop stop, Idle idle) {
#pragma unroll 1
  for (uint32_t i = 0; i < limit; ++i) {
    if (count() > t) return true;
    if (stop()) return false;
    idle();
  }
  return false;
}

}  // namespace certkv
