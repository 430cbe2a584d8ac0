// follow.cuh — following a warp that does not wait for its followers, and bounded looking.
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

// Looks until `done()`: true; false when `stop()` says so, which is asked every 256 looks, or after
// `limit` of them, and then `give_up()`.
template <class Done, class Stop, class GiveUp>
__host__ __device__ inline bool look(uint32_t limit, Done done, Stop stop, GiveUp give_up) {
#pragma unroll 1
  for (uint32_t i = 0; i < limit; ++i) {
    if (done()) return true;
    if ((i & 255u) == 255u && stop()) return false;
  }
  give_up();
  return false;
}

}  // namespace certkv
