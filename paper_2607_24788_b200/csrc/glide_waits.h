// What bounded waits decide, apart from the instructions that wait: plain C++, so that the host can try it too.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define GLIDE_WAIT_FN __device__ __forceinline__
#else
#define GLIDE_WAIT_FN inline
#endif

namespace glide {

// A wait that may last as long as other threads' work, which has no limit that is known beforehand: `landed` tries for a bounded time,
// `gave_up` says whether another thread has given up, `moves` counts pieces of the work that is waited for.  Gives up after `limit` tries in
// a row in which the count stood still.
template <typename Landed, typename GaveUp, typename Moves>
GLIDE_WAIT_FN bool wait_while_moving(Landed &&landed, GaveUp &&gave_up, Moves &&moves, int limit) {
  if (landed()) return true;
  uint32_t count = moves();
  for (int still = 1; still < limit && !gave_up(); ++still) {
    if (landed()) return true;
    const uint32_t now = moves();
    if (now != count) count = now, still = 0;
  }
  return false;
}

}  // namespace glide
