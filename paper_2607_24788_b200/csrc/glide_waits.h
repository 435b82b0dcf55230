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

// What a loader has asked for: copies into two buffers q (a barrier each, every copy a phase), tiles into a ring of `stages` buffers (a
// barrier each), of which some came by the barrier of tails instead and let their ring barrier go only when they had been trimmed.
struct AskedCopies {
  uint32_t q[2] = {0, 0};
  int tiles = 0;
  uint32_t tails = 0;
  int untrimmed = -1;   // the tile, if any, whose tail has been asked for and not been trimmed: nobody lets its ring barrier go
};
enum : int { kCopyQ, kCopyTile, kCopyTail };
// wait(what, which barrier, parity) for every phase that a copy may still be on its way to: none but the last one of each barrier can be.
template <typename Wait>
GLIDE_WAIT_FN void wait_for_copies(const AskedCopies &asked, int stages, Wait &&wait) {
  for (int x = 0; x < 2; ++x)
    if (asked.q[x]) wait(kCopyQ, x, (asked.q[x] - 1) & 1u);
  for (int tile = asked.tiles > stages ? asked.tiles - stages : 0; tile < asked.tiles; ++tile)
    if (tile != asked.untrimmed) wait(kCopyTile, tile % stages, uint32_t(tile / stages) & 1u);
  if (asked.tails) wait(kCopyTail, 0, (asked.tails - 1) & 1u);
}

}  // namespace glide
