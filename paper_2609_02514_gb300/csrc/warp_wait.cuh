// A wait that a whole warp makes with one answer.
//
// Every try is voted on (`all` is the warp's vote, which every lane has to reach), so
// all lanes make the same number of tries and leave together.  A lane that left on a
// try of its own could be past a vote that the others are still at: such a vote names
// lanes that never come, and nothing bounds that wait.  A lane whose try succeeded
// while another's did not simply tries again: the phase it saw cannot end a second
// time before the warp goes on.
//   ready  one quick try;  slow  a longer one, which gives up at its own limit
#pragma once

#ifdef __CUDACC__
#define ACES_LANE __device__ __forceinline__
#else
#define ACES_LANE inline  // the test runs it with a thread a lane
#endif

namespace aces {

constexpr int WARP_TRIES = 16;

template <class Ready, class Slow, class All>
ACES_LANE bool warp_wait(Ready ready, Slow slow, All all) {
    for (int t = 0; t < WARP_TRIES; ++t)
        if (all(ready())) return true;
    return all(slow());
}

}  // namespace aces
