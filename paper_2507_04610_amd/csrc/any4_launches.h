// One long grid as several launches: HIP takes fewer than 2^32 threads along an axis of the grid, 2^24 blocks of 256 threads.
#pragma once
#include <stdint.h>

namespace any4 {

constexpr int64_t kLaunchThreads = ((int64_t)1 << 32) - 1;

// launch(first, count) for blocks first .. first + count - 1 of `blocks` blocks of `threads` threads, one piece behind the other, until one is
// refused (anything but `ok`); no blocks, no launch
template <class E, class F> E launch_blocks(int64_t blocks, int threads, E ok, F launch) {
    const int64_t most = kLaunchThreads / threads;
    for (int64_t first = 0; first < blocks; first += most)
        if (const E e = launch(first, blocks - first < most ? blocks - first : most); e != ok) return e;
    return ok;
}

}  // namespace any4
