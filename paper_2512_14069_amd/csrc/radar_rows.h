// Rows of a batch's new tokens, [B, T_max] or one sequence's behind the other's (gfx950).
#pragma once

#include "radar_device.h"

namespace radar {

// The last of n (1 to 2^30) sequences whose value(b) is at most x, -1 if there is none; values that never fall.  Sixty-four are looked at at a time,
// so that up to 64 sequences take one round trip, 4096 two.  The same x in every lane; all lanes call.  Any values keep the result within [-1, n).
template <typename Value>
__device__ __forceinline__ int last_at_most(int n, int64_t x, Value value) {
    int first = 0, left = n;
    for (;;) {
        const int step = (left + kWave - 1) / kWave, at = lane_id() * step;
        const uint64_t yes = __ballot(at < left && value(first + min(at, left - 1)) <= x);
        if (yes == 0) return first == 0 ? -1 : first - 1;
        const int hit = 63 - __clzll((long long)yes);
        first += hit * step;
        left = min(step, left - hit * step);
        if (step == 1) return first;
    }
}

}  // namespace radar
