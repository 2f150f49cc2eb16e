// How long a bounded wait on the device lasts.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define POS_HD __host__ __device__ __forceinline__
#else
#define POS_HD inline
#endif

namespace pos {

// Two seconds of a wait's own time, told by the readings of a clock between its tries,
// which sleep for a millisecond at most.  A longer gap between two readings is time in
// which the GPU ran something else (it is shared in time with another process, or a
// debugger holds it) and nothing could arrive: it counts as four milliseconds.
constexpr uint64_t kWaitNs = 2000000000ull, kWaitGapNs = 4000000ull;

struct WaitLimit {
    uint64_t last, spent;
    explicit POS_HD WaitLimit(uint64_t now) : last(now), spent(0) {}
    // Called after a try that failed: whether the wait is over.
    POS_HD bool reached(uint64_t now) {
        const uint64_t gap = now - last;
        last = now;
        spent += gap < kWaitGapNs ? gap : kWaitGapNs;
        return spent > kWaitNs;
    }
};

}  // namespace pos
