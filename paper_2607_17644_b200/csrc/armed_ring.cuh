// The barriers of a ring that one lane arms in turn, use n at barrier n % kSize: which phases are still open when the lane has to stop, wherever
// in its loop it does.  Counted where a barrier is armed, so that a use whose turn of the loop was not finished belongs to it.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define LAGA_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define LAGA_HOST_DEVICE inline
#endif

namespace laga {

template <uint32_t kSize>
struct ArmedRing {
    uint32_t n = 0;                                  // uses armed
    LAGA_HOST_DEVICE uint32_t at() const { return n % kSize; }         // the barrier that is armed next
    LAGA_HOST_DEVICE void arm() { ++n; }
    // wait(barrier, parity) for the last phase that each barrier was armed for
    template <class Wait>
    LAGA_HOST_DEVICE void last_phases(Wait wait) const {
        for (uint32_t k = 1; k <= kSize && k <= n; ++k) wait((n - k) % kSize, ((n - k) / kSize) & 1u);
    }
};

}  // namespace laga
