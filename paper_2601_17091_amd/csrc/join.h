// Where the wavefronts of a workgroup meet (rms_norm.hip).  A host test compiles it too:
// who includes it brings __device__, threadIdx and __syncthreads, and it takes no more.
#pragma once

#include <cstdint>

namespace rocket {

// The sum of s and the largest top over a workgroup's wavefronts, of which each brings its
// own, to all of them.  `shared` has two halves of 2 WAVES words that take turns, so that
// one barrier a join is enough: who writes a half again has passed the next join's barrier,
// and so have read it all who joined in it.  It is joins that take turns, not rows or
// anything else that a caller counts (a row without data has no barrier): `turn`, 0 at
// first, is this function's alone.
template <int WAVES, bool TOP>
__device__ inline void join_waves(float &s, uint32_t &top, float *shared, int &turn) {
    float *at = shared + turn * 2 * WAVES;
    turn ^= 1;
    const int wave = threadIdx.x / 64;
    if (threadIdx.x % 64 == 0) {
        at[wave] = s;
        if (TOP) at[WAVES + wave] = __builtin_bit_cast(float, top);
    }
    __syncthreads();
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < WAVES; k++) s += at[k];
    if (TOP) {
        top = 0;
#pragma unroll
        for (int k = 0; k < WAVES; k++) {
            const uint32_t t = __builtin_bit_cast(uint32_t, at[WAVES + k]);
            top = t > top ? t : top;
        }
    }
}

}  // namespace rocket
