// Which request an extend token belongs to.
#pragma once

#include "common.h"

namespace pa {

// The request of extend token t: how many of ext_offsets[1 .. B) are <= t.
__device__ __forceinline__ int request_of(const int32_t* __restrict__ ext_offsets, int B, int64_t t) {
    constexpr int kDirect = 256;  // up to this many: all offsets in one round trip; beyond, a search
    if (B <= kDirect) {
        int r = 0;
#pragma unroll
        for (int c = 0; c < kDirect; c += 64) {
            const int k = c + static_cast<int>(threadIdx.x & 63);
            r += __popcll(__ballot(k >= 1 && k < B && ext_offsets[k] <= t));
        }
        return r;
    }
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (ext_offsets[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
}

}  // namespace pa
