// Latent attention: what its files share.  A cached token is one row (c, r) of R latent and kRope rotary values, the same for all
// query heads.
//
// Pool: rows by slot (a row belongs to no KV head, so pages do not show in it).  PA_F32, PA_BF16: R + kRope elements a row.
// PA_BF16_KV8: a row is R codes (fp8_rows.h) and kRope bfloat16 values, 2 * kRope + R bytes, and behind the last row lies one
// int8 exponent per slot.  All rows start at multiples of 128 bytes.
#pragma once

#include "common.h"

namespace pa {

constexpr int kRope = 64;  // rotary values of a row
constexpr int kMostGroups = 1 << 20;  // workgroups of a launch with one for each item, at most (a launch has fewer than 2^32 threads)

inline bool latent_shape_ok(int H, int R, int P) { return H > 0 && (R == 256 || R == 512) && P == kRope; }

// bytes of a row of the caller's tensors, and of the pool
inline int latent_row_bytes(int R, int dtype) { return (R + kRope) * static_cast<int>(elt_size(dtype)); }
__host__ __device__ inline int latent_pool_row_bytes(int R, int dtype) {
    return dtype == PA_F32 ? 4 * (R + kRope) : dtype == PA_BF16 ? 2 * (R + kRope) : R + 2 * kRope;
}

// A batch as the attention calls are given it (device pointers; T: rows of c_ext).
struct LatentBatch {
    const void *c_ext, *pool;
    const int32_t *slot_idx, *slot_offsets, *prefix_len, *ext_len, *ext_offsets;
    int B;
    int64_t T, num_slots;
};

}  // namespace pa
