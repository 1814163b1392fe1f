// The second launch of a bf16 latent attention: the parts of tiles that were cut, joined (latent_work.h).
#pragma once

#include <hip/hip_bf16.h>

#include "latent_work.h"
#include "wave_ops.h"

namespace pa {

// The parts of a tile joined: workgroup (w, y) of the launch takes the tile that workgroup w of the attention began and did not finish, if there
// is one, and kJoinRows of its rows.
constexpr int kJoinRows = 4;
template <int R>
__global__ __launch_bounds__(256) void latent_merge_kernel(LatentParts parts, int M, __hip_bfloat16* __restrict__ out) {
    constexpr int kCols = R / 4, kRowsAtOnce = 256 / kCols;  // threads of a row
    __shared__ float s_w[512][kJoinRows];
    const int w = blockIdx.x, n = parts.hdr[6];
    if (w >= n) return;
    const int4 rec = parts.rec[2 * w + 1];
    const int row0 = blockIdx.y * kJoinRows;
    if (!(rec.z & kPartHead) || row0 >= rec.y) return;
    // parts: slot 2 w + 1, then 2 (w + 1), 2 (w + 2), ... up to the one that ends the tile
    const int tid = threadIdx.x, lane = tid & 63;
    int count = 1;
    for (bool more = true; more;) {
        const int i = w + count + lane;
        const int flags = i < n ? parts.rec[2 * i].z : kPartLast;
        const unsigned long long ends = __ballot(flags & kPartLast);
        count += ends ? __builtin_ctzll(ends) + 1 : 64;
        more = ends == 0;
    }
    auto slot = [&](int p) { return p == 0 ? 2 * w + 1 : 2 * (w + p); };
    const int rows = min(kJoinRows, rec.y - row0);
    // weights of the parts: 2^(their maximum - the largest) over the sum
    if (tid < 64 * kJoinRows) {
        const int row = tid >> 6;
        if (row < rows) {
            float mx = -INFINITY, sum = 0.f;
            for (int p = lane; p < count; p += 64) {
                const float2 ml = parts.ml[static_cast<size_t>(slot(p)) * M + row0 + row];
                if (ml.y != 0.f) mx = fmaxf(mx, ml.x);  // (a part whose keys the row does not see says nothing)
            }
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
            const float ref = mx == -INFINITY ? 0.f : mx;
            for (int p = lane; p < count; p += 64) {
                const float2 ml = parts.ml[static_cast<size_t>(slot(p)) * M + row0 + row];
                const float a = ml.y != 0.f ? __builtin_amdgcn_exp2f(ml.x - ref) : 0.f;
                s_w[p][row] = a;
                sum += a * ml.y;
            }
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) sum += __shfl_xor(sum, off);
            for (int p = lane; p < count; p += 64) s_w[p][row] /= sum;
        }
    }
    __syncthreads();
    const int c = tid % kCols;
    for (int row = tid / kCols; row < rows; row += kRowsAtOnce) {
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int p = 0; p < count; ++p) {
            const float a = s_w[p][row];
            const float4 v = *reinterpret_cast<const float4*>(parts.o + (static_cast<size_t>(slot(p)) * M + row0 + row) * R + 4 * c);
            if (a != 0.f) {
                acc.x += a * v.x;
                acc.y += a * v.y;
                acc.z += a * v.z;
                acc.w += a * v.w;
            }
        }
        *reinterpret_cast<uint2*>(out + (rec.x + static_cast<int64_t>(row0 + row) * rec.w) * R + 4 * c) = make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
    }
}

inline void launch_latent_merge(const LatentParts& parts, int n_wg, int M, int width, void* out, hipStream_t stream) {
    const dim3 grid(n_wg, M / kJoinRows);
    __hip_bfloat16* const o = static_cast<__hip_bfloat16*>(out);
    if (width == 512) hipLaunchKernelGGL(latent_merge_kernel<512>, grid, dim3(256), 0, stream, parts, M, o);
    else if (width == 256) hipLaunchKernelGGL(latent_merge_kernel<256>, grid, dim3(256), 0, stream, parts, M, o);
    else if (width == 128) hipLaunchKernelGGL(latent_merge_kernel<128>, grid, dim3(256), 0, stream, parts, M, o);
    else hipLaunchKernelGGL(latent_merge_kernel<64>, grid, dim3(256), 0, stream, parts, M, o);
}

}  // namespace pa
