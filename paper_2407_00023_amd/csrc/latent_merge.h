// The second launch of a bf16 latent attention: the parts of tiles that were cut, joined (latent_work.h).
#pragma once

#include <hip/hip_bf16.h>

#include "latent_work.h"
#include "wave_ops.h"

namespace pa {

// The parts of tiles joined.  Every workgroup looks at all records, 512 at most, and counts what there is to join, in pieces of kJoinRows rows; the
// pieces are dealt out in turn.  8 us with a few parts, of which the launch and three dependent reads are most; 35 us for 20 MB of them.  (A workgroup for every piece that there could be took 40 us to find that most of it had nothing to do.)
constexpr int kMergeGroups = 2048;  // eight on a compute unit, at most
constexpr int kMaxParts = 512;
template <int R>
__global__ __launch_bounds__(256) void latent_merge_kernel(LatentParts parts, int M, int n_max, __hip_bfloat16* __restrict__ out) {
    constexpr int kCols = R / 4, kRowsAtOnce = 256 / kCols, kJoinRows = kRowsAtOnce > 4 ? kRowsAtOnce : 4;  // threads of a row
    __shared__ int s_last[kMaxParts], s_sum[4], s_found[2];
    __shared__ float s_w[kMaxParts][kJoinRows];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = parts.hdr[6];
    int pieces[2], before[2];
    int4 rec[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int w = 2 * tid + i;
        rec[i] = w < n_max ? parts.rec[2 * w + 1] : make_int4(0, 0, 0, 0);
        s_last[w] = w < n_max ? parts.rec[2 * w].z & kPartLast : kPartLast;
        pieces[i] = w < n && (rec[i].z & kPartHead) ? (rec[i].y + kJoinRows - 1) / kJoinRows : 0;
    }
    int in = pieces[0] + pieces[1];
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(in, off);
        if (lane >= off) in += y;
    }
    if (lane == 63) s_sum[wave] = in;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < 4; ++w) {
        if (w < wave) in += s_sum[w];
        all += s_sum[w];
    }
    before[0] = in - pieces[0] - pieces[1];
    before[1] = before[0] + pieces[0];
    for (int piece = blockIdx.x; piece < all; piece += gridDim.x) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (before[i] <= piece && piece < before[i] + pieces[i]) {
                s_found[0] = 2 * tid + i;
                s_found[1] = piece - before[i];
            }
        __syncthreads();
        const int w = __builtin_amdgcn_readfirstlane(s_found[0]), row0 = __builtin_amdgcn_readfirstlane(s_found[1]) * kJoinRows;
        const int4 r = parts.rec[2 * w + 1];
        const int here = min(kJoinRows, r.y - row0);
        // parts: slot 2 w + 1, then 2 (w + 1), 2 (w + 2), ... up to the one that ends the tile
        int count = 1;
        for (bool more = true; more;) {
            const int i = w + count + lane;
            const unsigned long long ends = __ballot(i < n ? s_last[i] : 1);
            count += ends ? __builtin_ctzll(ends) + 1 : 64;
            more = ends == 0;
        }
        count = min(count, n_max - w);
        auto slot = [&](int p) { return p == 0 ? 2 * w + 1 : 2 * (w + p); };
        // weights of the parts: 2^(their maximum - the largest) over the sum
        for (int row = wave; row < here; row += 4) {
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
        __syncthreads();
        const int c = tid % kCols;
        for (int row = tid / kCols; row < here; row += kRowsAtOnce) {
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            // (eight at once: 82 registers, few waves, 47 us for the 20 MB; two: 9 us for a few parts)
#pragma unroll 4
            for (int p = 0; p < count; ++p) {
                const float a = s_w[p][row];
                const float4 v = *reinterpret_cast<const float4*>(parts.o + (static_cast<size_t>(slot(p)) * M + row0 + row) * R + 4 * c);
                acc.x += a * v.x;  // (a part with nothing for a row holds zeros, or NaN where a value seen there is not finite)
                acc.y += a * v.y;
                acc.z += a * v.z;
                acc.w += a * v.w;
            }
            *reinterpret_cast<uint2*>(out + (r.x + static_cast<int64_t>(row0 + row) * r.w) * R + 4 * c) = make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
        }
        __syncthreads();
    }
}

// rows: of the output, all heads; requests: times the heads that a tile does not hold together
inline void launch_latent_merge(const LatentParts& parts, int n_wg, int M, int width, int64_t rows, int64_t requests, void* out, hipStream_t stream) {
    const int64_t pieces = rows / 4 + requests;  // there are no more
    const dim3 grid(static_cast<unsigned>(pieces < kMergeGroups ? pieces : kMergeGroups));
    __hip_bfloat16* const o = static_cast<__hip_bfloat16*>(out);
    if (width == 512) hipLaunchKernelGGL(latent_merge_kernel<512>, grid, dim3(256), 0, stream, parts, M, n_wg, o);
    else if (width == 256) hipLaunchKernelGGL(latent_merge_kernel<256>, grid, dim3(256), 0, stream, parts, M, n_wg, o);
    else if (width == 128) hipLaunchKernelGGL(latent_merge_kernel<128>, grid, dim3(256), 0, stream, parts, M, n_wg, o);
    else hipLaunchKernelGGL(latent_merge_kernel<64>, grid, dim3(256), 0, stream, parts, M, n_wg, o);
}

}  // namespace pa
