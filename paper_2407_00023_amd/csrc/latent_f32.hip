// Latent attention, fp32 tensors: one workgroup per new token and four of its heads.
//
// Query head h of extend row i of request r sees the P_r cached rows named by slot_idx and the extend rows 0..i; a row (c, r) is its
// own key, and c its value:  out = sum_j softmax_j(scale <q, (c_j, r_j)>) c_j.
//
// A wave takes every fourth key: its lanes hold R / 64 latent and one rotary value of the row each, the heads' dot products are sums over
// the wave, and the same registers are the value that the running sums take up (one pass: maximum and sum move along).  The four
// waves are joined through LDS at the end.
//
// For checks and small models, not for speed: 4 requests of 16 to 32 tokens and 96 cached rows, 4 heads, R = 256, take 24 us, the length of one
// workgroup's walk over its keys.
#include "latent.h"
#include "requests.h"

namespace pa {

constexpr int kF32Heads = 4;   // heads of a workgroup
constexpr int kF32Unroll = 4;  // keys that a wave asks for together

template <int R>
__global__ __launch_bounds__(256) void latent_f32_kernel(const float* __restrict__ q_ext, LatentBatch b, int H, float scale, float* __restrict__ out) {
    constexpr int L = R + kRope, EPL = R / 64;  // latent elements per lane
    __shared__ float s_acc[4][kF32Heads][R];
    __shared__ float s_m[4][kF32Heads], s_l[4][kF32Heads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int h0 = blockIdx.y * kF32Heads, n_heads = min(kF32Heads, H - h0);
    for (int64_t t = blockIdx.x; t < b.T; t += gridDim.x) {
        const int r = request_of(b.ext_offsets, b.B, t);
        const int64_t e0 = b.ext_offsets[r];
        const int P = max(b.prefix_len[r], 0), E = b.ext_len[r], i = static_cast<int>(t - e0);
        if (i < 0 || i >= E) continue;  // inconsistent offsets: produce nothing rather than read out of range
        const int nvis = P + i + 1;
        const int32_t* __restrict__ slots = b.slot_idx + b.slot_offsets[r];
        const float *const c_ext = static_cast<const float*>(b.c_ext), *const pool = static_cast<const float*>(b.pool);

        float q[kF32Heads][EPL + 1], acc[kF32Heads][EPL], m[kF32Heads], l[kF32Heads];
#pragma unroll
        for (int x = 0; x < kF32Heads; ++x) {
            const float* const row = q_ext + (t * H + h0 + min(x, n_heads - 1)) * L;
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
                q[x][e] = row[lane * EPL + e] * scale;
                acc[x][e] = 0.f;
            }
            q[x][EPL] = row[R + lane] * scale;
            m[x] = -INFINITY;
            l[x] = 0.f;
        }
        auto load_row = [&](int j, float (&k)[EPL + 1]) {
            const float* const row = j < P ? pool + min(static_cast<int64_t>(max(slots[j], 0)), b.num_slots - 1) * L  // never outside the pool
                                           : c_ext + (e0 + (j - P)) * L;
#pragma unroll
            for (int e = 0; e < EPL; ++e) k[e] = row[lane * EPL + e];
            k[EPL] = row[R + lane];
        };
        for (int j0 = wave; j0 < nvis; j0 += 4 * kF32Unroll) {
            float k[kF32Unroll][EPL + 1];
#pragma unroll
            for (int u = 0; u < kF32Unroll; ++u) load_row(min(j0 + 4 * u, nvis - 1), k[u]);
#pragma unroll
            for (int x = 0; x < kF32Heads; ++x) {
                float s[kF32Unroll];
#pragma unroll
                for (int u = 0; u < kF32Unroll; ++u) {
                    float d = 0.f;
#pragma unroll
                    for (int e = 0; e <= EPL; ++e) d += q[x][e] * k[u][e];
#pragma unroll
                    for (int off = 1; off < 64; off <<= 1) d += __shfl_xor(d, off);
                    s[u] = j0 + 4 * u < nvis ? d : -INFINITY;
                }
                float mx = m[x];
#pragma unroll
                for (int u = 0; u < kF32Unroll; ++u) mx = fmaxf(mx, s[u]);
                const float ref = mx == -INFINITY ? 0.f : mx;
                const float alpha = expf(m[x] - ref);
                m[x] = mx;
                l[x] *= alpha;
#pragma unroll
                for (int e = 0; e < EPL; ++e) acc[x][e] *= alpha;
#pragma unroll
                for (int u = 0; u < kF32Unroll; ++u) {
                    if (j0 + 4 * u >= nvis) break;  // (a key past the end must not meet an infinity of the row that stands for it)
                    const float p = expf(s[u] - ref);
                    l[x] += p;
#pragma unroll
                    for (int e = 0; e < EPL; ++e) acc[x][e] += p * k[u][e];
                }
            }
        }
#pragma unroll
        for (int x = 0; x < kF32Heads; ++x) {
#pragma unroll
            for (int e = 0; e < EPL; ++e) s_acc[wave][x][lane * EPL + e] = acc[x][e];
            if (lane == 0) {
                s_m[wave][x] = m[x];
                s_l[wave][x] = l[x];
            }
        }
        __syncthreads();
        for (int y = tid; y < n_heads * R; y += 256) {
            const int x = y / R, d = y % R;
            float mx = s_m[0][x];  // (wave 0 has seen key 0)
#pragma unroll
            for (int w = 1; w < 4; ++w) mx = fmaxf(mx, s_m[w][x]);
            float num = 0.f, den = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if (w >= nvis) break;  // (a wave without a key)
                const float a = expf(s_m[w][x] - mx);
                num += a * s_acc[w][x][d];
                den += a * s_l[w][x];
            }
            out[(t * H + h0 + x) * R + d] = num / den;
        }
        __syncthreads();
    }
}

int latent_attention_f32(const void* q, const LatentBatch& b, int H, int R, float scale, void* out, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(b.T < kMostGroups ? b.T : kMostGroups), static_cast<unsigned>((H + kF32Heads - 1) / kF32Heads));
    PA_REQUIRE(grid.y <= 65535, "pa_latent_attention: too many heads (%d)", H);
    ProfScope scope(kProfLatentF32, stream);
    const float* const qf = static_cast<const float*>(q);
    float* const of = static_cast<float*>(out);
    if (R == 512) hipLaunchKernelGGL(latent_f32_kernel<512>, grid, dim3(256), 0, stream, qf, b, H, scale, of);
    else hipLaunchKernelGGL(latent_f32_kernel<256>, grid, dim3(256), 0, stream, qf, b, H, scale, of);
    PA_HIP(hipGetLastError());
    return PA_OK;
}

// The expanded form is the absorbed one between two products: of token and head, W_k[h]^T x before it (its rotary part as it is) and W_v[h] x behind it.
// W [H, N, R].  A workgroup per token and head; the columns, or for W_v the sums, lie across the lanes, so that W is read in lines.
template <bool kKeys>
__global__ __launch_bounds__(256) void head_product_kernel(LatentBatch b, const float* __restrict__ x, const float* __restrict__ w, float* __restrict__ y, int H, int N,
                                                           int R) {
    __shared__ float s_x[512];
    for (int64_t th = blockIdx.x; th < b.T * H; th += gridDim.x) {  // token and head
        const int64_t t = th / H;
        const int h = static_cast<int>(th - t * H);
        const int r = request_of(b.ext_offsets, b.B, t);
        const int64_t i = t - b.ext_offsets[r];
        if (i < 0 || i >= b.ext_len[r]) continue;  // (a row of no request)
        const int in = kKeys ? N : R, in_stride = kKeys ? N + kRope : R, out_stride = kKeys ? R + kRope : N;
        const float* const xr = x + th * in_stride;
        float* const yr = y + th * out_stride;
        const float* const wh = w + static_cast<int64_t>(h) * N * R;
        for (int k = threadIdx.x; k < in; k += 256) s_x[k] = xr[k];
        __syncthreads();
        if (kKeys) {
            for (int o = threadIdx.x; o < R; o += 256) {
                float d = 0.f;
                for (int k = 0; k < N; ++k) d += wh[static_cast<int64_t>(k) * R + o] * s_x[k];
                yr[o] = d;
            }
            for (int o = threadIdx.x; o < kRope; o += 256) yr[R + o] = xr[N + o];
        } else {
            const int lane = threadIdx.x & 63;
            for (int o = threadIdx.x >> 6; o < N; o += 4) {
                float d = 0.f;
                for (int k = lane; k < R; k += 64) d += wh[static_cast<int64_t>(o) * R + k] * s_x[k];
#pragma unroll
                for (int off = 1; off < 64; off <<= 1) d += __shfl_xor(d, off);
                if (lane == 0) yr[o] = d;
            }
        }
        __syncthreads();
    }
}

int latent_expanded_f32(const void* q, const LatentBatch& b, const void* w_k, const void* w_v, int H, int R, int N, float scale, void* out, void* scratch,
                        hipStream_t stream) {
    float* const q_lat = static_cast<float*>(scratch);
    float* const o_lat = q_lat + b.T * H * (R + kRope);
    const dim3 grid(static_cast<unsigned>(b.T * H < kMostGroups ? b.T * H : kMostGroups));
    {
        ProfScope scope(kProfLatentExpand, stream);
        hipLaunchKernelGGL(head_product_kernel<true>, grid, dim3(256), 0, stream, b, static_cast<const float*>(q), static_cast<const float*>(w_k), q_lat, H, N, R);
    }
    PA_HIP(hipGetLastError());
    if (const int rc = latent_attention_f32(q_lat, b, H, R, scale, o_lat, stream)) return rc;
    {
        ProfScope scope(kProfLatentExpand, stream);
        hipLaunchKernelGGL(head_product_kernel<false>, grid, dim3(256), 0, stream, b, o_lat, static_cast<const float*>(w_v), static_cast<float*>(out), H, N, R);
    }
    PA_HIP(hipGetLastError());
    return PA_OK;
}
size_t latent_expanded_f32_bytes(int64_t T, int H, int R) { return static_cast<size_t>(T) * H * (2 * R + kRope) * 4; }

}  // namespace pa
