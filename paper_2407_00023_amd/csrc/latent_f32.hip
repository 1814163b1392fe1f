// Latent attention by rows: fp32 arithmetic throughout, one workgroup per new token and four of its heads.
//
// Query head h of extend row i of request r sees the P_r cached rows named by slot_idx and the extend rows 0..i; a row (c, r) is its
// own key, and c its value:  out = sum_j softmax_j(scale <q, (c_j, r_j)>) c_j.
//
// A wave takes every fourth key: its lanes hold R / 64 latent and one rotary value of the row each, the heads' dot products are sums over
// the wave, and the same registers are the value that the running sums take up (one pass: maximum and sum move along).  The four
// waves are joined through LDS at the end.
#include "fp8_rows.h"
#include "latent.h"
#include "requests.h"

#include <hip/hip_bf16.h>

namespace pa {

constexpr int kF32Heads = 4;   // heads of a workgroup
constexpr int kF32Unroll = 4;  // keys that a wave asks for together

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__hip_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float* p, float x) { *p = x; }
__device__ __forceinline__ void from_f32(__hip_bfloat16* p, float x) { *p = __float2bfloat16(x); }

// QT: type of q and out; CT: of the rows; KV8: the pool in 8 bits
template <typename QT, typename CT, bool KV8, int R>
__global__ __launch_bounds__(256) void latent_rows_attention_kernel(const QT* __restrict__ q_ext, LatentBatch b, int H, float scale,
                                                                    QT* __restrict__ out) {
    constexpr int L = R + kRope, EPL = R / 64;  // latent elements per lane
    __shared__ float s_acc[4][kF32Heads][R];
    __shared__ float s_m[4][kF32Heads], s_l[4][kF32Heads];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t t = blockIdx.x;
    const int h0 = blockIdx.y * kF32Heads, n_heads = min(kF32Heads, H - h0);
    const int r = request_of(b.ext_offsets, b.B, t);
    const int64_t e0 = b.ext_offsets[r];
    const int P = max(b.prefix_len[r], 0), E = b.ext_len[r], i = static_cast<int>(t - e0);
    if (i < 0 || i >= E) return;  // inconsistent offsets: produce nothing rather than read out of range
    const int nvis = P + i + 1;
    const int32_t* __restrict__ slots = b.slot_idx + b.slot_offsets[r];
    const CT* const c_ext = static_cast<const CT*>(b.c_ext);

    float q[kF32Heads][EPL + 1], acc[kF32Heads][EPL], m[kF32Heads], l[kF32Heads];
#pragma unroll
    for (int x = 0; x < kF32Heads; ++x) {
        const QT* const row = q_ext + (t * H + h0 + min(x, n_heads - 1)) * L;
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
            q[x][e] = to_f32(row[lane * EPL + e]) * scale;
            acc[x][e] = 0.f;
        }
        q[x][EPL] = to_f32(row[R + lane]) * scale;
        m[x] = -INFINITY;
        l[x] = 0.f;
    }
    auto load_row = [&](int j, float (&k)[EPL + 1]) {
        const CT* row;
        if (j < P) {
            const int64_t s = min(static_cast<int64_t>(max(slots[j], 0)), b.num_slots - 1);  // never outside the pool
            if constexpr (KV8) {
                const unsigned char* const p = static_cast<const unsigned char*>(b.pool);
                const float two_k = fp8_scale(reinterpret_cast<const signed char*>(p + b.num_slots * (R + 2 * kRope))[s]);
                const unsigned char* const codes = p + s * (R + 2 * kRope);
#pragma unroll
                for (int e = 0; e < EPL; e += 4) {
                    const uint2 v = fp8_decode4(*reinterpret_cast<const unsigned*>(codes + lane * EPL + e), two_k);
                    k[e] = __uint_as_float(v.x << 16);
                    k[e + 1] = __uint_as_float(v.x & 0xFFFF0000u);
                    k[e + 2] = __uint_as_float(v.y << 16);
                    k[e + 3] = __uint_as_float(v.y & 0xFFFF0000u);
                }
                k[EPL] = to_f32(reinterpret_cast<const CT*>(codes + R)[lane]);
                return;
            } else {
                row = static_cast<const CT*>(b.pool) + s * L;
            }
        } else {
            row = c_ext + (e0 + (j - P)) * L;
        }
#pragma unroll
        for (int e = 0; e < EPL; ++e) k[e] = to_f32(row[lane * EPL + e]);
        k[EPL] = to_f32(row[R + lane]);
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
        from_f32(out + (t * H + h0 + x) * R + d, num / den);
    }
}

template <typename QT, typename CT, bool KV8>
static int launch_rows(const void* q, const LatentBatch& b, int H, int R, float scale, void* out, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(b.T), static_cast<unsigned>((H + kF32Heads - 1) / kF32Heads));
    PA_REQUIRE(grid.y <= 65535, "pa_latent_attention: too many heads (%d)", H);
    ProfScope scope(kProfLatentF32, stream);
    if (R == 512)
        hipLaunchKernelGGL((latent_rows_attention_kernel<QT, CT, KV8, 512>), grid, dim3(256), 0, stream, static_cast<const QT*>(q), b, H, scale,
                           static_cast<QT*>(out));
    else
        hipLaunchKernelGGL((latent_rows_attention_kernel<QT, CT, KV8, 256>), grid, dim3(256), 0, stream, static_cast<const QT*>(q), b, H, scale,
                           static_cast<QT*>(out));
    PA_HIP(hipGetLastError());
    return PA_OK;
}

// The products around the rows' attention in its expanded form: row t, head h:  y[t, h, :] = W[h] x[t, h, :] over `in` elements, W [H, out_n, in]
// (kTransposed: W [H, in, out_n]); x and y rows have a stride of their own.  Fp32 sums; a wave per output element.
template <typename XT, typename WT, typename YT, bool kTransposed>
__global__ __launch_bounds__(256) void head_product_kernel(LatentBatch b, const XT* __restrict__ x, int64_t x_stride, const WT* __restrict__ w, YT* __restrict__ y,
                                                           int64_t y_stride, int H, int in, int out_n, const XT* __restrict__ tail, int n_tail) {
    const int64_t th = blockIdx.x;  // token and head
    const int h = static_cast<int>(th % H);
    const int64_t t = th / H;
    const int r = request_of(b.ext_offsets, b.B, t);
    const int64_t i = t - b.ext_offsets[r];
    if (i < 0 || i >= b.ext_len[r]) return;  // (a row of no request)
    const XT* const xr = x + th * x_stride;
    YT* const yr = y + th * y_stride;
    for (int o = threadIdx.x; o < out_n; o += 256) {
        float d = 0.f;
        for (int k = 0; k < in; ++k)
            d += to_f32(w[kTransposed ? (static_cast<int64_t>(h) * in + k) * out_n + o : (static_cast<int64_t>(h) * out_n + o) * in + k]) * to_f32(xr[k]);
        from_f32(yr + o, d);
    }
    for (int o = threadIdx.x; o < n_tail; o += 256) from_f32(yr + out_n + o, to_f32(tail[th * x_stride + o]));
}

int latent_attention_rows(const void* q, const LatentBatch& b, int H, int R, int dtype, float scale, void* out, hipStream_t stream) {
    if (dtype == PA_F32) return launch_rows<float, float, false>(q, b, H, R, scale, out, stream);
    if (dtype == PA_BF16) return launch_rows<__hip_bfloat16, __hip_bfloat16, false>(q, b, H, R, scale, out, stream);
    return launch_rows<__hip_bfloat16, __hip_bfloat16, true>(q, b, H, R, scale, out, stream);
}

template <typename T, bool KV8>
static int expanded_rows(const void* q, const LatentBatch& b, const void* w_k, const void* w_v, int H, int R, int N, float scale, void* out,
                         float* scratch, hipStream_t stream) {
    const int L = R + kRope;
    float* const q_lat = scratch;
    float* const o_lat = scratch + b.T * H * L;
    const dim3 grid(static_cast<unsigned>(b.T * H));
    hipLaunchKernelGGL((head_product_kernel<T, T, float, true>), grid, dim3(256), 0, stream, b, static_cast<const T*>(q), int64_t{N + kRope},
                       static_cast<const T*>(w_k), q_lat, int64_t{L}, H, N, R, static_cast<const T*>(q) + N, kRope);
    PA_HIP(hipGetLastError());
    if (const int rc = launch_rows<float, T, KV8>(q_lat, b, H, R, scale, o_lat, stream)) return rc;
    hipLaunchKernelGGL((head_product_kernel<float, T, T, false>), grid, dim3(256), 0, stream, b, o_lat, int64_t{R}, static_cast<const T*>(w_v),
                       static_cast<T*>(out), int64_t{N}, H, R, N, static_cast<const float*>(nullptr), 0);
    PA_HIP(hipGetLastError());
    return PA_OK;
}

int latent_expanded_rows(const void* q, const LatentBatch& b, const void* w_k, const void* w_v, int H, int R, int N, int dtype, float scale, void* out,
                         void* scratch, hipStream_t stream) {
    float* const f = static_cast<float*>(scratch);
    if (dtype == PA_F32) return expanded_rows<float, false>(q, b, w_k, w_v, H, R, N, scale, out, f, stream);
    if (dtype == PA_BF16) return expanded_rows<__hip_bfloat16, false>(q, b, w_k, w_v, H, R, N, scale, out, f, stream);
    return expanded_rows<__hip_bfloat16, true>(q, b, w_k, w_v, H, R, N, scale, out, f, stream);
}
size_t latent_expanded_rows_bytes(int64_t T, int H, int R) { return static_cast<size_t>(T) * H * (2 * R + kRope) * 4; }

}  // namespace pa
