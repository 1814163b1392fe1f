// The pool of latent rows: size, scatter of new rows, and the way back (layout: latent.h).
//
// Pure data movement, bound by memory from some thousand rows on and by the launch below.  A row of R + kRope elements is 72 (bf16,
// R = 512) or more pieces of 16 bytes; a thread moves one at a time, rows lie behind one another on the caller's side, so whole
// lines are read and written on both.  With the 8-bit pool R / 8 lanes share a row's latent part, 8 elements each (16 bytes on the
// caller's side, 8 bytes of codes): the row's exponent needs the largest magnitude of all of it, a maximum over these lanes, which
// sit side by side in one wave.
// Measured: 16 384 rows of 512 + 64 into the 8-bit pool and back 16 us (3.6 TB/s); 100 003 rows back 44 us (4.1 TB/s, of 5.1 that a large copy reaches).
#include "fp8_rows.h"
#include "latent.h"

namespace pa {

template <bool kToPool>
__global__ __launch_bounds__(256) void latent_rows_kernel(uint4* __restrict__ pool, const int32_t* __restrict__ slots, uint4* __restrict__ dense,
                                                          int64_t n, unsigned vec_per_row, int64_t num_slots) {
    const int64_t total = n * vec_per_row;
    for (int64_t x = blockIdx.x * 256ll + threadIdx.x; x < total; x += gridDim.x * 256ll) {
        const int64_t t = total <= UINT32_MAX ? static_cast<unsigned>(x) / vec_per_row : x / vec_per_row;
        const unsigned c = static_cast<unsigned>(x - t * vec_per_row);
        const int64_t slot = slots[t];
        if (slot < 0 || slot >= num_slots) continue;  // never touch memory outside the pool
        if (kToPool) pool[slot * vec_per_row + c] = dense[x];
        else dense[x] = pool[slot * vec_per_row + c];
    }
}

// A wave takes 64 / (R / 8) rows at a time: all lanes for the latent parts, then the first eight of each row's for the rotary part.
template <int R, bool kToPool>
__global__ __launch_bounds__(256) void latent8_rows_kernel(unsigned char* __restrict__ pool, signed char* __restrict__ exps,
                                                           const int32_t* __restrict__ slots, uint4* __restrict__ dense, int64_t n,
                                                           int64_t num_slots) {
    constexpr int LPR = R / 8, ROWB = R + 2 * kRope, DV = (R + kRope) / 8;  // lanes per row; bytes of a pool row; 16-byte pieces of a dense one
    const int c = threadIdx.x % LPR;
    for (int64_t t = blockIdx.x * (256ll / LPR) + threadIdx.x / LPR; t < n; t += gridDim.x * (256ll / LPR)) {
        const int64_t slot = slots[t];
        if (slot < 0 || slot >= num_slots) continue;  // (the whole row agrees)
        unsigned char* const row = pool + slot * ROWB;
        uint4* const d = dense + t * DV;
        if (kToPool) {
            const uint4 in = d[c];
            if (c < kRope / 8) reinterpret_cast<uint4*>(row + R)[c] = d[LPR + c];
            const unsigned w[4] = {in.x, in.y, in.z, in.w};
            unsigned amax = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) amax = max(amax, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
#pragma unroll
            for (int off = 1; off < LPR; off <<= 1) amax = max(amax, static_cast<unsigned>(__shfl_xor(static_cast<int>(amax), off)));
            const int k = fp8_row_exponent(amax);
            unsigned o[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                o[i] = fp8_encode(w[2 * i] & 0xFFFFu, k) | (fp8_encode(w[2 * i] >> 16, k) << 8) | (fp8_encode(w[2 * i + 1] & 0xFFFFu, k) << 16) |
                       (fp8_encode(w[2 * i + 1] >> 16, k) << 24);
            reinterpret_cast<uint2*>(row)[c] = make_uint2(o[0], o[1]);
            if (c == 0) exps[slot] = static_cast<signed char>(k);
        } else {
            const uint2 in = reinterpret_cast<const uint2*>(row)[c];
            const float scale = fp8_scale(exps[slot]);
            if (c < kRope / 8) d[LPR + c] = reinterpret_cast<const uint4*>(row + R)[c];
            const uint2 a = fp8_decode4(in.x, scale), b = fp8_decode4(in.y, scale);
            d[c] = make_uint4(a.x, a.y, b.x, b.y);
        }
    }
}

static int check_latent_pool(const char* fn, const void* pool, const void* slots, const void* rows, int64_t n, int R, int P, int64_t num_slots,
                             int dtype) {
    PA_REQUIRE(n >= 0 && n <= INT32_MAX, "%s: bad row count %lld", fn, static_cast<long long>(n));
    PA_REQUIRE(dtype == PA_F32 || dtype == PA_BF16 || dtype == PA_BF16_KV8, "%s: unknown dtype %d", fn, dtype);
    PA_REQUIRE(latent_shape_ok(1, R, P), "%s: unsupported shape R=%d P=%d", fn, R, P);
    PA_REQUIRE(num_slots > 0 && num_slots <= INT32_MAX, "%s: bad num_slots %lld", fn, static_cast<long long>(num_slots));
    if (n == 0) return PA_OK;
    PA_REQUIRE(pool && slots && rows, "%s: NULL pointer", fn);
    PA_REQUIRE(aligned16(pool) && aligned16(rows), "%s: buffers must be 16-byte aligned", fn);
    return PA_OK;
}

template <bool kToPool>
static int move_rows(const char* fn, int prof, void* pool, const int32_t* slots, void* dense, int64_t n, int R, int P, int64_t num_slots, int dtype,
                     hipStream_t stream) {
    const int rc = check_latent_pool(fn, pool, slots, dense, n, R, P, num_slots, dtype);
    if (rc != PA_OK || n == 0) return rc;
    auto blocks = [](int64_t items) { return dim3(static_cast<unsigned>(items < 256 * 32 ? (items > 0 ? items : 1) : 256 * 32)); };
    ProfScope scope(prof, stream);
    if (dtype == PA_BF16_KV8) {
        unsigned char* const p = static_cast<unsigned char*>(pool);
        signed char* const exps = reinterpret_cast<signed char*>(p + num_slots * (R + 2 * kRope));
        if (R == 512)
            hipLaunchKernelGGL((latent8_rows_kernel<512, kToPool>), blocks((n + 3) / 4), dim3(256), 0, stream, p, exps, slots,
                               static_cast<uint4*>(dense), n, num_slots);
        else
            hipLaunchKernelGGL((latent8_rows_kernel<256, kToPool>), blocks((n + 7) / 8), dim3(256), 0, stream, p, exps, slots,
                               static_cast<uint4*>(dense), n, num_slots);
    } else {
        const unsigned vpr = static_cast<unsigned>(latent_row_bytes(R, dtype) / 16);
        hipLaunchKernelGGL(latent_rows_kernel<kToPool>, blocks((n * vpr + 255) / 256), dim3(256), 0, stream, static_cast<uint4*>(pool), slots,
                           static_cast<uint4*>(dense), n, vpr, num_slots);
    }
    PA_HIP(hipGetLastError());
    return PA_OK;
}

}  // namespace pa

extern "C" size_t pa_latent_pool_bytes(int64_t num_slots, int R, int P, int dtype) {
    if (num_slots <= 0 || num_slots > INT32_MAX || !pa::latent_shape_ok(1, R, P)) return 0;
    if (dtype != PA_F32 && dtype != PA_BF16 && dtype != PA_BF16_KV8) return 0;
    return static_cast<size_t>(num_slots) * (pa::latent_pool_row_bytes(R, dtype) + (dtype == PA_BF16_KV8 ? 1 : 0));
}

extern "C" int pa_append_latent(void* latent_pool, const int32_t* new_slots, const void* c_ext, int64_t T, int R, int P, int64_t num_slots,
                                int dtype, void* stream) {
    return pa::move_rows<true>("pa_append_latent", pa::kProfAppendLatent, latent_pool, new_slots, const_cast<void*>(c_ext), T, R, P, num_slots,
                               dtype, static_cast<hipStream_t>(stream));
}

extern "C" int pa_gather_latent(const void* latent_pool, const int32_t* slots, int64_t n, int R, int P, int64_t num_slots, int dtype, void* c_out,
                                void* stream) {
    return pa::move_rows<false>("pa_gather_latent", pa::kProfGatherLatent, const_cast<void*>(latent_pool), slots, c_out, n, R, P, num_slots, dtype,
                                static_cast<hipStream_t>(stream));
}
