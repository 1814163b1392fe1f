// pa_latent_attention and pa_latent_attention_expanded: argument validation and dispatch on dtype.
#include <cmath>

#include "latent.h"

namespace pa {
int latent_attention_f32(const void* q, const LatentBatch& b, int H, int R, float scale, void* out, hipStream_t stream);
int latent_expanded_f32(const void* q, const LatentBatch& b, const void* w_k, const void* w_v, int H, int R, int N, float scale, void* out, void* scratch,
                        hipStream_t stream);
size_t latent_expanded_f32_bytes(int64_t T, int H, int R);
size_t latent_workspace_bytes_bf16(int64_t T, int H, int R);
int latent_attention_bf16(const void* q, const LatentBatch& b, int64_t max_kv_len, int H, int R, bool kv8, float scale, void* out, void* workspace,
                          hipStream_t stream);
size_t latent_expanded_bytes(int B, int64_t T, int64_t max_kv_len, int H, int R, int N, int64_t num_slots);
int latent_expanded_bf16(const void* q, const LatentBatch& b, const void* w_k, const void* w_v, int64_t max_kv_len, int H, int R, int N, bool kv8,
                         float scale, void* out, void* workspace, hipStream_t stream);

constexpr int kMaxRequests = 65536;

static bool sizes_ok(int B, int64_t T, int64_t max_kv_len, int H, int R, int P, int dtype) {
    return B >= 0 && B <= kMaxRequests && T >= 0 && max_kv_len >= 0 && latent_shape_ok(H, R, P) && T <= INT32_MAX / H - 256 &&
           max_kv_len <= INT32_MAX / 2 && (dtype == PA_F32 || dtype == PA_BF16 || dtype == PA_BF16_KV8);
}

// What both forms ask of their arguments.  *nothing: an empty batch (no pointer is looked at then).
static int check(const char* fn, const void* q, const LatentBatch& b, int64_t max_kv_len, int H, int R, int P, int dtype, float scale,
                 const void* out, const void* workspace, size_t workspace_bytes, size_t need, bool* nothing) {
    *nothing = false;
    PA_REQUIRE(dtype == PA_F32 || dtype == PA_BF16 || dtype == PA_BF16_KV8, "%s: unknown dtype %d", fn, dtype);
    PA_REQUIRE(latent_shape_ok(H, R, P), "%s: unsupported shape H=%d R=%d P=%d", fn, H, R, P);
    PA_REQUIRE(b.B >= 0 && b.T >= 0 && max_kv_len >= 0, "%s: negative size", fn);
    PA_REQUIRE(sizes_ok(b.B, b.T, max_kv_len, H, R, P, dtype), "%s: batch too large", fn);
    PA_REQUIRE(b.num_slots > 0 && b.num_slots <= INT32_MAX, "%s: bad num_slots %lld", fn, static_cast<long long>(b.num_slots));
    PA_REQUIRE(std::isfinite(scale) && scale > 0.f, "%s: scale must be positive and finite", fn);
    if (b.B == 0 || b.T == 0) {
        *nothing = true;
        return PA_OK;
    }
    PA_REQUIRE(q && b.c_ext && b.pool && b.slot_offsets && b.prefix_len && b.ext_len && b.ext_offsets && out, "%s: NULL pointer", fn);
    PA_REQUIRE(aligned16(q) && aligned16(b.c_ext) && aligned16(b.pool) && aligned16(out), "%s: tensors must be 16-byte aligned", fn);
    PA_REQUIRE(out != q && out != b.c_ext, "%s: out aliases an input", fn);
    if (need > workspace_bytes || workspace == nullptr)
        return fail(PA_ENOMEM, "%s: workspace of %zu bytes, %zu needed", fn, workspace ? workspace_bytes : size_t{0}, need);
    PA_REQUIRE((reinterpret_cast<uintptr_t>(workspace) & 255u) == 0, "%s: workspace must be 256-byte aligned", fn);
    return PA_OK;
}

}  // namespace pa

extern "C" size_t pa_latent_workspace_bytes(int B, int64_t T, int64_t max_kv_len, int H, int R, int P, int dtype) {
    if (!pa::sizes_ok(B, T, max_kv_len, H, R, P, dtype)) return 0;
    return dtype == PA_F32 ? 256 : pa::latent_workspace_bytes_bf16(T, H, R);  // (fp32 needs none; 0 means invalid)
}

extern "C" int pa_latent_attention(const void* q_ext, const void* c_ext, const void* latent_pool, const int32_t* slot_idx,
                                   const int32_t* slot_offsets, const int32_t* prefix_len, const int32_t* ext_len, const int32_t* ext_offsets,
                                   int B, int64_t T, int64_t max_kv_len, int H, int R, int P, int64_t num_slots, int dtype, float scale, void* out,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    const pa::LatentBatch b = {c_ext, latent_pool, slot_idx, slot_offsets, prefix_len, ext_len, ext_offsets, B, T, num_slots};
    bool nothing = false;
    const size_t need = pa_latent_workspace_bytes(B, T, max_kv_len, H, R, P, dtype);
    if (const int rc = pa::check("pa_latent_attention", q_ext, b, max_kv_len, H, R, P, dtype, scale, out, workspace, workspace_bytes, need, &nothing))
        return rc;
    if (nothing) return PA_OK;
    if (dtype != PA_F32)
        return pa::latent_attention_bf16(q_ext, b, max_kv_len, H, R, dtype == PA_BF16_KV8, scale, out, workspace, static_cast<hipStream_t>(stream));
    return pa::latent_attention_f32(q_ext, b, H, R, scale, out, static_cast<hipStream_t>(stream));
}

extern "C" size_t pa_latent_expanded_workspace_bytes(int B, int64_t T, int64_t max_kv_len, int H, int R, int P, int N, int64_t num_slots, int dtype) {
    if (!pa::sizes_ok(B, T, max_kv_len, H, R, P, dtype) || (N != 64 && N != 128) || num_slots <= 0 || num_slots > INT32_MAX) return 0;
    if (dtype != PA_F32) return pa::latent_expanded_bytes(B, T, max_kv_len, H, R, N, num_slots);  // (0: too many rows)
    const size_t n = pa::latent_expanded_f32_bytes(T, H, R);
    return n > 256 ? n : 256;  // (an empty batch needs none; 0 means invalid)
}

extern "C" int pa_latent_attention_expanded(const void* q_ext, const void* c_ext, const void* w_k, const void* w_v, const void* latent_pool,
                                            const int32_t* slot_idx, const int32_t* slot_offsets, const int32_t* prefix_len, const int32_t* ext_len,
                                            const int32_t* ext_offsets, int B, int64_t T, int64_t max_kv_len, int H, int R, int P, int N,
                                            int64_t num_slots, int dtype, float scale, void* out, void* workspace, size_t workspace_bytes,
                                            void* stream) {
    const char* const fn = "pa_latent_attention_expanded";
    const pa::LatentBatch b = {c_ext, latent_pool, slot_idx, slot_offsets, prefix_len, ext_len, ext_offsets, B, T, num_slots};
    PA_REQUIRE(N == 64 || N == 128, "%s: unsupported shape N=%d", fn, N);
    bool nothing = false;
    const size_t need = pa_latent_expanded_workspace_bytes(B, T, max_kv_len, H, R, P, N, num_slots, dtype);
    if (const int rc = pa::check(fn, q_ext, b, max_kv_len, H, R, P, dtype, scale, out, workspace, workspace_bytes, need, &nothing)) return rc;
    if (nothing) return PA_OK;
    PA_REQUIRE(need != 0, "%s: batch too large", fn);
    PA_REQUIRE(w_k && w_v, "%s: NULL pointer", fn);
    PA_REQUIRE(pa::aligned16(w_k) && pa::aligned16(w_v), "%s: tensors must be 16-byte aligned", fn);
    PA_REQUIRE(out != w_k && out != w_v, "%s: out aliases an input", fn);
    if (dtype != PA_F32)
        return pa::latent_expanded_bf16(q_ext, b, w_k, w_v, max_kv_len, H, R, N, dtype == PA_BF16_KV8, scale, out, workspace, static_cast<hipStream_t>(stream));
    return pa::latent_expanded_f32(q_ext, b, w_k, w_v, H, R, N, scale, out, workspace, static_cast<hipStream_t>(stream));
}
