// Latent attention on the bf16 matrix cores, absorbed form (MFMA 16x16x32, fp32 accumulation), gfx950.
//
// A row (c, r) of R latent and kRope rotary values is the key of all H query heads, and c their value:
//     S = Q K^T (R + kRope deep),  P = 2^(c S - m),  O = P C (R columns),  out = O / sum P.
// Per cached row 2 (2 R + kRope) H operations for 2 (R + kRope) bytes: with 16 heads memory bounds it, with 128 the matrix cores about as
// much as memory, from two new tokens on the matrix cores.
//
// Tiles.  The rows of q of a request (token, head) are one axis, so that a tile of M rows reads every cached row once for all of its heads and
// tokens.  Four waves, M = 128, 64 or 32.  What decides the layout is the width of the output: 512 fp32 columns for 128 rows are 256 KB, half of a
// compute unit's registers, so one workgroup is resident, a wave per SIMD with 512 registers, and the two products are split differently:
//   scores: a wave computes 32 rows x 32 keys (M = 64: 32 x 16, M = 32: 16 x 16), its rows of Q in registers (M = 128: four of 18 slices in LDS);
//   output: a wave computes all M rows x a quarter of the columns, so that a fragment of C read from LDS is multiplied with eight blocks of
//           rows; the probabilities go through LDS in between.  (A wave with the output of its own 32 rows would read every fragment of C for
//           two products only: 68 KB of LDS reads per wave and step instead of 52, and LDS, not the matrix cores, would be the bound.)
// Scores are computed transposed (S^T = K Q^T): a lane holds one row of q per block and four keys, the output as O^T = C^T P^T, C^T by the
// transposing LDS read, so that row maxima and sums are per lane and O's rows too.
//
// Pipeline.  A step is 32 keys.  In one interval between two barriers a wave computes the scores of step i + 1, then the output of step i and beside its
// products the probabilities of step i + 1.  Rows are loaded straight into LDS, two steps ahead of the output (M = 128) or three, their loads set out beside the first
// products of the scores.  The running maximum of a row moves only when a lane's probabilities of a step sum to more than kMost: the wave that sees it sets a
// flag, which all waves find in the next interval, and they settle on new maxima together (settle()), the scores computed once more; until then a
// probability may be as large as kMost, which fp32 and bf16 hold as exactly as 1.  Against maxima so large that their rounding shows (moved_maximum()) those of the
// settlement itself are held to 2^kCap; the step counts as done then.
//
// Measured: 64 heads, 16 requests of 20 to 80 new tokens over 4 documents of 16 384 rows (1.9 TFLOP): 1800 us, 1.05 PFLOP/s, where a plain product of 16 384
// squared reaches 1.39; the matrix cores are busy 45 % of the cycles, LDS 23 %, a wave waits a quarter of its own: none is full, but there is one wave on a SIMD, and
// nothing beside it while it waits.  128 heads, 128 requests of one token, 500 to 7800 keys: 258 us (27 %, 14 %, 39 %).
// 16 heads, 48 requests, 2000 to 24 000 keys of the 8-bit pool: 172 us, 2.7 TB/s, bound by what a step does outside its products, most of it turning codes into bf16.
//
// LDS is swizzled in pieces of 16 bytes (swz()) so that reading 16 bytes down 16 rows and the transposing reads of 8 bytes across 8 rows are both
// free of bank conflicts; direct loads write 1 KB of consecutive LDS, so the swizzle is applied to the address in memory.
//
// 8-bit pool: codes land in a buffer of their own and are turned into bf16 rows by the wave that loaded them, one step before they are used.
#include <hip/hip_bf16.h>

#include <type_traits>

#include "fp8_rows.h"
#include "latent_merge.h"
#include "latent_work.h"
#include "wave_ops.h"

namespace pa {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// The products of the scores, with their results in vector registers: left to the compiler they take accumulation registers, of which the output needs all
// 256, and are copied.  What reads the results waits for them first (products_done).
__device__ __forceinline__ void mfma_first(f32x4& d, bf16x8 a, bf16x8 b) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, 0" : "=&v"(d) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_next(f32x4& d, bf16x8 a, bf16x8 b) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(d) : "v"(a), "v"(b));
}
// ... and one whose result the compiler may move right behind it: the wait is part of it
__device__ __forceinline__ void mfma_next_done(f32x4& d, bf16x8 a, bf16x8 b) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0\n\ts_nop 15\n\ts_nop 1" : "+v"(d) : "v"(a), "v"(b));
}
__device__ __forceinline__ void products_done() { asm volatile("s_nop 15\n\ts_nop 3" ::: "memory"); }

constexpr int kStep = 32;       // keys of a step
constexpr float kMost = 1099511627776.f;  // 2^40
constexpr float kCap = 36.f;    // log2 of a probability against a maximum that has just moved, at most: eight of them are less than kMost

__device__ const uint4 g_zero_row[128] = {};  // stands for keys behind the last one of a tile

// XOR of the 16-byte piece of a latent row in LDS, by the row's number within 16; and of its rotary part (8 pieces)
// (A read of 16 bytes per lane is served 16 lanes at a time, not in their order but 0 .. 3, 12 .. 15, 20 .. 27 and so on: a quarter of the lanes has its
// neighbour's piece.  With another order of the row's bits, right for lanes in their order, two fifths of the LDS cycles were conflicts.)
__device__ __forceinline__ int swz(int row) { return ((row & 1) << 3) | ((row & 2) << 1) | ((((row >> 2) ^ (row >> 3)) & 1) << 1) | ((row >> 2) & 1); }
// ... of a row of 64 bytes (4 pieces)
__device__ __forceinline__ int swz_64(int row) { return ((((row >> 2) ^ (row >> 3)) & 1) << 1) | ((row >> 3) & 1); }
__device__ __forceinline__ int swz_rope(int row) { return (row >> 1) & 7; }

template <int R, int M, bool KV8>
struct LatentShape {
    static constexpr int kAhead = M == 128 ? 2 : 3;  // steps that loads are ahead of the step whose output is computed
    static constexpr int kLatRow = 2 * R, kLat = kStep * kLatRow;  // bytes of a latent row and of a step's
    static constexpr int kLatSlots = KV8 ? 3 : kAhead + 1, kRopeSlots = kAhead + 1, kRopeStep = kStep * 2 * kRope;
    static constexpr int kCodes = KV8 ? kStep * R : 0, kCodeSlots = kAhead - 1;
    static constexpr int kProb = M * kStep * 2;
    // slices of 32 values of Q that lie in LDS and not in registers
    static constexpr int kQLds = M == 128 && R == 512 ? (KV8 ? 2 : 4) : 0, kQSlice = M * 64;
    static constexpr int kRopeAt = kLatSlots * kLat, kCodesAt = kRopeAt + kRopeSlots * kRopeStep, kProbAt = kCodesAt + kCodeSlots * kCodes,
                         kQAt = kProbAt + 2 * kProb, kMaxAt = kQAt + kQLds * kQSlice, kRedAt = kMaxAt + 4 * M, kFlagAt = kRedAt + 8 * M, kSlotsAt = kFlagAt + 16,
                         kExpAt = kSlotsAt + 4 * 2 * 256, kBytes = kExpAt + (KV8 ? 4 * 2 * 32 : 0);
    static_assert(kBytes <= 160 * 1024, "LDS");
};

template <int R, int M, bool KV8>
__global__ __launch_bounds__(256, 1) void latent_bf16_kernel(const __hip_bfloat16* __restrict__ q_ext, LatentBatch b, LatentSplit split, float scale_log2e,
                                                             __hip_bfloat16* __restrict__ out, LatentParts parts) {
    using X = LatentShape<R, M, KV8>;
    constexpr int L = R + kRope, KS = R / 32, KSR = kRope / 32;    // k-slices of the latent and the rotary part
    constexpr int RW = M >= 64 ? 2 : 1, KW = M == 128 ? 2 : 1;    // blocks of 16 rows and of 16 keys of a wave's scores
    constexpr int KG = M == 128 ? 1 : 2;                           // waves that share a row's scores
    constexpr int RB = M / 16, NB = R / 64;                        // blocks of the output: rows, and 16 columns each of the wave's quarter
    constexpr int RPL = 512 / R;                                   // latent rows of a 1 KB load
    constexpr int PROW = KV8 ? R + 2 * kRope : 2 * L;              // bytes of a pool row
    constexpr int kLoads = KV8 ? 8 * R / 1024 + 2 : 8 / RPL + 1;   // loads per wave of a step whose rows are all in the pool
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g4 = lane >> 4;
    int wl = 0, at_work = 0;
    LatentPlace at, end;
    bool over = false;
    const bool any = latent_share(b, split, blockIdx.x, reinterpret_cast<LatentScratch*>(smem), &wl, &at_work, &at, &end, &over);
    if (blockIdx.x == 0 && tid == 0) {
        parts.hdr[3] = over;
        parts.hdr[6] = at_work;
    }
    if (!any) return;

    const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));
    auto* const lds = (__attribute__((address_space(3))) unsigned char*)smem;
    auto* const s_max = reinterpret_cast<float*>(smem + X::kMaxAt);
    auto* const s_red = reinterpret_cast<float*>(smem + X::kRedAt);  // [KG][M]
    auto* const s_flag = reinterpret_cast<int*>(smem + X::kFlagAt);
    auto* const s_slots = reinterpret_cast<int*>(smem + X::kSlotsAt) + wave * 128;

    // the wave's part of the scores
    const int wrow = M == 128 ? 32 * wave : 16 * RW * (wave & 1), wkey = M == 128 ? 0 : 16 * (wave >> 1), kgroup = M == 128 ? 0 : wave >> 1;
    // LDS read addresses: K fragments (16 rows from wkey on, piece 4 s + g4), by s mod 4; rotary; C^T fragments; probabilities
    unsigned k_at[4], r_at[KSR], v_at;
#pragma unroll
    for (int s = 0; s < 4; ++s) k_at[s] = (wkey + n) * X::kLatRow + 16 * ((4 * s + g4) ^ swz(n));
#pragma unroll
    for (int s = 0; s < KSR; ++s) r_at[s] = X::kRopeAt + (wkey + n) * 2 * kRope + 16 * ((4 * s + g4) ^ swz_rope(n));
    {
        const int row = 8 * g4 + (n >> 2);  // and 4 more
        const int piece = (16 * NB * wave >> 3) + ((n & 3) >> 1);
        v_at = row * X::kLatRow + 16 * (piece ^ swz(row & 15)) + 8 * (n & 1);
    }
    // (probabilities: 64 bytes a row, in pieces of 16; the second block of 16 keys by XOR)
    const unsigned p_wr = X::kProbAt + (wrow + n) * 64 + 16 * (((wkey >> 3) + (g4 >> 1)) ^ swz_64(n)) + 8 * (g4 & 1);
    [[maybe_unused]] const unsigned q_at = X::kQAt + (wrow + n) * 64 + 16 * (g4 ^ swz_64(n));
    const unsigned p_rd = X::kProbAt + n * 64 + 16 * (g4 ^ swz_64(n));

    bool used[2] = {false, false};  // partial results left in this workgroup's two slots
    while (!(at.r == end.r && at.tile == end.tile && at.k == end.k)) {
        bool unused = false;
        LatentRequest req = latent_request(b, split, at.r, &unused);
        req.P = __builtin_amdgcn_readfirstlane(req.P);
        req.rows = __builtin_amdgcn_readfirstlane(req.rows);
        req.tiles = __builtin_amdgcn_readfirstlane(req.tiles);
        if (at.tile >= req.tiles) {
            if (++at.r >= b.B) break;
            at.tile = at.k = 0;
            continue;
        }
        const int H = split.rpt, P = req.P, row0 = at.tile * M, rows_here = min(M, req.rows - row0);
        const int64_t e0 = __builtin_amdgcn_readfirstlane(b.ext_offsets[at.r]);
        const int32_t* __restrict__ slots = b.slot_idx + __builtin_amdgcn_readfirstlane(b.slot_offsets[at.r]);
        const int key_end = latent_keys(split, req, at.tile), all_steps = (key_end + kStep - 1) / kStep;
        const int k0 = at.k, k1 = at.r == end.r && at.tile == end.tile ? end.k : all_steps, steps = k1 - k0;
        const int vis_min = P + row0 / H + 1;  // every row of the tile sees the keys before this one
        const int64_t out_row0 = e0 * H + row0;

        // ---- loads of a step: the wave's rows 8 wave .. + 7 ----
        const unsigned char* const pool = static_cast<const unsigned char*>(b.pool);
        const unsigned char* const c_rows = static_cast<const unsigned char*>(b.c_ext) + e0 * (2 * L);
        auto row_address = [&](int j, int slot) -> uint64_t {
            const unsigned s = min(static_cast<unsigned>(max(slot, 0)), static_cast<unsigned>(b.num_slots - 1));  // never outside the pool
            const uint64_t in_pool = reinterpret_cast<uint64_t>(pool) + static_cast<uint64_t>(s) * PROW;
            const uint64_t in_ext = reinterpret_cast<uint64_t>(c_rows) + static_cast<uint64_t>(max(j - P, 0)) * (2 * L);
            uint64_t not_cached = j < key_end ? in_ext : reinterpret_cast<uint64_t>(g_zero_row);
            if (KV8 && M < 128) asm("" : "+v"(not_cached));  // (chosen, not branched around: a step asks for six addresses here, 16 heads of long requests 181 to 174 us)
            return j < P ? in_pool : not_cached;
        };
        // slot ids of eight steps from step k0 + 8 blk on, lane: step lane / 8, row lane % 8
        auto load_slots = [&](int blk) {
            const int first = (k0 + 8 * blk) * kStep;
            if (first < P) {
                const int j = first + (lane >> 3) * kStep + 8 * wave + (lane & 7);
                load_to_lds_4(slots + min(j, P - 1), lds0 + X::kSlotsAt + wave * 512 + (blk & 1) * 256);
            }
        };
        // The loads of a step, in kIssue pieces, so that they can stand between matrix instructions: what they need, then one or two at a time.  (Steps behind
        // the last are loaded too, as rows of zeros: every interval has the same loads.)
        uint64_t row_at = 0, rope_at = 0;
        int slot_a = 0, slot_b = 0;
        constexpr int kRowLoads = KV8 ? 8 * R / 1024 : 8 / RPL, kIssue = 3 + kRowLoads;
        auto issue_piece = [&](int piece, int rel, int lat_slot, int rope_slot) __attribute__((always_inline)) {
            const int lane = static_cast<int>(worked_out_here(tid)) & 63;
            const int j0 = (k0 + rel) * kStep + 8 * wave;
            const int* const sl = s_slots + ((rel >> 3) & 1) * 64 + (rel & 7) * 8;
            if (piece == 0) {
                slot_a = sl[lane & 7];
                slot_b = sl[lane >> 3];
            } else if (piece == 1) {
                row_at = row_address(j0 + (lane & 7), slot_a);
                const int row = lane >> 3, j = j0 + row;
                rope_at = row_address(j, slot_b) + ((KV8 && j < P ? R : 2 * R) + 16 * ((lane & 7) ^ swz_rope((8 * wave + row) & 15)));
            } else if (piece == 2) {
                load_to_lds_16(reinterpret_cast<const void*>(rope_at), lds0 + X::kRopeAt + rope_slot * X::kRopeStep + 8 * wave * 2 * kRope);
                if constexpr (KV8) {
                    const unsigned char* const exps = pool + static_cast<uint64_t>(b.num_slots) * PROW;
                    if (lane < 8 && j0 + lane < P)
                        load_to_lds_1(exps + min(static_cast<unsigned>(max(slot_a, 0)), static_cast<unsigned>(b.num_slots - 1)),
                                      lds0 + X::kExpAt + wave * 64 + (rel & 1) * 32);
                }
            } else {
                const int i = piece - 3;
                if constexpr (KV8) {
                    const int row = i * (1024 / R) + lane / (R / 16);
                    if (j0 + row < P)
                        load_to_lds_16(reinterpret_cast<const unsigned char*>(row_address(j0 + row, sl[row])) + 16 * (lane % (R / 16)),
                                       lds0 + X::kCodesAt + (rel & (X::kCodeSlots - 1)) * X::kCodes + 8 * wave * R + i * 1024);
                } else if constexpr (RPL == 1) {
                    const unsigned lo = static_cast<unsigned>(row_at), hi = static_cast<unsigned>(row_at >> 32);
                    // (readlane gives a signed word: it must not be extended by its sign)
                    const uint64_t base = static_cast<unsigned>(__builtin_amdgcn_readlane(lo, i)) | static_cast<uint64_t>(static_cast<unsigned>(__builtin_amdgcn_readlane(hi, i))) << 32;
                    load_to_lds_16(reinterpret_cast<const void*>(base), 16u * (lane ^ swz((8 * wave + i) & 15)), lds0 + lat_slot * X::kLat + (8 * wave + i) * X::kLatRow);
                } else {
                    const int row = i * RPL + lane / (64 / RPL);
                    load_to_lds_16(reinterpret_cast<const unsigned char*>(row_address(j0 + row, sl[row])) + 16 * ((lane & (64 / RPL - 1)) ^ swz((8 * wave + row) & 15)),
                                   lds0 + lat_slot * X::kLat + 8 * wave * X::kLatRow + i * 1024);
                }
            }
        };
        auto issue = [&](int rel, int lat_slot, int rope_slot) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kIssue; ++i) issue_piece(i, rel, lat_slot, rope_slot);
        };
        // 8-bit pool.  All rows of a step are in the pool: its loads are kLoads, no row goes to its place in LDS directly.
        auto pure = [&](int rel) { return !KV8 || (k0 + rel + 1) * kStep <= P; };
        // rows that are bf16 in memory (extend tokens, and what stands for keys behind the last), to their place
        auto issue_direct = [&](int rel, int lat_slot) {
            const int j0 = (k0 + rel) * kStep + 8 * wave;
            const unsigned lat = lds0 + lat_slot * X::kLat + 8 * wave * X::kLatRow;
#pragma unroll
            for (int i = 0; i < 8 / RPL; ++i) {
                const int row = i * RPL + lane / (64 / RPL);
                if (j0 + row >= P)
                    load_to_lds_16(reinterpret_cast<const unsigned char*>(row_address(j0 + row, 0)) + 16 * ((lane & (64 / RPL - 1)) ^ swz((8 * wave + row) & 15)),
                                   lat + i * 1024);
            }
        };
        // codes that landed, to bf16 rows (the wave's own)
        auto convert = [&](int rel, int lat_slot) __attribute__((always_inline)) {
            const int j0 = (k0 + rel) * kStep + 8 * wave;
            const unsigned from = X::kCodesAt + (rel & (X::kCodeSlots - 1)) * X::kCodes + 8 * wave * R, exps = X::kExpAt + wave * 64 + (rel & 1) * 32;
            const unsigned to = lat_slot * X::kLat + 8 * wave * X::kLatRow;
            const int piece = lane & (64 / RPL - 1);
            // (Reads before the first write, whose order the compiler keeps: all of a step, 16 heads of long requests 191 to 178 us, except in tiles of 128 rows, whose
            // accumulators leave no registers for it.)
            constexpr int kTogether = M == 128 ? 1 : 8 / RPL;
#pragma unroll
            for (int i0 = 0; i0 < 8 / RPL; i0 += kTogether) {
                u32x2 codes[kTogether];
                signed char k[kTogether];
#pragma unroll
                for (int i = 0; i < kTogether; ++i) {
                    const int row = (i0 + i) * RPL + lane / (64 / RPL);
                    codes[i] = *reinterpret_cast<__attribute__((address_space(3))) const u32x2*>(lds + from + row * R + 8 * piece);
                    k[i] = *reinterpret_cast<__attribute__((address_space(3))) const signed char*>(lds + exps + 4 * row);
                }
#pragma unroll
                for (int i = 0; i < kTogether; ++i) {
                    const int row = (i0 + i) * RPL + lane / (64 / RPL);
                    const float two_k = fp8_scale(k[i]);
                    const uint2 x = fp8_decode4(codes[i][0], two_k), y = fp8_decode4(codes[i][1], two_k);
                    if (j0 + row < P)
                        *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(lds + to + row * X::kLatRow + 16 * (piece ^ swz((8 * wave + row) & 15))) =
                            u32x4{x.x, x.y, y.x, y.y};
                }
            }
        };

        // ---- the wave's rows of Q ----
        constexpr int KQ = KS + KSR - X::kQLds;  // slices in registers
        bf16x8 q[RW][KQ];
        load_slots(0);
#pragma unroll
        for (int rb = 0; rb < RW; ++rb) {
            const int row = min(wrow + 16 * rb + n, rows_here - 1);  // (rows behind the last repeat it)
            const uint4* const src = reinterpret_cast<const uint4*>(q_ext + (out_row0 + row) * L);
#pragma unroll
            for (int s = 0; s < KQ; ++s) q[rb][s] = __builtin_bit_cast(bf16x8, src[4 * s + g4]);
#pragma unroll
            for (int s = KQ; s < KS + KSR; ++s)
                *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(lds + q_at + (s - KQ) * X::kQSlice + rb * 1024) = __builtin_bit_cast(u32x4, src[4 * s + g4]);
        }
        float m[RW], l[RW];
#pragma unroll
        for (int rb = 0; rb < RW; ++rb) m[rb] = l[rb] = 0.f;
        if (tid < 3) s_flag[tid] = tid < 2 ? -1 : 0;
        wait_vm_all();
        load_slots(1);
        issue(0, 0, 0);
        if (KV8 && !pure(0)) issue_direct(0, 0);
        if (!KV8 || X::kAhead == 3) {
            if (steps > 1) issue(1, 1, 1);
            if (KV8 && steps > 1 && !pure(1)) issue_direct(1, 1);
        }
        if (!KV8 && X::kAhead == 3 && steps > 2) issue(2, 2, 2);

        // ---- the pieces of an interval ----
        // Keys that some row of the tile does not see may hold an infinity or NaN, and 0 times that is NaN: before the output of a step with such keys, when
        // its scores are done, the wave that loaded a row takes such values out of it; the end of the tile makes the column NaN for the rows that see them.
        auto has_hidden = [&](int rel) { return vis_min < key_end && (k0 + rel + 1) * kStep > vis_min; };
        auto clean = [&](int lat_slot) {
            const unsigned at_row = lat_slot * X::kLat + 8 * wave * X::kLatRow + 16 * worked_out_here(lane);
#pragma unroll
            for (int i = 0; i < 8 / RPL; ++i) {
                auto* const c8 = reinterpret_cast<__attribute__((address_space(3))) s16x8*>(lds + at_row + 1024 * i);
                s16x8 y = *c8;
                bool odd = false;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if ((y[e] & 0x7F80) == 0x7F80) {
                        odd = true;
                        y[e] = 0;
                    }
                if (odd) {
                    *c8 = y;
                    s_flag[2] = 1;
                }
            }
        };
        f32x4 sc[KW][RW];
        // Scores of a step; fragments are read kAhead ahead.  Between the products, the loads of step load_rel.
        auto scores = [&](int rel, int lat_slot, int rope_slot, auto with, int load_rel, int load_lat, int load_rope) __attribute__((always_inline)) {
            constexpr bool loads = decltype(with)::value;
            constexpr int kFrags = KW * (KS + KSR), kAhead = 4;
            static_assert(kIssue <= kFrags, "a product for each of them");
            const unsigned lat = lat_slot * X::kLat, rope = rope_slot * X::kRopeStep;
            u32x4 kf[kAhead + 1];
            u32x4 qf[2][RW];  // (of the slices of Q in LDS, one ahead)
            auto read_q = [&](int s) __attribute__((always_inline)) {
#pragma unroll
                for (int rb = 0; rb < RW; ++rb) qf[s & 1][rb] = *reinterpret_cast<__attribute__((address_space(3))) const u32x4*>(lds + q_at + (s - KQ) * X::kQSlice + rb * 1024);
            };
            auto read = [&](int f) __attribute__((always_inline)) {
                const int s = f / KW, kb = f % KW;
                kf[f % (kAhead + 1)] = *reinterpret_cast<__attribute__((address_space(3))) const u32x4*>(
                    s < KS ? lds + (k_at[s & 3] + lat) + kb * 16 * X::kLatRow + (s >> 2) * 256 : lds + (r_at[s < KS ? 0 : s - KS] + rope) + kb * 16 * 2 * kRope);
            };
#pragma unroll
            for (int f = 0; f < kAhead; ++f) read(f);
            in_this_order();
#pragma unroll
            for (int f = 0; f < kFrags; ++f) {
                const int s = f / KW, kb = f % KW;
                if (f + kAhead < kFrags) read(f + kAhead);
                if (kb == 0 && s + 1 >= KQ && s + 1 < KS + KSR) read_q(s + 1);
#pragma unroll
                for (int rb = 0; rb < RW; ++rb)
                    if (s == 0) mfma_first(sc[kb][rb], __builtin_bit_cast(bf16x8, kf[f % (kAhead + 1)]), q[rb][0]);
                    else mfma_next(sc[kb][rb], __builtin_bit_cast(bf16x8, kf[f % (kAhead + 1)]), s < KQ ? q[rb][s < KQ ? s : 0] : __builtin_bit_cast(bf16x8, qf[s & 1][rb]));
                if constexpr (loads) {
                    // (as early as can be: spread over all of the products, a step of 128 rows took a tenth longer)
                    if (f < kIssue) issue_piece(f, load_rel, load_lat, load_rope);
                }
                in_this_order();
            }
            products_done();
            in_this_order();
            const int j0 = (k0 + rel) * kStep;
            if (j0 + kStep > vis_min) {
                const int lane_now = static_cast<int>(worked_out_here(lane));
#pragma unroll
                for (int rb = 0; rb < RW; ++rb) {
                    const int row = min(wrow + 16 * rb + (lane_now & 15), rows_here - 1);
                    const int sees = P + (row0 + row) / H + 1 - j0 - wkey - 4 * (lane_now >> 4);
#pragma unroll
                    for (int kb = 0; kb < KW; ++kb)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (16 * kb + i >= sees) sc[kb][rb][i] = -INFINITY;
                }
            }
        };
        // a piece of the probabilities of the scores against the maxima as they stand, into buffer rel % 2; their sums
        // (Rounded to bf16, since a matrix instruction takes one type and the rows are bf16: a result is 1.7e-3 to 2.4e-3 off, relatively, of which 1.7e-3 is the rounding of
        // the result itself.  A second product with what the rounding left would cost as much as the first.)
        float sum[RW];
        auto probabilities = [&](int rel, int kb, int rb, auto moved) __attribute__((always_inline)) {
            float p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float z = fmaf(sc[kb][rb][i], scale_log2e, -m[rb]);
                p[i] = __builtin_amdgcn_exp2f(decltype(moved)::value && z > kCap ? kCap : z);
                sum[rb] += p[i];
            }
            *reinterpret_cast<__attribute__((address_space(3))) u32x2*>(lds + ((p_wr + (rel & 1) * X::kProb + rb * 1024) ^ (kb * 32))) =
                u32x2{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3])};
        };
        auto largest = [&](int rb) {
            float mx = sc[0][rb][0];
#pragma unroll
            for (int kb = 0; kb < KW; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[kb][rb][i]);
            return mx * scale_log2e;
        };
        // All waves agree on new maxima of all rows, from the scores at hand (step rel), and write their probabilities.  What has been summed up
        // against the old ones moves to the workgroup's scratch memory (flush), multiplied accordingly, and the accumulators begin anew.
        auto settle = [&](int rel, bool first, auto flush) {
#pragma unroll
            for (int rb = 0; rb < RW; ++rb) {
                const float mx = moved_maximum(row_max(largest(rb)));
                if (g4 == 0) s_red[kgroup * M + wrow + 16 * rb + n] = mx;
            }
            lds_barrier();
            if (tid < 2) s_flag[tid] = -1;  // (all waves have looked)
            auto new_max = [&](int row) {
                float x = s_red[row];
                if (KG == 2) x = fmaxf(x, s_red[M + row]);
                if (first) return x == -INFINITY ? kNoMaximum : x;
                return fmaxf(x, s_max[row]);
            };
            if (!first) flush([&](int row) { return __builtin_amdgcn_exp2f(s_max[row] - new_max(row)); });
#pragma unroll
            for (int rb = 0; rb < RW; ++rb) {
                const float mn = new_max(wrow + 16 * rb + n);
                l[rb] = first ? 0.f : l[rb] * __builtin_amdgcn_exp2f(m[rb] - mn);
                m[rb] = mn;
                sum[rb] = 0.f;
            }
            const float mine = tid < M ? new_max(tid) : 0.f;
            lds_barrier();
            if (tid < M) s_max[tid] = mine;
#pragma unroll
            for (int rb = 0; rb < RW; ++rb)
#pragma unroll
                for (int kb = 0; kb < KW; ++kb) probabilities(rel, kb, rb, std::true_type{});
            lds_barrier();
        };
        // Output of step rel, and beside it the probabilities of the scores at hand, of step rel + 1.
        bf16x8 pf[RB];
        s16x4 vf[4][2];
        constexpr int kVAhead = NB < 3 ? NB : 3;
        auto read_v = [&](int cb, unsigned v_here, unsigned lat) __attribute__((always_inline)) {
            const unsigned a = (v_here ^ (32 * cb)) + lat;
            vf[cb & 3][0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + a));
            vf[cb & 3][1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + (a ^ 48) + 4 * X::kLatRow));
        };
        auto output_reads = [&](int rel, int lat_slot) __attribute__((always_inline)) {
            const unsigned lat = lat_slot * X::kLat, prob = p_rd + (rel & 1) * X::kProb, v_here = worked_out_here(v_at);
            read_v(0, v_here, lat);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) pf[rb] = *reinterpret_cast<__attribute__((address_space(3))) const bf16x8*>(lds + prob + rb * 1024);
#pragma unroll
            for (int cb = 1; cb < kVAhead; ++cb) read_v(cb, v_here, lat);
            in_this_order();
        };
        auto output = [&](int rel, int lat_slot, f32x4 (&o)[RB][NB]) __attribute__((always_inline)) {
            const unsigned lat = lat_slot * X::kLat, v_here = worked_out_here(v_at);
#pragma unroll
            for (int rb = 0; rb < RW; ++rb) sum[rb] = 0.f;
            constexpr int kPieces = RW * KW, kEvery = NB / kPieces, kInVector = KV8 ? 1 : 2;
#pragma unroll
            for (int cb = 0; cb < NB; ++cb) {
                if (cb + kVAhead < NB) read_v(cb + kVAhead, v_here, lat);
                const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vf[cb & 3][0], vf[cb & 3][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    // (128 rows and 512 columns are all accumulation registers there are; what else the compiler wants some for would cost a block of the
                    // output a place in memory, and a wait for all loads each time: a few blocks have vector registers)
                    if (RB * NB == 64 && rb == RB - 1 && cb >= NB - kInVector) mfma_next_done(o[rb][cb], v, pf[rb]);
                    else o[rb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[rb], o[rb][cb], 0, 0, 0);
                }
                if (cb % kEvery == 0) probabilities(rel + 1, (cb / kEvery) % KW, (cb / kEvery) / KW, std::false_type{});
                in_this_order();
            }
        };

        // ---- the loop ----
        // (ring slots of step rel and of the steps behind it)
        int lat_slot = 0, rope_slot = 0;
        auto lat_on = [](int x, int by) { return x + by >= X::kLatSlots ? x + by - X::kLatSlots : x + by; };
        auto rope_on = [](int x, int by) { return x + by >= X::kRopeSlots ? x + by - X::kRopeSlots : x + by; };
        if constexpr (KV8) {
            wait_vm_all();
            convert(0, 0);
            if (X::kAhead == 3 && steps > 1) convert(1, 1);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the codes are read: their buffer is free)
            if (X::kAhead == 3) {
                if (steps > 2) issue(2, 2, 2);
            } else if (steps > 1) {
                issue(1, 1, 1);
                if (!pure(1)) issue_direct(1, 1);
            }
            lds_barrier();
            scores(0, 0, 0, std::false_type{}, 0, 0, 0);
            if (X::kAhead == 2 && steps > 1) {
                wait_vm_all();
                convert(1, 1);
            }
        } else {
            if (X::kAhead == 3 && steps > 2) wait_vm<2 * kLoads>();
            else if (steps > 1) wait_vm<kLoads>();
            else wait_vm_all();
            lds_barrier();
            scores(0, 0, 0, std::false_type{}, 0, 0, 0);
            if (X::kAhead == 3 && steps > 2) wait_vm<kLoads>();
            else wait_vm_all();
        }
        settle(0, true, [](auto) {});
        bool flushed = false;
        auto scratch = [&](unsigned lane_now) {
            return parts.o + (static_cast<size_t>(2 * split.n_wg + wl) * M + (lane_now & 15)) * R + 16 * NB * wave + 4 * (lane_now >> 4);
        };
        int rel = 0;  // (the sums of its probabilities are taken up when these are used)
        f32x4 o[RB][NB];
        while (true) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int cb = 0; cb < NB; ++cb) o[rb][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
            bool grown = false;
            while (true) {
                const int flag = s_flag[rel & 1];
                if ((rel & 7) == 8 - X::kAhead) load_slots((rel + X::kAhead) / 8 + 1);
                if (KV8 && rel + 2 < steps && !pure(rel + 2)) issue_direct(rel + 2, lat_on(lat_slot, 2));
                // (behind the last step: of whatever lies there, not used)
                scores(rel + 1, lat_on(lat_slot, 1), rope_on(rope_slot, 1), std::true_type{}, rel + X::kAhead, KV8 ? 0 : lat_on(lat_slot, X::kAhead), rope_on(rope_slot, X::kAhead));
                if (__builtin_amdgcn_readfirstlane(flag) == rel) {
                    grown = true;
                    break;
                }
#pragma unroll
                for (int rb = 0; rb < RW; ++rb) l[rb] += sum[rb];
                if (has_hidden(rel)) {
                    clean(lat_slot);
                    lds_barrier();
                }
                output_reads(rel, lat_slot);
                output(rel, lat_slot, o);
                bool outgrown = false;
#pragma unroll
                for (int rb = 0; rb < RW; ++rb) outgrown |= sum[rb] > kMost;
                if (__any(outgrown) && lane == 0) s_flag[(rel + 1) & 1] = rel + 1;
                if (X::kAhead == 3 && pure(rel + 3)) wait_vm<kLoads>();
                else wait_vm_all();
                if (KV8 && rel + 2 < steps) convert(rel + 2, lat_on(lat_slot, 2));
                lds_barrier();
                ++rel;
                lat_slot = lat_on(lat_slot, 1);
                rope_slot = rope_on(rope_slot, 1);
                if (rel >= steps) break;
            }
            if (!grown) {
                wait_vm_all();  // (nothing is on its way to LDS any more)
                break;
            }
            // (the scores of this step once more, and what is on its way to LDS has landed before it is asked for again)
            wait_vm_all();
            scores(rel, lat_slot, rope_slot, std::false_type{}, 0, 0, 0);
            settle(rel, false, [&](auto alpha) {
                const unsigned lane_now = worked_out_here(lane);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    const float a = alpha(16 * rb + (lane_now & 15));
#pragma unroll
                    for (int cb = 0; cb < NB; ++cb) {
                        f32x4* const to = reinterpret_cast<f32x4*>(scratch(lane_now) + 16 * rb * R + 16 * cb);
                        f32x4 x = o[rb][cb];
                        if (flushed) x += *to;
                        *to = x * a;
                    }
                }
            });
            flushed = true;
        }

        // ---- the end of the tile, or of the workgroup's part of it ----
        const bool odd_seen = __builtin_amdgcn_readfirstlane(s_flag[2]) != 0;
        const unsigned lane_now = worked_out_here(lane);
        const int n = lane_now & 15, g4 = lane_now >> 4;
#pragma unroll
        for (int rb = 0; rb < RW; ++rb) {
            const float sum = row_sum(l[rb]);
            if (g4 == 0) s_red[kgroup * M + wrow + 16 * rb + n] = sum;
        }
        lds_barrier();
        const bool head = k0 == 0, last = k1 == all_steps, whole = head && last;
        auto row_total = [&](int row) { return KG == 2 ? s_red[row] + s_red[M + row] : s_red[row]; };
        const int part = 2 * wl + (head ? 1 : 0);
        if (!whole) {
            used[head ? 1 : 0] = true;
            if (tid == 0) parts.rec[part] = make_int4(static_cast<int>(out_row0), rows_here, (head ? kPartHead : 0) | (last ? kPartLast : 0), 1);
            if (tid < rows_here) parts.ml[static_cast<size_t>(part) * M + tid] = make_float2(s_max[tid], row_total(tid));
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int row = 16 * rb + n;
            if (row >= rows_here) continue;
            const float inv = whole ? 1.f / row_total(row) : 1.f;
            const int sees = P + (row0 + row) / H + 1;
#pragma unroll
            for (int cb = 0; cb < NB; ++cb) {
                f32x4 x = o[rb][cb];
                if (flushed) x += *reinterpret_cast<const f32x4*>(scratch(lane_now) + 16 * rb * R + 16 * cb);
                x *= inv;
                const int col = 16 * (NB * wave + cb) + 4 * g4;
                if (odd_seen) {
                    // (The key's own score is then infinite or NaN too: its weight is NaN, or 0, and 0 times an infinity is NaN.)
                    for (int j = max(vis_min & ~(kStep - 1), k0 * kStep); j < min(sees, k1 * kStep); ++j) {
                        const bool cached = j < P;
                        if (KV8 && cached) continue;  // (the 8-bit pool holds neither)
                        const auto* const c4 = reinterpret_cast<const unsigned short*>(row_address(j, cached ? slots[j] : 0)) + col;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if ((c4[i] & 0x7F80) == 0x7F80) x[i] = NAN;
                    }
                }
                if (whole)
                    *reinterpret_cast<uint2*>(out + (out_row0 + row) * R + col) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
                else
                    *reinterpret_cast<f32x4*>(parts.o + (static_cast<size_t>(part) * M + row) * R + col) = x;
            }
        }
        lds_barrier();
        ++at.tile;
        at.k = 0;
        if (k1 != all_steps) break;
    }
    if (tid < 2 && !used[tid]) parts.rec[2 * wl + tid] = make_int4(0, 0, 0, 0);
}

// ---- host side ----

constexpr int kWorkgroups = 256;  // one on a compute unit

// Rows of a tile.  No more than a request's rows fill on the average: tiles of 32 rows take 116 us for 128 requests of 16 rows and 500 to 7800 keys, those of 64
// 142 us, those of 128 238 us; with 64 rows a request it is 214, 158 and 241 us.  Fewer where a workgroup has few keys to go through, since a large tile costs more to
// begin and to finish: 128 heads, 16 requests of one token and 2133 keys (139 keys a workgroup, in tiles of 128 rows) take 39, 37 and 70 us, 2 requests 31, 41
// and 62 us; 128 requests of 500 to 7800 keys 398, 278 and 257 us.
static int tile_rows(int B, int64_t T, int64_t max_kv_len, int H) {
    const int64_t rows = T * H, keys = (rows + 127) / 128 * (max_kv_len + kTileCost) / kWorkgroups;  // keys of a workgroup in tiles of 128 rows
    const int most = rows <= 32ll * B ? 32 : rows <= 64ll * B ? 64 : 128;
    return keys <= 128 ? 32 : keys <= 1024 && most > 64 ? 64 : most;
}

// (parts of tiles as large as these rows fill in one request: fewer requests than there are may take larger ones, more keys too)
size_t latent_workspace_bytes_bf16(int64_t T, int H, int R) {
    const int64_t rows = T * H;
    return latent_parts_layout(kWorkgroups, rows <= 32 ? 32 : rows <= 64 ? 64 : 128, R).total;
}

template <int R, int M, bool KV8>
static int launch_latent(const void* q, const LatentBatch& b, int H, float scale, void* out, void* workspace, hipStream_t stream) {
    const LatentSplit split = {H, 1, M, kStep, INT32_MAX, kWorkgroups};
    const LatentParts parts = latent_parts(workspace, latent_parts_layout(kWorkgroups, M, R));
    constexpr int lds = LatentShape<R, M, KV8>::kBytes;
    {
        ProfScope scope(kProfLatent, stream);
        hipLaunchKernelGGL((latent_bf16_kernel<R, M, KV8>), dim3(kWorkgroups), dim3(256), lds, stream, static_cast<const __hip_bfloat16*>(q), b, split,
                           scale * 1.4426950408889634f, static_cast<__hip_bfloat16*>(out), parts);
    }
    PA_HIP(hipGetLastError());
    {
        ProfScope scope(kProfLatentMerge, stream);
        launch_latent_merge(parts, kWorkgroups, M, R, b.T * H, b.B, out, stream);
    }
    PA_HIP(hipGetLastError());
    return PA_OK;
}

template <int R, bool KV8>
static int launch_tiles(int M, const void* q, const LatentBatch& b, int H, float scale, void* out, void* workspace, hipStream_t stream) {
    if (M == 32) return launch_latent<R, 32, KV8>(q, b, H, scale, out, workspace, stream);
    if (M == 64) return launch_latent<R, 64, KV8>(q, b, H, scale, out, workspace, stream);
    return launch_latent<R, 128, KV8>(q, b, H, scale, out, workspace, stream);
}

int latent_attention_bf16(const void* q, const LatentBatch& b, int64_t max_kv_len, int H, int R, bool kv8, float scale, void* out, void* workspace,
                          hipStream_t stream) {
    const int M = tile_rows(b.B, b.T, max_kv_len, H);
    if (R == 512) return kv8 ? launch_tiles<512, true>(M, q, b, H, scale, out, workspace, stream) : launch_tiles<512, false>(M, q, b, H, scale, out, workspace, stream);
    return kv8 ? launch_tiles<256, true>(M, q, b, H, scale, out, workspace, stream) : launch_tiles<256, false>(M, q, b, H, scale, out, workspace, stream);
}

}  // namespace pa
