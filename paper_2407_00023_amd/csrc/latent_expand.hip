// Latent attention, expanded form, bf16 tensors: keys and values of every head from the latent rows, once per distinct row, then attention over them.
//
// A row of q meets N + kRope values of a key and N of a value in place of R + kRope and R, 3.4 times less arithmetic at R = 512, N = 128; the expansion
// costs 4 N R operations per row and head, as much as 171 rows of q save.  So it is done once for each row the batch sees, however many
// requests share it:
//   mark     every slot of the lists takes a number, the first time it is met (a word per slot of the pool, cleared before)
//   collect  the rows with numbers, decoded, and the extend rows before them, behind one another: A [rows, R], A_r [rows, kRope]; the lists become row numbers
//   expand   K [head, row, N] = A W_k^T, V likewise, on the matrix cores; fp16 out of fp32 sums
//   attend   softmax(Q K^T + Q_r A_r^T) V
// Expanded keys and values lie in the workspace for as many heads at a time as fit kExpandedBytes.
//
// Measured: 24 requests of 200 to 1000 new tokens over 4 documents, 32 heads, R = 512, N = 128 (21 400 rows; 0.9 TFLOP): mark and collect 25 us, expand 200 us,
// attend 1000 us, join 30 us.  The expansion writes 350 MB and multiplies 180 GFLOP (0.9 PFLOP/s): bound by its stores beside the matrix cores, which are busy
// 50 % of the cycles.  In the attention these are busy 38 % of the cycles and LDS 22 %; a wave waits 29 % of its own, and 5.7 GB come past the L2s, 16 times the
// keys and values that there are, since a tile of 128 rows of q reads all of its head's.  (Waves of 64 rows, one to a SIMD, halve the LDS reads and take longer,
// 1320 us, since nothing is beside a wave that waits.)  The branch `scaled` (below) takes a quarter to a third longer: 1360 us.
//
// fp16 and not bf16, because a rounding of keys, one of values and one of probabilities would each cost as much as the result's own: with 11
// bits they are an eighth of it each.  What fp16 lacks in range is made up for: a row of K or V of a head whose largest value is out of
// [2^-8, 2^15) is stored times a power of two of its own, and the attention of that head puts it back (the branch `scaled`): what other rows hold, of
// other requests or of none, and where a row lies, decide nothing about it.  A row of q is brought to a common size by a power of two, which goes into the
// factor of its scores.
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

#include <type_traits>

#include "fp8_rows.h"
#include "latent_merge.h"
#include "latent_work.h"
#include "wave_ops.h"

namespace pa {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
using Global = __attribute__((address_space(1))) T;  // (an address that was a number is of no known memory otherwise)

// max(m, |a|, |b|) in one instruction, NaN aside.  The operands are results of matrix instructions that are done (products_done).
__device__ __forceinline__ void larger_of(float& m, float a, float b) { asm volatile("v_max3_f32 %0, |%1|, |%2|, %0" : "+v"(m) : "v"(a), "v"(b)); }
__device__ __forceinline__ void products_done() { asm volatile("s_nop 15\n\ts_nop 3" ::: "memory"); }

constexpr size_t kExpandedBytes = size_t{4} << 30;
constexpr int kExpandWorkgroups = 256;  // one on a compute unit
constexpr int kExpWorkgroups = 512;     // two
constexpr int kExpM = 128;           // rows of q of a tile
constexpr int kExpStep = 32;         // keys of a step
constexpr int kExpLow = -8;          // a row of K or V is stored as it is if its largest value is in [2^kExpLow, 2^15)
constexpr int kBlockRows = 64;       // rows of K or V that a wave of the expansion makes at a time

__device__ __forceinline__ unsigned pack_f16x2(float a, float b) {
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2_t{a, b}), f16x2));
}
__device__ __forceinline__ float power_of_two(int k) { return __int_as_float((k + 127) << 23); }  // k in [-126, 127]

struct ExpandArgs {
    int32_t *hdr;      // [3], [6]: see LatentParts; [8]: distinct cached rows
    int32_t *scaled;   // [H] some row of K or V of this head is stored times a power of two
    int32_t *map;      // [num_slots]
    int32_t *list;     // [cached_cap]
    int32_t *row_of;   // [B][max_keys] rows of A of a request's keys, cached and new
    uint4 *a, *rope;   // latent parts [rows_cap / 16][R / 32][64 lanes], as fragments (see collect); rotary parts [rows_cap][8]
    signed char *k_exp, *v_exp;  // [heads at once][rows_cap] a row is what is stored times 2^this
    unsigned short *k, *v;       // [heads at once][rows_cap][N] fp16
    int64_t cached_cap, rows_cap;
    int max_keys;
};

__global__ __launch_bounds__(256) void latent_clear_kernel(ExpandArgs x, int64_t num_slots, int H) {
    const int64_t i0 = blockIdx.x * 256ll + threadIdx.x;
    for (int64_t i = i0; i < num_slots; i += gridDim.x * 256ll) x.map[i] = -1;
    for (int64_t i = i0; i < H; i += gridDim.x * 256ll) x.scaled[i] = 0;
    if (i0 == 0) x.hdr[8] = 0;
}

// A lane per key of a list.  Which number a slot gets depends on the order of atomics; a row's keys and values do not, wherever they lie.
__global__ __launch_bounds__(256) void latent_mark_kernel(LatentBatch b, ExpandArgs x, int chunks) {
    const int64_t pieces = static_cast<int64_t>(b.B) * chunks;
    for (int64_t piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
        const int r = static_cast<int>(piece / chunks), j = static_cast<int>(piece - static_cast<int64_t>(r) * chunks) * 256 + threadIdx.x;
        const int P = min(b.prefix_len[r], x.max_keys);
        bool first = false;
        int slot = 0;
        if (j < P && b.ext_len[r] > 0) {
            slot = static_cast<int>(min(static_cast<int64_t>(max(b.slot_idx[b.slot_offsets[r] + j], 0)), b.num_slots - 1));  // never outside the pool
            first = x.map[slot] == -1 && atomicCAS(&x.map[slot], -1, -2) == -1;
        }
        const unsigned long long all = __ballot(first);
        if (all == 0) continue;
        const int lane = threadIdx.x & 63, leader = __builtin_ctzll(all);
        int at = 0;
        if (lane == leader) at = atomicAdd(&x.hdr[8], __popcll(all));
        at = __shfl(at, leader) + __popcll(all & ((1ull << lane) - 1));
        if (first && at < x.cached_cap) {
            x.list[at] = slot;
            x.map[slot] = static_cast<int>(b.T) + at;
        }
    }
}

// Waves take 16 rows of A at a time and, when these are done, 64 keys of a request.
// A lies in memory as the fragments that the matrix cores take: of 16 rows and 32 columns, 16 bytes (row lane % 16, columns 8 (lane / 16) on) of every lane
// behind one another, so that the expansion reads 1 KB of consecutive memory an instruction, straight into registers.
template <int R, bool KV8>
__global__ __launch_bounds__(256) void latent_collect_kernel(LatentBatch b, ExpandArgs x) {
    constexpr int L = R + kRope, PROW = KV8 ? R + 2 * kRope : 2 * L;
    const int lane = threadIdx.x & 63, n = lane & 15, g4 = lane >> 4, waves = gridDim.x * 4, wave = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t rows = b.T + min(static_cast<int64_t>(x.hdr[8]), x.cached_cap);
    const unsigned char* const pool = static_cast<const unsigned char*>(b.pool);
    for (int64_t block = wave; block < (rows + 15) / 16; block += waves) {
        const int64_t row = min(16 * block + n, rows - 1);  // (rows behind the last repeat it)
        uint4* const to = x.a + block * (2 * R) + lane;
        const uint4* rope;
        if (row < b.T || !KV8) {
            const uint4* const from = row < b.T ? reinterpret_cast<const uint4*>(static_cast<const __hip_bfloat16*>(b.c_ext) + row * L)
                                                : reinterpret_cast<const uint4*>(pool + static_cast<int64_t>(x.list[row - b.T]) * PROW);
#pragma unroll 8
            for (int s = 0; s < R / 32; ++s) to[64 * s] = from[4 * s + g4];
            rope = from + R / 8;
        } else {
            const int64_t slot = x.list[row - b.T];
            const uint2* const from = reinterpret_cast<const uint2*>(pool + slot * PROW);
            const float two_k = fp8_scale(reinterpret_cast<const signed char*>(pool + b.num_slots * PROW)[slot]);
#pragma unroll 8
            for (int s = 0; s < R / 32; ++s) {
                const uint2 codes = from[4 * s + g4];
                const uint2 p = fp8_decode4(codes.x, two_k), q = fp8_decode4(codes.y, two_k);
                to[64 * s] = make_uint4(p.x, p.y, q.x, q.y);
            }
            rope = reinterpret_cast<const uint4*>(from + R / 8);
        }
        if (16 * block + n < rows) {
            x.rope[row * 8 + g4] = rope[g4];
            x.rope[row * 8 + 4 + g4] = rope[4 + g4];
        }
    }
    const int chunks = (x.max_keys + 63) / 64;
    for (int64_t i = wave; i < static_cast<int64_t>(b.B) * chunks; i += waves) {
        const int r = static_cast<int>(i / chunks), j = static_cast<int>(i - static_cast<int64_t>(r) * chunks) * 64 + lane;
        const int P = min(max(b.prefix_len[r], 0), x.max_keys), E = b.ext_len[r];
        if (E <= 0 || j >= x.max_keys || j - P >= E) continue;
        int number = b.ext_offsets[r] + (j - P);
        if (j < P) {
            const int64_t slot = min(static_cast<int64_t>(max(b.slot_idx[b.slot_offsets[r] + j], 0)), b.num_slots - 1);
            number = x.map[slot];
        }
        x.row_of[static_cast<int64_t>(r) * x.max_keys + j] = number;
    }
}

// K and V of the heads h0 .. h0 + heads - 1, as one product of A with sets of 128 of a head's 2 N columns (its keys', then its values').  A wave multiplies
// 64 rows with the 128 columns: those of W stay in LDS, 128 KB at R = 512, where a fragment is read for four products; A's fragments
// come straight from memory.  An XCD has an eighth of the rows, so that they stay in its L2, and its 32 workgroups equal shares of the (set, 64 rows)
// there, set by set; the eight waves of a workgroup go through a set's part of the share one beside the other,
// without waiting for each other, so that of the two on a SIMD one multiplies while the other packs and stores.
template <int R, int N>
__global__ __launch_bounds__(512, 1) void latent_expand_kernel(ExpandArgs x, const __hip_bfloat16* __restrict__ w_k, const __hip_bfloat16* __restrict__ w_v,
                                                               int64_t T, int h0, int heads) {
    constexpr int KS = R / 32, kSets = 2 * N / 128;  // slices of 32 values; sets of 128 columns per head
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    auto* const lds = (__attribute__((address_space(3))) unsigned char*)smem;
    const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(smem));
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g4 = lane >> 4;
    const int64_t rows = T + min(static_cast<int64_t>(x.hdr[8]), x.cached_cap);
    const int blocks = static_cast<int>((rows + 63) / 64), last16 = static_cast<int>((rows + 15) / 16) - 1;
    // (workgroups go to the XCDs in turn)
    constexpr int kXcds = 8, kPerXcd = kExpandWorkgroups / kXcds;
    const int xcd = blockIdx.x % kXcds, mine = blockIdx.x / kXcds;
    const int first = static_cast<int>(static_cast<int64_t>(blocks) * xcd / kXcds), here = static_cast<int>(static_cast<int64_t>(blocks) * (xcd + 1) / kXcds) - first;
    const int64_t units = static_cast<int64_t>(here) * heads * kSets;
    int64_t unit = units * mine / kPerXcd;
    const int64_t end = units * (mine + 1) / kPerXcd;
    // A block's fragments are asked for kAhead slices ahead, the first of the next block's beside the last products of this one's.
    constexpr int kAhead = 2;
    uint64_t from[4];
    auto point_at = [&](int block) {
#pragma unroll
        for (int r = 0; r < 4; ++r)  // (see collect)
            from[r] = reinterpret_cast<uint64_t>(x.a) + static_cast<uint64_t>(static_cast<unsigned>(__builtin_amdgcn_readfirstlane(min(4 * block + r, last16)))) * (32 * R);
    };
    u32x4 af[kAhead][4];
    auto fetch = [&](int s) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            af[s % kAhead][r] = *reinterpret_cast<Global<const u32x4>*>(reinterpret_cast<Global<const unsigned char>*>(from[r] + 1024 * s) + 16u * static_cast<unsigned>(lane));
    };
    // Fragments 2 p and 2 p + 1 of W have the columns 32 p + 8 (n / 4) + n % 4, and 4 more, so that a lane's sums of both are 8 columns behind one another, and
    // are stored in 16 bytes.  The pieces of 16 bytes of a column are XORed by n.
    unsigned w_at[4];  // LDS address of a fragment, by its slice mod 4
#pragma unroll
    for (int s = 0; s < 4; ++s) w_at[s] = (8 * (n >> 2) + (n & 3)) * 2 * R + 16 * ((4 * s + g4) ^ n);
    while (unit < end) {
        const int set = static_cast<int>(unit / here), h = set / kSets;
        const int from_block = static_cast<int>(unit - static_cast<int64_t>(set) * here), blocks_here = static_cast<int>(min(end - unit, static_cast<int64_t>(here - from_block)));
        unit += blocks_here;
        lds_barrier();  // (nobody reads the old columns any more)
        constexpr int kRowsPerLoad = 512 / R;
        for (int i = wave; i < 128 / kRowsPerLoad; i += 8) {
            const int row = i * kRowsPerLoad + lane / (64 / kRowsPerLoad);
            const int col = (set % kSets) * 128 + row;  // among the head's 2 N
            const __hip_bfloat16* const w = (col < N ? w_k : w_v) + (static_cast<int64_t>(h0 + h) * N + (col < N ? col : col - N)) * R;
            load_to_lds_16(w + 8 * ((lane & (64 / kRowsPerLoad - 1)) ^ ((row & 3) | (row >> 1 & 12))), lds0 + i * 1024);
        }
        int at = wave;
        if (at < blocks_here) {
            point_at(first + from_block + at);
#pragma unroll
            for (int s = 0; s < kAhead; ++s) fetch(s);
        }
        wait_vm_all();
        lds_barrier();
        for (; at < blocks_here; at += 8) {
            const int64_t row0 = 64ll * (first + from_block + at);
            f32x4 acc[8][4];
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[c][r] = f32x4{0.f, 0.f, 0.f, 0.f};
            constexpr int kWAhead = 3;
            u32x4 wf[kWAhead + 1];
            auto read = [&](int f) __attribute__((always_inline)) {
                const int s = f >> 3, c = f & 7;
                wf[f % (kWAhead + 1)] = *reinterpret_cast<__attribute__((address_space(3))) const u32x4*>(lds + w_at[s & 3] + (32 * (c >> 1) + 4 * (c & 1)) * 2 * R + (s >> 2) * 256);
            };
#pragma unroll
            for (int f = 0; f < kWAhead; ++f) read(f);
            in_this_order();
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                if (s + kAhead == KS) point_at(first + from_block + (at + 8 < blocks_here ? at + 8 : at));
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    if (s * 8 + c + kWAhead < KS * 8) read(s * 8 + c + kWAhead);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        acc[c][r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wf[(s * 8 + c) % (kWAhead + 1)]), __builtin_bit_cast(bf16x8, af[s % kAhead][r]), acc[c][r], 0, 0, 0);
                    if (c == 7) fetch((s + kAhead) % KS);
                    in_this_order();
                }
            }
            products_done();
            in_this_order();
            // lane: row 16 r + n, columns 32 p + 8 g4 .. + 7 in c = 2 p, 2 p + 1
            constexpr int CK = N / 16;  // column blocks of one of the head's two matrices
#pragma unroll
            for (int part = 0; part < 8 / CK; ++part) {
                const bool is_v = (set % kSets) * 128 + part * N >= N;
                // The exponents of the rows 16 r + n, a byte for every r.  A row whose largest value is out of [2^kExpLow, 2^15) is brought to the edge of that
                // range, no further: a product of one stored as it is and one that is not then differ by as little as can be.  (0 otherwise, and for zeros.)
                unsigned e = 0;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float top = 0.f;
#pragma unroll
                    for (int c = part * CK; c < (part + 1) * CK; ++c)
#pragma unroll
                        for (int i = 0; i < 4; i += 2) larger_of(top, acc[c][r][i], acc[c][r][i + 1]);
                    in_this_order();
                    if (__any(top == INFINITY)) [[unlikely]] {  // (of the finite ones)
                        asm volatile("");  // (a branch, so that nobody else works it out)
                        top = 0.f;
#pragma unroll
                        for (int c = part * CK; c < (part + 1) * CK; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (fabsf(acc[c][r][i]) < INFINITY) top = fmaxf(top, fabsf(acc[c][r][i]));
                    }
                    top = row_max(top);
                    const int log2_top = static_cast<int>(__float_as_uint(top) >> 23) - 127;
                    if (top != 0.f) e |= static_cast<unsigned>(max(log2_top - 14, min(log2_top - kExpLow, 0)) & 255) << (8 * r);
                }
                const unsigned lane_now = worked_out_here(lane);
                (is_v ? x.v_exp : x.k_exp)[h * x.rows_cap + row0 + lane_now] = static_cast<signed char>(e >> (8 * (lane_now >> 4)));
                const bool any_scaled = __any(e != 0);
                if (any_scaled && lane == 0) x.scaled[h0 + h] = 1;
                unsigned char* const to = reinterpret_cast<unsigned char*>((is_v ? x.v : x.k) + (h * x.rows_cap + row0) * N);
                const int rows_here = static_cast<int>(min(rows - row0, static_cast<int64_t>(64)));
                const unsigned row = lane_now & 15, lane_at = row * (2 * N) + 16 * (lane_now >> 4);
                // (two copies, so that the sums are read where they are in both)
                auto store = [&](auto times) __attribute__((always_inline)) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * r + static_cast<int>(row) < rows_here)
#pragma unroll
                            for (int c = part * CK; c < (part + 1) * CK; c += 2) {
                                const float by = power_of_two(-static_cast<int>(static_cast<signed char>(e >> (8 * r))));
                                const f32x4 y = decltype(times)::value ? acc[c][r] * by : acc[c][r], z = decltype(times)::value ? acc[c + 1][r] * by : acc[c + 1][r];
                                *reinterpret_cast<uint4*>(to + r * (16 * 2 * N) + (c - part * CK) * 32 + lane_at) =
                                    make_uint4(pack_f16x2(y[0], y[1]), pack_f16x2(y[2], y[3]), pack_f16x2(z[0], z[1]), pack_f16x2(z[2], z[3]));
                            }
                };
                if (any_scaled) store(std::true_type{});
                else store(std::false_type{});
            }
        }
    }
}

// XOR of the 16-byte piece of a row in LDS: K is read 16 bytes per lane down 16 rows, V 8 bytes per lane across 32 bytes of 8 rows (by half a wave)
template <int N>
__device__ __forceinline__ int swz_k(int row) { return N == 128 ? row & 15 : (row >> 1) & 7; }
template <int N>
__device__ __forceinline__ int swz_v(int row) {
    return N == 128 ? ((row & 3) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1) : (((row >> 1) & 3) << 1) | ((row >> 3) & 1);
}

// Attention of the heads h0 .. h0 + heads - 1.  A tile is 128 new tokens of a request and one head; a wave has 32 of them and all keys, with running
// maxima of its own, and exchanges nothing with the others.  Two workgroups on a compute unit, so that the exponentials of one
// wave of a SIMD pass beside the matrix instructions of the other.
// Scores are computed transposed, as S^T = K Q^T: what a lane has of them is what it needs of P^T as an operand of O^T = V^T P^T, if the keys
// are taken in the order 4 g .. 4 g + 3, 16 + 4 g .. 16 + 4 g + 3 by the lanes 16 g .. 16 g + 15; V^T comes by the transposing LDS read.
// In the loop the scores of step i + 1 and the output of step i are computed, the probabilities of step i in between; keys of step i + 3 and values of
// step i + 2 are on their way to LDS, each in a ring of three.  A row's maximum moves when a lane's probabilities of a step sum to more than kExpMost: the wave leaves
// the loop, what it has summed up goes to memory, multiplied accordingly, and the accumulators begin anew (inside the loop the compiler
// would keep a second copy of them).  A maximum so large that its rounding shows (moved_maximum()) does not help the step it was taken from: if a step makes the
// wave leave the loop a second time, its probabilities are worked out there, held to 2^kExpCap, and the loop goes on whatever they sum to.
// A settled maximum stands for a probability of 2^kExpBits: fp16 holds what is as far below it as 2^-22 in 11 bits then, and what is lost is
// 2^-33 of it.  (With 1 for the maximum these are 2^-14 and 2^-25: many keys of little weight each, behind one that has nearly all of it and a small value, lost
// a fortieth at 2^-22.6, a fifth at 2^-26.)
constexpr float kExpBits = 8.f;
constexpr float kExpMost = 32768.f;  // 2^15 is the last power of two that fp16 holds
constexpr unsigned short kHalfMost = 0x7800, kHalfInfinity = 0x7C00;  // kExpMost and infinity in fp16
constexpr float kExpCap = 12.f;      // log2 of what probabilities are held to then: eight of them are kExpMost
constexpr int kExpSlots = 3;

template <int N>
struct ExpShape {
    static constexpr int kRow = 2 * N, kK = kExpStep * kRow, kR = kExpStep * 2 * kRope;
    static constexpr int kKExp = 2 * kK + kR, kVExp = kKExp + 4 * kExpStep, kSlot = kVExp + 4 * kExpStep;  // (exponents: a word per row)
    static constexpr int kRowsAt = kExpSlots * kSlot, kOddAt = kRowsAt + 4 * 2 * 256, kBytes = kOddAt + 16;
};

template <int N>
__global__ __launch_bounds__(256, 2) void latent_expanded_kernel(const __hip_bfloat16* __restrict__ q_ext, LatentBatch b, LatentSplit split, ExpandArgs x, int H,
                                                                 int h0, float scale_log2e, __hip_bfloat16* __restrict__ out, LatentParts parts) {
    using X = ExpShape<N>;
    constexpr int QW = N + kRope, KS = N / 32, KSR = kRope / 32, RB = 2, NB = N / 16;
    constexpr int RPL = 1024 / X::kRow, kRowLoads = 8 / RPL;    // K or V rows of a 1 KB load; loads of a wave's 8 rows
    constexpr int kLoads = 2 * kRowLoads + 1;
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
    const int wrow = 32 * wave;
    int* const s_odd = reinterpret_cast<int*>(smem + X::kOddAt);

    // LDS read addresses within a slot
    unsigned k_at[KS], r_at[KSR];
#pragma unroll
    for (int s = 0; s < KS; ++s) k_at[s] = n * X::kRow + 16 * ((4 * s + g4) ^ swz_k<N>(n));
#pragma unroll
    for (int s = 0; s < KSR; ++s) r_at[s] = 2 * X::kK + n * 2 * kRope + 16 * ((4 * s + g4) ^ ((n >> 1) & 7));
    unsigned v_at;  // and 32 cb more, by XOR; the second half of the keys 16 rows on (whose XOR is the same)
    {
        const int row = 4 * g4 + (n >> 2);
        v_at = X::kK + row * X::kRow + 16 * (((n & 3) >> 1) ^ swz_v<N>(row)) + 8 * (n & 1);
    }
    // the pieces of rows that a lane loads: rows RPL i + lane / (64 / RPL) of the wave's 8, i = 0, 1 (the XOR of i is put to these)
    const int load_row = lane / (64 / RPL), load_piece = lane & (64 / RPL - 1);
    const unsigned k_piece = 16 * (load_piece ^ swz_k<N>((8 * wave + load_row) & 15)), v_piece = 16 * (load_piece ^ swz_v<N>((8 * wave + load_row) & 15));
    const unsigned r_piece = 16 * ((lane & 7) ^ ((((8 * wave + (lane >> 3)) & 15) >> 1) & 7));

    bool used[2] = {false, false};
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
        const int per = req.tiles / split.copies, copy = at.tile / per, tile = at.tile - copy * per;
        const int P = req.P, row0 = tile * kExpM, rows_here = min(kExpM, req.rows - row0), h = h0 + copy;
        const int e0 = __builtin_amdgcn_readfirstlane(b.ext_offsets[at.r]);
        const int32_t* const row_of = x.row_of + static_cast<int64_t>(at.r) * x.max_keys;
        const int key_end = P + row0 + rows_here, all_steps = (key_end + kExpStep - 1) / kExpStep;
        const int k0 = at.k, k1 = at.r == end.r && at.tile == end.tile ? end.k : all_steps, steps = k1 - k0;
        const int vis_min = P + row0 + min(wrow, rows_here - 1) + 1;  // every row of the wave sees the keys before this one
        const bool is_scaled = __builtin_amdgcn_readfirstlane(x.scaled[h]) != 0;
        const unsigned char* const k_rows = reinterpret_cast<const unsigned char*>(x.k + copy * x.rows_cap * N);
        const unsigned char* const v_rows = reinterpret_cast<const unsigned char*>(x.v + copy * x.rows_cap * N);

        // ---- loads of a step: the wave's rows 8 wave .. + 7 ----
        // row numbers of eight steps from step k0 + 8 blk on, lane: step lane / 8, row lane % 8 (keys behind the last repeat it)
        auto load_row_numbers = [&](int blk) {
            const int first = (k0 + 8 * blk) * kExpStep;
            if (first < key_end)
                load_to_lds_4(row_of + min(first + (lane >> 3) * kExpStep + 8 * wave + (lane & 7), key_end - 1), lds0 + X::kRowsAt + wave * 512 + (blk & 1) * 256);
        };
        // (offsets of 32 bits: the host has seen to it that they suffice)
        auto number = [&](int rel, int row) __attribute__((always_inline)) {
            return *reinterpret_cast<__attribute__((address_space(3))) const unsigned*>(lds + X::kRowsAt + wave * 512 + (rel & 15) * 32 + 4 * row);
        };
        // (with_exps: the rows' powers of two too, a load more)
        auto issue_exps = [&](const signed char* of, int rel, unsigned to) __attribute__((always_inline)) {
            if (lane < 8) load_to_lds_1(of + copy * x.rows_cap + number(rel, lane), lds0 + to + 32 * wave);
        };
        auto issue_k = [&](int rel, unsigned slot, auto with_exps) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kRowLoads; ++i)
                load_to_lds_16(k_rows, number(rel, i * RPL + load_row) * X::kRow | (k_piece ^ (64 * i)), lds0 + slot + 8 * wave * X::kRow + i * 1024);
            load_to_lds_16(x.rope, number(rel, lane >> 3) * (2 * kRope) + r_piece, lds0 + slot + 2 * X::kK + 8 * wave * 2 * kRope);
            if constexpr (decltype(with_exps)::value) issue_exps(x.k_exp, rel, slot + X::kKExp);
        };
        auto issue_v = [&](int rel, unsigned slot, auto with_exps) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kRowLoads; ++i)
                load_to_lds_16(v_rows, number(rel, i * RPL + load_row) * X::kRow | (v_piece ^ (32 * i)), lds0 + slot + X::kK + 8 * wave * X::kRow + i * 1024);
            if constexpr (decltype(with_exps)::value) issue_exps(x.v_exp, rel, slot + X::kVExp);
        };

        // Steps with keys that some row of the tile does not see, or behind the last: 0 times an infinity or NaN of such a key would be NaN.  The wave
        // that loaded a row of V takes such values out of it, and the end of the tile makes the column NaN for the rows that see them.
        auto clean = [&](int rel, unsigned slot) __attribute__((always_inline)) {
            if ((k0 + rel + 1) * kExpStep <= P + row0 + 1) return;
            const unsigned at_v = slot + X::kK + 8 * wave * X::kRow + 16 * lane;
#pragma unroll
            for (int i = 0; i < kRowLoads; ++i) {
                auto* const v = reinterpret_cast<__attribute__((address_space(3))) s16x8*>(lds + at_v + 1024 * i);
                s16x8 y = *v;
                bool odd = false;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if ((y[e] & 0x7C00) == 0x7C00) {
                        odd = true;
                        y[e] = 0;
                    }
                if (odd) {
                    *v = y;
                    *s_odd = 1;
                }
            }
        };

        // ---- the wave's rows of Q, times a power of two that brings the largest of a row to [2^8, 2^9) ----
        // (A head with keys of powers of their own: what meets them by itself, its power relative to the row's goes with theirs.  Small ones would be out of
        // fp16's range beside rotary values otherwise, and decide for large keys all the same.)
        load_row_numbers(0);
        f16x8 q[RB][KS];
        bf16x8 qr[RB][KSR];
        float c[RB];
        int q_exp[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int row = min(wrow + 16 * rb + n, rows_here - 1);  // (rows behind the last repeat it)
            const uint4* const src = reinterpret_cast<const uint4*>(q_ext + (static_cast<int64_t>(e0 + row0 + row) * H + h) * QW);
            uint4 raw[KS + KSR];
            unsigned top = 0, top_n = 0;
#pragma unroll
            for (int s = 0; s < KS + KSR; ++s) {
                if (s == KS) top_n = top;
                raw[s] = src[4 * s + g4];
                const unsigned w[4] = {raw[s].x, raw[s].y, raw[s].z, raw[s].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
            }
            auto exponent_of = [](unsigned t) {
                t = max(t, static_cast<unsigned>(__shfl_xor(static_cast<int>(t), 16)));
                t = max(t, static_cast<unsigned>(__shfl_xor(static_cast<int>(t), 32)));
                const int e = static_cast<int>(t >> 7);
                return e == 0 || e == 255 ? 0 : max(min(e - 127 - 8, 126), -126);
            };
            const int k = exponent_of(top), alone = min(exponent_of(top_n), k), k_n = is_scaled ? alone : k;
            const float by = power_of_two(-k), by_n = power_of_two(-k_n);
            q_exp[rb] = k_n - k;
            c[rb] = fmaxf(scale_log2e * power_of_two(k), 1.401298464324817e-45f);  // (never 0, which would make NaN of a hidden key's -infinity)
#pragma unroll
            for (int s = 0; s < KS + KSR; ++s) {
                const unsigned w[4] = {raw[s].x, raw[s].y, raw[s].z, raw[s].w};
                unsigned y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float times = s < KS ? by_n : by, lo = __uint_as_float(w[i] << 16) * times, hi = __uint_as_float(w[i] & 0xFFFF0000u) * times;
                    y[i] = s < KS ? pack_f16x2(lo, hi) : pack_bf16x2(lo, hi);
                }
                const uint4 z = make_uint4(y[0], y[1], y[2], y[3]);
                if (s < KS) q[rb][s] = __builtin_bit_cast(f16x8, z);
                else qr[rb][s - KS] = __builtin_bit_cast(bf16x8, z);
            }
        }
        wait_vm_all();
        load_row_numbers(1);
        if (tid == 0) *s_odd = 0;

        const bool head = k0 == 0, last = k1 == all_steps, whole = head && last;
        const int part = 2 * wl + (head ? 1 : 0);
        const int out_row0 = (e0 + row0) * H + h;
        // The tile, with keys and values as they are (the usual case) or with powers of two of their own, 2^a of a key and 2^b of a value.  A key's comes into its
        // score.  A value's goes with its probability, which is then measured against a maximum of its own: with z the score in log2 units against the
        // row's reference m, and d the running maximum of z + b, rounded to an integer, less kExpBits:   sum = sum 2^z,   O = sum 2^(z + b - d) V,   out = 2^d O / sum.  What
        // a product with V is worth beside the others decides so how many bits its probability has, however far apart the sizes are; with b = 0 throughout d
        // is 0, and every number is what it is without.
        auto walk = [&](auto scaled_c) __attribute__((always_inline)) {
            constexpr bool scaled = decltype(scaled_c)::value;
            constexpr int kVLoads = kRowLoads + scaled, kKVLoads = kLoads + 2 * scaled;
            issue_k(0, 0, scaled_c);
            issue_v(0, 0, scaled_c);
            if (steps > 1) issue_k(1, X::kSlot, scaled_c);
            if (steps > 1) issue_v(1, X::kSlot, scaled_c);
            if (steps > 2) issue_k(2, 2 * X::kSlot, scaled_c);
            if (steps > 2) wait_vm<kKVLoads>();
            else if (steps > 1) wait_vm<kVLoads>();
            else wait_vm_all();
            lds_barrier();
            clean(0, 0);
            lds_barrier();
            f32x4 sc[2][RB], next[2][RB];  // scores of this step and of the one behind it
            float m[RB], l[RB];
            float d[RB];                         // (scaled)
            bool fresh = true, flushed = false;  // fresh: no maxima yet
            unsigned slot = 0;  // of step rel
            // the exponents of the keys or values 16 kb + 4 g4 .. + 3 of a step
            auto exponents = [&](unsigned at, int kb) __attribute__((always_inline)) {
                return *reinterpret_cast<__attribute__((address_space(3))) const u32x4*>(lds + at + 64 * kb + 16 * g4);
            };
            auto exponent = [](unsigned word) { return static_cast<int>(static_cast<signed char>(word)); };
            // a score against the row's reference; moved: which has just moved
            auto score = [&](int kb, int rb, int i, auto moved) __attribute__((always_inline)) {
                const float z = fmaf(sc[kb][rb][i], c[rb], -m[rb]);
                return decltype(moved)::value && z > kExpCap ? kExpCap : z;
            };
            // a quarter of the probabilities of the scores of step rel, [rb][kb], and their sums
            f16x8 pr[RB];
            unsigned pw[RB][4];
            float sum[RB];
            auto probabilities = [&](int kb, int rb, auto moved) __attribute__((always_inline)) {
                float p[4];
                u32x4 b = {0, 0, 0, 0};
                if constexpr (scaled) b = exponents(slot + X::kVExp, kb);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float z = score(kb, rb, i, moved);
                    p[i] = __builtin_amdgcn_exp2f(z);
                    if constexpr (scaled) p[i] = __uint_as_float(worked_out_here(__float_as_uint(p[i])));  // (here: scores are not kept for it)
                    sum[rb] += p[i];
                    if constexpr (scaled) {
                        p[i] = __builtin_amdgcn_exp2f(z + (exponent(b[i]) - d[rb]));
                    }
                }
                pw[rb][2 * kb] = worked_out_here(pack_f16x2(p[0], p[1]));  // (here, and not where it is used)
                pw[rb][2 * kb + 1] = worked_out_here(pack_f16x2(p[2], p[3]));
            };
            // The scores of a step into `next`, and beside them the probabilities of the step before, whose scores are at hand: a piece of these behind every few products.
            // Fragments are read four ahead.
            constexpr int kFrags = 2 * (KS + KSR), kAhead = 4;
            auto scores = [&](int rel1, unsigned slot1, auto with) __attribute__((always_inline)) {
                constexpr bool probs = decltype(with)::value;
                if constexpr (probs) {
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) sum[rb] = 0.f;
                }
                const int j0 = (k0 + rel1) * kExpStep;
                u32x4 kf[kFrags];
                auto read = [&](int f) __attribute__((always_inline)) {
                    const int s = f >> 1, kb = f & 1;
                    kf[f] = *reinterpret_cast<__attribute__((address_space(3))) const u32x4*>(
                        lds + (s < KS ? k_at[s] + kb * 16 * X::kRow : r_at[s - KS] + kb * 16 * 2 * kRope) + slot1);
                };
#pragma unroll
                for (int f = 0; f < kAhead; ++f) read(f);
                in_this_order();
#pragma unroll
                for (int f = 0; f < kFrags; ++f) {
                    const int s = f >> 1, kb = f & 1;
                    if (scaled && f == 2 * KS) {
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const u32x4 a = exponents(slot1 + X::kKExp, y);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
#pragma unroll
                                for (int rb = 0; rb < RB; ++rb) next[y][rb][i] *= power_of_two(max(exponent(a[i]) + q_exp[rb], -126));
                        }
                    }
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        const f32x4 before = s == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : next[kb][rb];
                        if (s < KS) next[kb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, kf[f]), q[rb][s < KS ? s : 0], before, 0, 0, 0);
                        else next[kb][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[f]), qr[rb][s < KS ? 0 : s - KS], before, 0, 0, 0);
                    }
                    if (f + kAhead < kFrags) read(f + kAhead);
                    if constexpr (probs) {
                        constexpr int kEvery = kFrags / 4;
                        if (f % kEvery == 0 && f / kEvery < 4) probabilities((f / kEvery) & 1, (f / kEvery) >> 1, std::false_type{});
                    }
                    in_this_order();
                }
                if (j0 + kExpStep > vis_min) {
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        const int sees = P + row0 + min(wrow + 16 * rb + n, rows_here - 1) + 1 - j0 - 4 * g4;
#pragma unroll
                        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (16 * kb + i >= sees) next[kb][rb][i] = -INFINITY;
                    }
                }
            };
            auto largest = [&](int rb) __attribute__((always_inline)) {
                float mx = sc[0][rb][0];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[kb][rb][i]);
                return mx * c[rb];
            };
            auto largest_product = [&](int rb) __attribute__((always_inline)) {
                float mx = -INFINITY;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    const u32x4 b = exponents(slot + X::kVExp, kb);
#pragma unroll
                    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, score(kb, rb, i, std::true_type{}) + exponent(b[i]));
                }
                return mx;
            };
            auto take_next = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) sc[kb][rb] = next[kb][rb];
            };
            auto output = [&](unsigned slot, f32x4 (&o)[RB][NB]) __attribute__((always_inline)) {
                const unsigned v_here = worked_out_here(v_at);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) pr[rb] = __builtin_bit_cast(f16x8, u32x4{pw[rb][0], pw[rb][1], pw[rb][2], pw[rb][3]});
                s16x4 vf[NB][2];
                auto read = [&](int cb) __attribute__((always_inline)) {
                    const unsigned a = (v_here ^ (32 * cb)) + slot;
                    vf[cb][0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + a));
                    vf[cb][1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + a + 16 * X::kRow));
                };
#pragma unroll
                for (int cb = 0; cb < 3; ++cb) read(cb);
                in_this_order();
#pragma unroll
                for (int cb = 0; cb < NB; ++cb) {
                    const f16x8 v = __builtin_bit_cast(f16x8, __builtin_shufflevector(vf[cb][0], vf[cb][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) o[rb][cb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pr[rb], o[rb][cb], 0, 0, 0);
                    if (cb + 3 < NB) read(cb + 3);
                    in_this_order();
                }
            };
            // scratch memory of the wave, this lane's part: row 16 rb + n, columns 16 cb + 4 g4 .. + 3
            auto scratch = [&](unsigned lane_now) {
                return parts.o + (static_cast<size_t>(2 * split.n_wg + wl) * kExpM + wrow + (lane_now & 15)) * N + 4 * (lane_now >> 4);
            };

#pragma unroll
            for (int rb = 0; rb < RB; ++rb) m[rb] = l[rb] = d[rb] = 0.f;
            int rel = 0;
            f32x4 o[RB][NB];
            auto behind = [](unsigned x) { return x == 2 * X::kSlot ? 0u : x + X::kSlot; };
            scores(0, 0, std::false_type{});
            take_next();
            bool grown = true, ready = false;  // ready: the probabilities of step rel are worked out
            int settled = -1;                  // the last step whose scores moved a maximum
            while (true) {
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int cb = 0; cb < NB; ++cb) o[rb][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
                while (rel < steps && !grown) {
                    const unsigned slot1 = behind(slot), slot2 = behind(slot1);
                    // (behind the last step: of whatever lies there, not used)
                    if (ready) {
                        scores(rel + 1, slot1, std::false_type{});
                        ready = false;
                    } else {
                        scores(rel + 1, slot1, std::true_type{});
                        bool outgrown = false;
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb) outgrown |= sum[rb] > kExpMost;
                        if constexpr (scaled) {
                            // (what V is multiplied with, as it stands: a half between kExpMost and infinity; a sum of it would cost a register in the loop)
                            u16x2 least = {0xFFFF, 0xFFFF};
#pragma unroll
                            for (int i = 0; i < 4 * RB; ++i) least = __builtin_elementwise_min(least, __builtin_bit_cast(u16x2, pw[i / 4][i % 4]) - u16x2{kHalfMost, kHalfMost});
                            outgrown |= min(least[0], least[1]) <= kHalfInfinity - kHalfMost;
                        }
                        grown = __any(outgrown);
                        if (grown) break;
                    }
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) l[rb] += sum[rb];
                    if ((rel & 7) == 6) load_row_numbers((rel + 2) / 8 + 1);
                    if (rel + 2 < steps) issue_v(rel + 2, slot2, scaled_c);
                    if (rel + 3 < steps) issue_k(rel + 3, slot, scaled_c);
                    output(slot, o);
                    take_next();
                    if (rel + 3 < steps) wait_vm<kKVLoads>();
                    else if (rel + 2 < steps) wait_vm<kVLoads>();
                    else wait_vm_all();
                    if (rel + 1 < steps) clean(rel + 1, slot1);
                    lds_barrier();
                    slot = slot1;
                    ++rel;
                }
                if (rel >= steps) break;
                {
                    // new maxima, from the scores at hand; what has been summed up moves to memory, multiplied accordingly
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        const float mx = moved_maximum(row_max(largest(rb))) - kExpBits;
                        const float mn = fresh ? (mx == -INFINITY ? kNoMaximum : mx) : fmaxf(mx, m[rb]);
                        const float a = fresh ? 0.f : __builtin_amdgcn_exp2f(m[rb] - mn);
                        const float by = m[rb] - mn;
                        m[rb] = mn;
                        float a_v = a;  // for what V has been multiplied with
                        if constexpr (scaled) {
                            float dn = rintf(row_max(largest_product(rb))) - kExpBits;
                            if (!fresh) dn = fmaxf(dn, rintf(d[rb] + by));
                            if (dn == -INFINITY) dn = 0.f;
                            a_v = __builtin_amdgcn_exp2f(d[rb] - dn + by);
                            d[rb] = dn;
                        }
                        if (!fresh) {
                            float* const to = scratch(worked_out_here(lane)) + 16 * rb * N;
#pragma unroll
                            for (int cb = 0; cb < NB; ++cb) {
                                f32x4 y = o[rb][cb];
                                if (flushed) y += *reinterpret_cast<const f32x4*>(to + 16 * cb);
                                *reinterpret_cast<f32x4*>(to + 16 * cb) = y * a_v;
                            }
                        }
                        l[rb] *= a;
                    }
                    if (!fresh) flushed = true;
                    fresh = grown = false;
                    ready = rel == settled;
                    settled = rel;
                    if (ready) [[unlikely]] {
#pragma unroll
                        for (int rb = 0; rb < RB; ++rb) {
                            sum[rb] = 0.f;
#pragma unroll
                            for (int kb = 0; kb < 2; ++kb) probabilities(kb, rb, std::true_type{});
                        }
                    }
                }
            }

            // ---- the end of the tile, or of the workgroup's part of it ----
            const unsigned lane_now = worked_out_here(lane);
            const int n = lane_now & 15, g4 = lane_now >> 4;
            const bool odd_seen = __builtin_amdgcn_readfirstlane(*s_odd) != 0;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const float sum = row_sum(l[rb]);
                const int row = wrow + 16 * rb + n;
                if (row >= rows_here) continue;
                // (values so large that a part's sum of them could be more than fp32 holds: their mean instead, with the weight in the maximum)
                const bool mean = !whole && scaled && d[rb] > 64.f && sum > 0.f;
                if (!whole && g4 == 0) parts.ml[static_cast<size_t>(part) * kExpM + row] = mean ? make_float2(m[rb] + __builtin_amdgcn_logf(sum), 1.f) : make_float2(m[rb], sum);
                const float inv = whole || mean ? 1.f / sum : 1.f;
#pragma unroll
                for (int cb = 0; cb < NB; ++cb) {
                    f32x4 y = o[rb][cb];
                    if (flushed) y += *reinterpret_cast<const f32x4*>(scratch(lane_now) + 16 * rb * N + 16 * cb);
                    y *= inv;
                    if constexpr (scaled) y *= __builtin_amdgcn_exp2f(d[rb]);
                    const int col = 16 * cb + 4 * g4;
                    if (odd_seen) {
                        // (A latent value that is not finite makes the key so too, and its score: the weight is NaN, or 0, and 0 times an infinity is NaN.  The keys
                        // of the steps they were taken out of.)
                        for (int j = max((P + row0 + 1) & ~(kExpStep - 1), k0 * kExpStep); j < min(P + row0 + row + 1, k1 * kExpStep); ++j) {
                            const int64_t at_row = row_of[j];
                            const unsigned short* const v4 = reinterpret_cast<const unsigned short*>(v_rows) + at_row * N + col;
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if ((v4[i] & 0x7C00) == 0x7C00) y[i] = NAN;
                        }
                    }
                    if (whole)
                        *reinterpret_cast<uint2*>(out + (out_row0 + static_cast<int64_t>(row) * H) * N + col) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
                    else
                        *reinterpret_cast<f32x4*>(parts.o + (static_cast<size_t>(part) * kExpM + row) * N + col) = y;
                }
            }
        };
        if (is_scaled) walk(std::true_type{});
        else walk(std::false_type{});
        if (!whole) {
            used[head ? 1 : 0] = true;
            if (tid == 0) parts.rec[part] = make_int4(out_row0, rows_here, (head ? kPartHead : 0) | (last ? kPartLast : 0), H);
        }
        lds_barrier();  // (nobody looks at the flag any more)
        ++at.tile;
        at.k = 0;
        if (k1 != all_steps) break;
    }
    if (tid < 2 && !used[tid]) parts.rec[2 * wl + tid] = make_int4(0, 0, 0, 0);
}

// ---- host side ----

struct ExpandLayout {
    int heads;  // at once
    int64_t cached_cap, rows_cap;
    size_t scaled, map, list, row_of, a, rope, k_exp, v_exp, k, v, parts, total;
};
static ExpandLayout expand_layout(int B, int64_t T, int64_t max_kv_len, int H, int R, int N, int64_t num_slots) {
    ExpandLayout l;
    const int64_t listed = static_cast<int64_t>(B) * max_kv_len;
    l.cached_cap = listed < num_slots ? listed : num_slots;
    l.rows_cap = (T + l.cached_cap + kBlockRows - 1) / kBlockRows * kBlockRows;
    if (l.rows_cap == 0) l.rows_cap = kBlockRows;  // (an empty batch has a size too)
    const size_t head_bytes = static_cast<size_t>(l.rows_cap) * (N * 4 + 2);  // keys, values, exponents
    const int most = static_cast<int>(kExpandedBytes / head_bytes < 1 ? 1 : kExpandedBytes / head_bytes > static_cast<size_t>(H) ? H : kExpandedBytes / head_bytes);
    const int groups = (H + most - 1) / most;
    l.heads = (H + groups - 1) / groups;
    size_t at = 256;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) & ~size_t{255};
        return here;
    };
    l.scaled = take(sizeof(int32_t) * H);
    l.map = take(sizeof(int32_t) * num_slots);
    l.list = take(sizeof(int32_t) * (l.cached_cap + 1));
    l.row_of = take(sizeof(int32_t) * (listed + 1));
    l.a = take(static_cast<size_t>(l.rows_cap) * R * 2);
    l.rope = take(static_cast<size_t>(l.rows_cap) * kRope * 2);
    // Room for all heads, or kExpandedBytes of it, or one: it does not fall when a batch grows, as what the heads at once take does where it holds one less, so that
    // a workspace is enough for every smaller batch.
    const size_t all = head_bytes * H, room = all <= kExpandedBytes ? all : head_bytes > kExpandedBytes ? head_bytes : kExpandedBytes;
    const size_t exps = static_cast<size_t>(l.heads) * l.rows_cap, values = exps * N * 2;
    l.k = take(room);
    l.v = l.k + values;
    l.k_exp = l.v + values;
    l.v_exp = l.k_exp + exps;
    l.parts = take(latent_parts_layout(kExpWorkgroups, kExpM, N).total);
    l.total = at;
    return l;
}

// 0: too many rows for offsets of 32 bits
size_t latent_expanded_bytes(int B, int64_t T, int64_t max_kv_len, int H, int R, int N, int64_t num_slots) {
    const int64_t listed = static_cast<int64_t>(B) * (max_kv_len + 256);
    const int64_t rows = T + (listed < num_slots ? listed : num_slots);
    if (rows + kBlockRows > UINT32_MAX / (2 * (R + kRope)) || listed / 64 > INT32_MAX) return 0;
    return expand_layout(B, T, max_kv_len, H, R, N, num_slots).total;
}

template <int R, int N>
static int launch_group(const void* q, const LatentBatch& b, const ExpandArgs& x, const void* w_k, const void* w_v, int H, int h0, int heads, float scale,
                        void* out, void* parts_at, hipStream_t stream) {
    {
        ProfScope scope(kProfLatentExpand, stream);
        hipLaunchKernelGGL((latent_expand_kernel<R, N>), dim3(kExpandWorkgroups), dim3(512), 256 * R, stream, x, static_cast<const __hip_bfloat16*>(w_k),
                           static_cast<const __hip_bfloat16*>(w_v), b.T, h0, heads);
    }
    PA_HIP(hipGetLastError());
    const LatentSplit split = {1, heads, kExpM, kExpStep, x.max_keys, kExpWorkgroups};
    LatentParts parts = latent_parts(parts_at, latent_parts_layout(kExpWorkgroups, kExpM, N));
    parts.hdr = x.hdr;
    {
        ProfScope scope(kProfLatentExpanded, stream);
        hipLaunchKernelGGL((latent_expanded_kernel<N>), dim3(kExpWorkgroups), dim3(256), ExpShape<N>::kBytes, stream, static_cast<const __hip_bfloat16*>(q), b, split, x, H,
                           h0, scale * 1.4426950408889634f, static_cast<__hip_bfloat16*>(out), parts);
    }
    PA_HIP(hipGetLastError());
    {
        ProfScope scope(kProfLatentMerge, stream);
        launch_latent_merge(parts, kExpWorkgroups, kExpM, N, b.T * heads, static_cast<int64_t>(b.B) * heads, out, stream);
    }
    PA_HIP(hipGetLastError());
    return PA_OK;
}

int latent_expanded_bf16(const void* q, const LatentBatch& b, const void* w_k, const void* w_v, int64_t max_kv_len, int H, int R, int N, bool kv8, float scale,
                         void* out, void* workspace, hipStream_t stream) {
    const ExpandLayout l = expand_layout(b.B, b.T, max_kv_len, H, R, N, b.num_slots);
    unsigned char* const w = static_cast<unsigned char*>(workspace);
    auto i32 = [&](size_t at) { return reinterpret_cast<int32_t*>(w + at); };
    const ExpandArgs x = {i32(0), i32(l.scaled), i32(l.map), i32(l.list), i32(l.row_of), reinterpret_cast<uint4*>(w + l.a), reinterpret_cast<uint4*>(w + l.rope),
                          reinterpret_cast<signed char*>(w + l.k_exp), reinterpret_cast<signed char*>(w + l.v_exp), reinterpret_cast<unsigned short*>(w + l.k),
                          reinterpret_cast<unsigned short*>(w + l.v), l.cached_cap, l.rows_cap, static_cast<int>(max_kv_len)};
    {
        ProfScope scope(kProfLatentExpand, stream);
        const int64_t words = b.num_slots > H ? b.num_slots : H, clear = (words + 255) / 256;
        hipLaunchKernelGGL(latent_clear_kernel, dim3(static_cast<unsigned>(clear < 2048 ? clear : 2048)), dim3(256), 0, stream, x, b.num_slots, H);
        const int chunks = static_cast<int>((max_kv_len + 255) / 256);
        const int64_t pieces = static_cast<int64_t>(b.B) * chunks;
        if (pieces > 0) hipLaunchKernelGGL(latent_mark_kernel, dim3(static_cast<unsigned>(pieces < kMostGroups ? pieces : kMostGroups)), dim3(256), 0, stream, b, x, chunks);
        const dim3 grid(2048);
        if (R == 512 && kv8) hipLaunchKernelGGL((latent_collect_kernel<512, true>), grid, dim3(256), 0, stream, b, x);
        else if (R == 512) hipLaunchKernelGGL((latent_collect_kernel<512, false>), grid, dim3(256), 0, stream, b, x);
        else if (kv8) hipLaunchKernelGGL((latent_collect_kernel<256, true>), grid, dim3(256), 0, stream, b, x);
        else hipLaunchKernelGGL((latent_collect_kernel<256, false>), grid, dim3(256), 0, stream, b, x);
    }
    PA_HIP(hipGetLastError());
    for (int h0 = 0; h0 < H; h0 += l.heads) {
        const int heads = H - h0 < l.heads ? H - h0 : l.heads;
        int rc = PA_OK;
        if (R == 512) rc = N == 128 ? launch_group<512, 128>(q, b, x, w_k, w_v, H, h0, heads, scale, out, w + l.parts, stream) : launch_group<512, 64>(q, b, x, w_k, w_v, H, h0, heads, scale, out, w + l.parts, stream);
        else rc = N == 128 ? launch_group<256, 128>(q, b, x, w_k, w_v, H, h0, heads, scale, out, w + l.parts, stream) : launch_group<256, 64>(q, b, x, w_k, w_v, H, h0, heads, scale, out, w + l.parts, stream);
        if (rc != PA_OK) return rc;
    }
    return PA_OK;
}

}  // namespace pa
