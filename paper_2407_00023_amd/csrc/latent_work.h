// How the work of a bf16 latent attention launch is dealt out: no list is built, every workgroup finds its own share.
//
// The rows of q of a request, packed as i * H + h (expanded form: a head's rows by themselves, `copies` heads after one another), are cut
// into tiles of M rows, the tiles of all requests laid end to end on one axis, a tile as long as the keys it walks (and kTileCost
// more, what starting and finishing it takes).  Each of n workgroups takes an n-th of that axis, wherever its ends fall: all of them finish
// together whatever the lengths are, and none has to be sorted or counted on the host.  Where an end falls inside a tile, the tile's
// two sides leave partial results (row sums, row maxima, un-normalised rows) that a second kernel joins.  An end within kSnap steps of a tile's
// own end moves there.
//
// A tile's length is taken as a linear function of its number, keys + its last row's token, so that a place on the axis is found from
// sums in closed form (64-bit integers in units of 1 / (2 H) keys), in one pass over the requests' lengths by the whole workgroup: a round trip
// and two barriers for up to 256 requests.
#pragma once

#include "latent.h"

namespace pa {

constexpr int kTileCost = 96;    // in keys
constexpr int kSnap = 3;         // steps
constexpr int kMinShare = 128;   // keys, besides kTileCost, that a workgroup has at least

struct LatentPlace {  // step k of tile `tile` of request r
    int r, tile, k;
};

struct LatentRequest {
    int P, rows, tiles;  // cached keys; packed rows of a copy; tiles of all copies
};

struct LatentSplit {
    int rpt;       // rows per token of a copy
    int copies;
    int M;
    int step;      // keys of a step of the loop
    int max_keys;  // of a request
    int n_wg;
};

struct LatentScratch {  // of the workgroup, 256 threads
    int64_t chunk[257];
    int64_t wave[4];
    int64_t at[2];
    int r[2];
    int over;
};

// A request as the launch may use it: one that does not fit the host's T has no rows (and marks the batch as too large).
__device__ __forceinline__ LatentRequest latent_request(const LatentBatch& b, const LatentSplit& s, int r, bool* over) {
    LatentRequest q = {0, 0, 0};
    if (r < b.B) {
        const int E = b.ext_len[r], e0 = b.ext_offsets[r];
        q.P = min(max(b.prefix_len[r], 0), INT32_MAX / 2);
        if (E > 0) {
            if (e0 < 0 || E > b.T - e0 || q.P > s.max_keys - E) *over = true;
            else q.rows = E * s.rpt;
            q.tiles = (q.rows + s.M - 1) / s.M * s.copies;
        }
    }
    return q;
}
// the axis up to tile t of a copy
__device__ __forceinline__ int64_t latent_upto(const LatentSplit& s, int P, int64_t t) {
    return t * (2ll * s.rpt * (P + kTileCost) + s.M * (t + 1));
}
__device__ __forceinline__ int64_t latent_length(const LatentSplit& s, const LatentRequest& q) {
    return q.tiles ? s.copies * latent_upto(s, q.P, q.tiles / s.copies) : 0;
}
// keys that the last row of tile t (of a copy) sees, and the steps it takes
__device__ __forceinline__ int latent_keys(const LatentSplit& s, const LatentRequest& q, int t) {
    const int last = min((t + 1) * s.M, q.rows) - 1;
    return q.P + last / s.rpt + 1;
}
__device__ __forceinline__ int latent_steps(const LatentSplit& s, const LatentRequest& q, int t) { return (latent_keys(s, q, t) + s.step - 1) / s.step; }

__device__ __forceinline__ int64_t wave_scan_64(int64_t x) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int64_t y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    return x;
}
// inclusive scan over the workgroup; *total
__device__ __forceinline__ int64_t block_scan_64(int64_t x, LatentScratch* sh, int64_t* total) {
    const int wave = threadIdx.x >> 6;
    const int64_t in = wave_scan_64(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sh->wave[wave] = in;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) before += sh->wave[w];
        all += sh->wave[w];
    }
    *total = all;
    return in + before;
}

// The place of y on request q's part of the axis.
__device__ __forceinline__ LatentPlace latent_place(const LatentSplit& s, const LatentRequest& q, int r, int64_t y) {
    LatentPlace p = {r, 0, 0};
    const int per = q.tiles / s.copies;
    const int64_t one = latent_upto(s, q.P, per);
    int copy = 0;
    if (s.copies > 1) {
        copy = static_cast<int>(y / one);
        y -= copy * one;
    }
    int lo = 0, hi = per;  // the last tile that begins at or before y
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (latent_upto(s, q.P, mid) <= y) lo = mid; else hi = mid;
    }
    const int64_t begin = latent_upto(s, q.P, lo);
    const int steps = latent_steps(s, q, lo);
    int k = static_cast<int>(static_cast<double>(y - begin) * steps / static_cast<double>(latent_upto(s, q.P, lo + 1) - begin));
    if (k < kSnap) k = 0;
    p.tile = copy * per + lo;
    if (steps - k < kSnap && k > 0) {
        ++p.tile;
        k = 0;
    }
    p.k = k;
    return p;
}

// The share of workgroup wl of the launch, [*from, *to).  Wave-uniform; false: it has none.  Every thread of the workgroup calls it.
// *at_work: workgroups that have one.  *over: the batch on the device does not fit the host's sizes: nothing is computed.
__device__ __forceinline__ bool latent_share(const LatentBatch& b, const LatentSplit& s, int bid, LatentScratch* sh, int* wl_out, int* at_work, LatentPlace* from,
                                             LatentPlace* to, bool* over_out) {
    const int tid = threadIdx.x, chunks = (b.B + 255) / 256;
    if (tid == 0) sh->over = 0;
    __syncthreads();
    bool over = false;
    int64_t all = 0, incl = 0, mine = 0;
    for (int c = 0; c < chunks; ++c) {
        mine = latent_length(s, latent_request(b, s, c * 256 + tid, &over));
        int64_t total = 0;
        incl = block_scan_64(mine, sh, &total);
        if (tid == 0) sh->chunk[c] = all;
        all += total;
    }
    if (over) sh->over = 1;
    __syncthreads();
    *over_out = sh->over != 0;
    *at_work = 0;
    if (sh->over || all == 0) return false;
    // workgroups at work: eight at least as many on every XCD (blocks are dealt round-robin to them), neighbours on the axis on one XCD
    const int64_t least = 2ll * s.rpt * (kTileCost + kMinShare);
    const int n = static_cast<int>(min(static_cast<int64_t>(s.n_wg), max(all / least, int64_t{1})));
    const int per_xcd = (n + 7) / 8, wl = (bid & 7) * per_xcd + (bid >> 3);
    *wl_out = wl;
    *at_work = n;
    if ((bid >> 3) >= per_xcd || wl >= n) return false;
    auto begin_of = [&](int w) { return all / n * w + all % n * w / n; };
    const int64_t x[2] = {begin_of(wl), begin_of(wl + 1)};
    const bool to_end = wl + 1 == n;
    if (tid < 2) sh->r[tid] = b.B;
    __syncthreads();
    for (int c = 0; c < chunks; ++c) {
        const bool here[2] = {sh->chunk[c] <= x[0] && (c + 1 == chunks || x[0] < sh->chunk[c + 1]),
                              !to_end && sh->chunk[c] <= x[1] && (c + 1 == chunks || x[1] < sh->chunk[c + 1])};
        if (!here[0] && !here[1]) continue;  // (the same for the whole workgroup)
        if (chunks > 1) {
            bool unused = false;
            mine = latent_length(s, latent_request(b, s, c * 256 + tid, &unused));
            int64_t total = 0;
            incl = block_scan_64(mine, sh, &total);
        }
        const int64_t first = sh->chunk[c] + incl - mine;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (here[i] && mine > 0 && first <= x[i] && x[i] < first + mine) {
                sh->r[i] = c * 256 + tid;
                sh->at[i] = x[i] - first;
            }
    }
    __syncthreads();
    bool unused = false;
    LatentPlace p[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = __builtin_amdgcn_readfirstlane(sh->r[i]);
        p[i] = {b.B, 0, 0};
        if (r < b.B) p[i] = latent_place(s, latent_request(b, s, r, &unused), r, sh->at[i]);
        p[i].tile = __builtin_amdgcn_readfirstlane(p[i].tile);
        p[i].k = __builtin_amdgcn_readfirstlane(p[i].k);
    }
    *from = p[0];
    *to = p[1];
    __syncthreads();
    return true;
}

// What scores are measured against, from the largest of them (both in log2 units).  A probability is 2^(c s - m) out of one fused multiply-add, but m itself is
// rounded to 32 bits: from 2^22 on by so much that it shows, from 2^28 on by so much that the largest score's own probability would be 2^16 or 2^-16 and beyond.
// Such a maximum is taken a few steps lower than it is, so that no row's largest probabilities vanish, and what they are too large by, its user holds
// to a limit; scores that fp32 cannot tell apart then weigh the same.
__device__ __forceinline__ float moved_maximum(float largest) {
    const float a = fabsf(largest);
    return a >= 4194304.f && a < INFINITY ? largest - a * 2.384185791015625e-7f : largest;
}

// ... of a row that has met no score but -infinity: the next one outgrows it, however small
constexpr float kNoMaximum = -3.4028234663852886e38f;

// Partial results: slot 2 w holds what workgroup w did of a tile that it did not begin, slot 2 w + 1 of one that it began and did not finish.
// Slots 2 n .. 3 n - 1 are the workgroups' scratch memory.  Records of a slot: {first row of the output, rows, kPartHead | kPartLast, rows of the output from one to the next}; flags 0: nothing.
constexpr int kPartHead = 1, kPartLast = 2;
struct LatentParts {
    int32_t* hdr;   // 64 words; [3]: the batch did not fit; [6]: workgroups at work
    int4* rec;      // [2 n_wg]
    float2* ml;     // [2 n_wg][M]  row maximum (log2 units) and sum
    float* o;       // [3 n_wg][M][width]
};
struct LatentPartsLayout {
    size_t rec, ml, o, total;
};
inline LatentPartsLayout latent_parts_layout(int n_wg, int M, int width) {
    LatentPartsLayout l;
    l.rec = 256;
    l.ml = l.rec + static_cast<size_t>(2 * n_wg) * sizeof(int4);
    l.o = l.ml + static_cast<size_t>(2 * n_wg) * M * sizeof(float2);
    l.total = l.o + static_cast<size_t>(3 * n_wg) * M * width * sizeof(float);
    return l;
}
inline LatentParts latent_parts(void* at, const LatentPartsLayout& l) {
    unsigned char* const p = static_cast<unsigned char*>(at);
    return {reinterpret_cast<int32_t*>(p), reinterpret_cast<int4*>(p + l.rec), reinterpret_cast<float2*>(p + l.ml), reinterpret_cast<float*>(p + l.o)};
}

}  // namespace pa
