// Eviction of distant tokens by score (dar_cache_evict, dar_cache_evict_paged).
//
// For each row (sequence, KV head): of the D distant tokens the first n_fixed
// stay, and of the others the K = left - n_fixed with the highest scores, where
// left = D - E. Kept tokens at or past slot `left` (tails) move into the slots
// that evicted tokens leave below it (holes); there are as many of one as of
// the other, and the r-th tail goes to the r-th hole. No destination is a
// source, so the moves need no order and no staging, and a cache that loses one
// window's worth of tokens moves at most that many latents, however long it is.
//
// evict_select_kernel: one workgroup per row. Scores become integer keys whose
//   order is the scores' order; rows of up to 34816 candidates are read once and
//   kept in LDS, longer ones read again at each pass. The K-th largest key is
//   found by histograms over ever narrower key ranges: 4096 (16384) bins of the
//   range that holds it, at most three levels of 32-bit keys (a bin whose keys all
//   stay ends the search). Then a bit per token says whether it stays, 64 tokens a
//   word, first for the slots below `left`, then for the others: a prefix sum of
//   the words' counts gives every hole and tail its rank, and a thread walks its
//   word's holes or tails. (Ranks by ballots in unrolled code over keys in
//   registers took 19000 cycles of 116000 at 33999 tokens, its instructions
//   missing the cache; here 16 waves run loops of a few instructions a key.)
//   Lists that fit LDS are followed by the same workgroup, else by
// evict_move_kernel on the whole chip.
#include "../../include/dar_serving.h"
#include "dar_common.hpp"
#include "dar_kernels.hpp"

namespace dar {

namespace {

typedef unsigned int eu32x4 __attribute__((ext_vector_type(4)));

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kBinBits = 12, kBinBitsStream = 14;  // with and without keys in LDS
constexpr int kKeysShort = 8192, kKeysLong = 34816;  // candidates whose keys LDS holds
constexpr int kStreamPool = 64 * 1024;               // bytes for lists where it holds none
constexpr int kChunk = 64 * kSelThreads;             // tokens whose words are made at a time

// What one row's eviction does; E == 0: nothing.
struct RowPlan {
    int len, D, E, left, K;
};

__device__ __forceinline__ RowPlan row_plan(int len, int cap, int w, int n_keep, int n_fixed) {
    RowPlan p{};
    p.len = len < 1 || len > cap ? 0 : len;
    p.D = imax(p.len - w, 0);
    const int over = p.D - n_keep;
    p.E = over <= 0 ? 0 : (w > 0 ? over / w * w : over);
    p.left = p.D - p.E;
    p.K = p.left - n_fixed;
    return p;
}

// Keys in the order of the scores: NaN 1, then -inf .. -0 = 0 .. inf (0: no
// candidate). On the bits: the build assumes that floating-point values are no
// NaN.
__device__ __forceinline__ uint32_t score_key(uint32_t u) {
    const uint32_t k = u & 0x80000000u ? (u == 0x80000000u ? 0x80000000u : ~u) : u | 0x80000000u;
    return (u & 0x7fffffffu) > 0x7f800000u ? 1u : k;
}

// Inclusive prefix sum over the 64 lanes by DPP moves: rows of 16, then the two
// row broadcasts.
__device__ __forceinline__ uint32_t wave_prefix(uint32_t v) {
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false);  // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);  // row_bcast:15
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);  // row_bcast:31
    return v;
}

}  // namespace

// The latents of a cache: dense (bt NULL), or pages named by the block table.
struct LatRows {
    const int* bt;
    int maxb, n_pages, ps_shift, cap, Hkv;
    // first row of `slot` of (sequence b, KV head g), -1: no such page
    __device__ __forceinline__ long long at(int b, int g, int slot) const {
        if (bt == nullptr) return ((long long)b * Hkv + g) * cap + slot;
        const int page = bt[(size_t)b * maxb + (slot >> ps_shift)];
        if (page < 0 || page >= n_pages) return -1;
        return (((long long)page * Hkv + g) << ps_shift) + (slot & ((1 << ps_shift) - 1));
    }
};

// The moves r = first, first + step, ... below n of one row: part c of U-sized
// parts (key latents for c < ru, else value latents), kFlight moves in flight.
// Loads and stores go past the caches, which hold nothing twice here (B8 Hkv8
// d_down32, 131072 tokens cut to half: 342 -> 308 us).
constexpr int kFlight = 8;
template <typename U>
__device__ __forceinline__ void move_rows(U* k_lat, U* v_lat, const LatRows& rows, int b, int g,
                                          const int* from, const int* to, int n, int first, int step,
                                          int c, int ru) {
    U* const lat = c < ru ? k_lat : v_lat;
    const int cc = c < ru ? c : c - ru;
    for (int r0 = first; r0 < n; r0 += kFlight * step) {
        long long rt[kFlight];
        U x[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int r = r0 + i * step;
            rt[i] = -1;
            x[i] = U(0);
            if (r < n) {
                const long long rf = rows.at(b, g, from[r]);
                rt[i] = rows.at(b, g, to[r]);
                if (rf >= 0) x[i] = __builtin_nontemporal_load(lat + rf * ru + cc);
            }
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
            if (rt[i] >= 0) __builtin_nontemporal_store(x[i], lat + rt[i] * ru + cc);
    }
}

// move_rows by `threads` threads, of which this is number tid, sharing the moves
// with `parts` such groups (this one number part).
template <typename U>
__device__ __forceinline__ void move_share(U* k_lat, U* v_lat, const LatRows& rows, int b, int g,
                                           const int* from, const int* to, int n, int ru, int tid,
                                           int threads, int part, int parts) {
    const int lanes = 2 * ru, per = threads / lanes;  // moves of a group at a time
    if (per > 0) {
        const int sub = tid / lanes, c = tid - sub * lanes;
        if (sub < per)
            move_rows(k_lat, v_lat, rows, b, g, from, to, n, part * per + sub, per * parts, c, ru);
    } else {
        for (int c = tid; c < lanes; c += threads)
            move_rows(k_lat, v_lat, rows, b, g, from, to, n, part, parts, c, ru);
    }
}

// info[row] = {moves, E}; lists holes[row * stride + r], tails[row * stride + r]
// (FUSED: not written; the moves are made here, U-sized parts, ru a latent row).
// KEYS: candidates that LDS holds the keys of (0: none, any number).
template <int KEYS, bool FUSED, typename U>
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(
    const uint32_t* scores, uint32_t* scores_out, int2* __restrict__ info, int* holes, int* tails,
    int stride, int Hkv, int w, int cap, int len_arg, const int* __restrict__ lens, int n_keep,
    int n_fixed, U* k_lat, U* v_lat, int ru, LatRows lat) {
    constexpr int POOL = KEYS > 0 ? KEYS * 4 : kStreamPool;  // bytes: the keys, then the lists
    constexpr int BITS = KEYS > 0 ? kBinBits : kBinBitsStream, BINS = 1 << BITS;
    constexpr int BPT = BINS / kSelThreads;  // bins of a thread
    static_assert(BPT % 4 == 0, "read by fours");
    constexpr int WORDS = KEYS > 0 ? (KEYS / 64 + 15) & ~15 : kChunk / 64;  // (made 4 or 16 at a time)
    __shared__ __attribute__((aligned(16))) uint32_t pool[POOL / 4];
    __shared__ __attribute__((aligned(16))) uint32_t hist[BINS];  // then the words
    __shared__ uint32_t wsum[kSelWaves];
    __shared__ uint32_t pick[3];  // bin, keys above it, keys in it
    const int row = wg_id_x(), b = row / Hkv, g = row - b * Hkv;
    const int tid = lane_id_x(), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const RowPlan p = row_plan(lens ? lens[b] : len_arg, cap, w, n_keep, n_fixed);
    const uint32_t* in = scores + (size_t)row * cap;
    uint32_t* out = scores_out + (size_t)row * cap;
    const bool copy = scores != scores_out;
    const bool vec = (cap & 3) == 0;  // rows of scores start on 16 bytes
    if (p.E == 0) {
        if (!FUSED && tid == 0) info[row] = make_int2(0, 0);
        if (copy)
            for (int e = tid; e < p.len; e += kSelThreads) out[e] = in[e];
        return;
    }
    if (copy)
        for (int e = tid; e < n_fixed; e += kSelThreads) out[e] = in[e];
    int* const lh = FUSED ? (int*)pool : holes + (size_t)row * stride;
    int* const lt = FUSED ? (int*)pool + POOL / 8 : tails + (size_t)row * stride;

    // exclusive prefix and total of a count over the workgroup
    auto scan = [&](uint32_t v, uint32_t& total) -> uint32_t {
        static_assert(kSelWaves == 16, "a row of lanes holds the wavefronts' sums");
        const uint32_t inc = wave_prefix(v);
        if (lane == 63) wsum[wave] = inc;
        __syncthreads();
        const uint32_t sums = wave_prefix(lane < kSelWaves ? wsum[lane] : 0);
        total = __builtin_amdgcn_readlane(sums, kSelWaves - 1);
        const uint32_t before = wave > 0 ? __builtin_amdgcn_readlane(sums, imax(wave - 1, 0)) : 0;
        __syncthreads();  // wsum is used again
        return before + inc - v;
    };
    int moves = 0;
    if (p.K > 0) {
        const int a0 = n_fixed & ~3, ngrp = (p.D - a0 + 3) >> 2;  // groups of four from a0 on
        auto fetch = [&](int e) -> uint4 {
            uint4 u = make_uint4(0, 0, 0, 0);
            if (vec) {
                if (e < p.D) u = *reinterpret_cast<const uint4*>(in + e);
            } else {
                if (e < p.D) u.x = in[e];
                if (e + 1 < p.D) u.y = in[e + 1];
                if (e + 2 < p.D) u.z = in[e + 2];
                if (e + 3 < p.D) u.w = in[e + 3];
            }
            return u;
        };
        auto keys_of = [&](int e, const uint4& u) -> uint4 {
            uint4 k = make_uint4(score_key(u.x), score_key(u.y), score_key(u.z), score_key(u.w));
            if (e < n_fixed || e + 3 >= p.D) {  // an end of the row
                k.x = e >= n_fixed && e < p.D ? k.x : 0;
                k.y = e + 1 >= n_fixed && e + 1 < p.D ? k.y : 0;
                k.z = e + 2 >= n_fixed && e + 2 < p.D ? k.z : 0;
                k.w = e + 3 >= n_fixed && e + 3 < p.D ? k.w : 0;
            }
            return k;
        };
        // scores below `left` to their places (holes are filled later)
        auto pass_on = [&](int e, const uint4& u) {
            if (e >= p.left) return;
            if (vec && e >= n_fixed && e + 3 < p.left) {
                *reinterpret_cast<uint4*>(out + e) = u;
            } else {
                const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (e + j >= n_fixed && e + j < p.left) out[e + j] = x[j];
            }
        };
        auto clear = [&]() {
#pragma unroll
            for (int i = 0; i < BPT / 4; ++i)
                reinterpret_cast<uint4*>(hist)[tid + i * kSelThreads] = make_uint4(0, 0, 0, 0);
            __syncthreads();
        };
        // ---- the K-th largest key (it lies in lo .. lo + span) and its rank from
        // the top among the keys there
        uint32_t lo = 1, span = 0xfffffffeu, want = (uint32_t)p.K;
        int sh = 32 - BITS;
        bool ties;  // of the keys equal to lo only `want` stay
        auto count = [&](const uint4& k) {
            if (k.x - lo <= span) atomicAdd(&hist[(k.x - lo) >> sh], 1u);
            if (k.y - lo <= span) atomicAdd(&hist[(k.y - lo) >> sh], 1u);
            if (k.z - lo <= span) atomicAdd(&hist[(k.z - lo) >> sh], 1u);
            if (k.w - lo <= span) atomicAdd(&hist[(k.w - lo) >> sh], 1u);
        };
        clear();
        constexpr int kAhead = KEYS > 0 ? 4 : 8;  // loads in flight a thread
        bool first = true;
        for (;;) {
            if (KEYS == 0 || first) {
                for (int i0 = tid; i0 < ngrp; i0 += kAhead * kSelThreads) {
                    uint4 u[kAhead];
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) u[i] = fetch(a0 + 4 * (i0 + i * kSelThreads));
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const int gi = i0 + i * kSelThreads, e = a0 + 4 * gi;
                        if (gi < ngrp) {
                            if (first && copy) pass_on(e, u[i]);
                            const uint4 k = keys_of(e, u[i]);
                            if constexpr (KEYS > 0) reinterpret_cast<uint4*>(pool)[gi] = k;
                            count(k);
                        }
                    }
                }
            } else {
                for (int gi = tid; gi < ngrp; gi += kSelThreads) count(reinterpret_cast<const uint4*>(pool)[gi]);
            }
            first = false;
            __syncthreads();
            // thread t: BPT bins from the top, thread 0 the highest
            const int b0 = BINS - BPT * (tid + 1);
            uint32_t c[BPT], mine = 0;
#pragma unroll
            for (int i = 0; i < BPT / 4; ++i) {
                const uint4 u = *reinterpret_cast<const uint4*>(hist + b0 + 4 * i);
                c[4 * i] = u.x;
                c[4 * i + 1] = u.y;
                c[4 * i + 2] = u.z;
                c[4 * i + 3] = u.w;
                mine += u.x + u.y + u.z + u.w;
            }
            uint32_t total;
            uint32_t above = scan(mine, total);
            if (want > above && want <= above + mine) {
#pragma unroll
                for (int i = BPT - 1; i >= 0; --i) {
                    if (want > above && want <= above + c[i]) {
                        pick[0] = b0 + i;
                        pick[1] = above;
                        pick[2] = c[i];
                    }
                    above += c[i];
                }
            }
            __syncthreads();
            lo += pick[0] << sh;
            span = (1u << sh) - 1u;
            want -= pick[1];
            ties = want != pick[2];
            if (sh == 0 || !ties) break;
            sh = sh > BITS ? sh - BITS : 0;
            clear();
        }
        const uint32_t T = lo, least = ties ? T + 1 : T;  // (T is below the keys' last value)
        // ---- ranks. Without ties every key >= T stays; else those above T, and of
        // the keys equal to it the first `want`. kept: those in front of the chunk.
        uint32_t kept = 0, equal = 0;
        static_assert(2 * WORDS * sizeof(uint64_t) <= sizeof(hist), "the words take the histogram's place");
        uint64_t* const above_bits = reinterpret_cast<uint64_t*>(hist);
        uint64_t* const equal_bits = above_bits + WORDS;
        __syncthreads();
        auto rank_region = [&](int ra, int rb, bool low, uint32_t kept_low) {
            for (int c0 = ra; c0 < rb; c0 += 64 * WORDS) {
                const int c1 = imin(c0 + 64 * WORDS, rb), nwords = (c1 - c0 + 63) >> 6;
                constexpr int kWide = KEYS > 0 ? 4 : 16;  // words in flight a wavefront
                for (int w0 = wave * kWide; w0 < nwords; w0 += kWide * kSelWaves) {
                    uint32_t k[kWide];
#pragma unroll
                    for (int i = 0; i < kWide; ++i) {
                        const int e = c0 + 64 * (w0 + i) + lane;
                        if constexpr (KEYS > 0) k[i] = e < c1 ? pool[e - a0] : 0;
                        else k[i] = e < c1 ? score_key(in[e]) : 0;
                    }
                    uint64_t ma[kWide], me[kWide];
#pragma unroll
                    for (int i = 0; i < kWide; ++i) {
                        ma[i] = __builtin_amdgcn_ballot_w64(k[i] >= least);
                        me[i] = ties ? __builtin_amdgcn_ballot_w64(k[i] == T) : 0;
                    }
                    if (lane == 0) {
#pragma unroll
                        for (int i = 0; i < kWide; ++i) {
                            above_bits[w0 + i] = ma[i];
                            equal_bits[w0 + i] = me[i];
                        }
                    }
                }
                __syncthreads();
                uint64_t mine = tid < nwords ? above_bits[tid] : 0;
                uint32_t total;
                if (ties) {
                    uint64_t me = tid < nwords ? equal_bits[tid] : 0;
                    const uint32_t before = equal + scan(__builtin_popcountll(me), total);
                    equal += total;
                    for (uint32_t take = before < want ? want - before : 0; take > 0 && me; --take) {
                        mine |= me & -me;
                        me &= me - 1;
                    }
                }
                const uint32_t kb = kept + scan(__builtin_popcountll(mine), total);
                kept += total;
                const int e0 = c0 + 64 * tid, nv = imin(c1 - e0, 64);
                uint64_t todo = low ? ~mine : mine;
                todo = nv <= 0 ? 0 : nv < 64 ? todo & ((1ull << nv) - 1) : todo;
                int r = low ? e0 - n_fixed - (int)kb : (int)(kb - kept_low);
                int* const list = low ? lh : lt;
                // a full word by the wavefront's lanes, a thin one by its thread
                uint64_t full = __builtin_amdgcn_ballot_w64(__builtin_popcountll(todo) > 8);
                for (uint64_t f = full; f; f &= f - 1) {
                    const int src = __builtin_ctzll(f);
                    const uint64_t bits = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(todo >> 32), src) << 32) |
                                          (uint32_t)__builtin_amdgcn_readlane((int)todo, src);
                    const int at = __builtin_amdgcn_readlane(r, src) +
                                   (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0));
                    if (bits >> lane & 1) list[at] = c0 + 64 * (64 * wave + src) + lane;
                }
                if (!(full >> lane & 1))
                    for (; todo; todo &= todo - 1) list[r++] = e0 + __builtin_ctzll(todo);
                __syncthreads();  // the words are used again
            }
        };
        // (FUSED: the lists lie where the keys were. The holes' list is no longer than
        // the low region, whose words are made; the tails' follows the high region's.)
        rank_region(n_fixed, p.left, true, 0);
        const uint32_t kept_low = kept;
        moves = p.K - (int)kept_low;
        rank_region(p.left, p.D, false, kept_low);
    }
    __syncthreads();  // the lists are complete, and `out` below `left` but for the holes
    constexpr int kGather = 4;
    for (int r0 = tid; r0 < moves; r0 += kGather * kSelThreads) {
        uint32_t z[kGather];
#pragma unroll
        for (int i = 0; i < kGather; ++i) {
            const int r = r0 + i * kSelThreads;
            z[i] = r < moves ? in[lt[r]] : 0;
        }
#pragma unroll
        for (int i = 0; i < kGather; ++i) {
            const int r = r0 + i * kSelThreads;
            if (r < moves) out[lh[r]] = z[i];
        }
    }
    if constexpr (FUSED)
        move_share(k_lat, v_lat, lat, b, g, lt, lh, moves, ru, tid, kSelThreads, 0, 1);
    __syncthreads();  // tails are read before entries past `left` change
    // The window's entries move down by E >= w, to a range that does not meet their
    // own; entries len - E .. len - 1 become zero, each of those in the window's
    // old range by the thread that has read it.
    for (int e = p.left + tid; e < p.len; e += kSelThreads) {
        if (e >= p.D) out[e - p.E] = in[e];
        if (e >= p.len - p.E) out[e] = 0;
    }
    if (!FUSED && tid == 0) info[row] = make_int2(moves, p.E);
}

// The moves of one row, parts of them spread over the grid's x.
template <typename U>
__global__ __launch_bounds__(256) void evict_move_kernel(U* k_lat, U* v_lat,
                                                         const int2* __restrict__ info,
                                                         const int* __restrict__ holes,
                                                         const int* __restrict__ tails, int stride,
                                                         int Hkv, int ru, LatRows lat, int* lens,
                                                         int parts) {
    const int row = wg_id_y(), b = row / Hkv, g = row - b * Hkv;
    const int2 inf = info[row];
    // the sequence's length: nothing in this launch reads it
    if (lens && g == 0 && wg_id_x() == 0 && lane_id_x() == 0 && inf.y > 0) lens[b] -= inf.y;
    move_share(k_lat, v_lat, lat, b, g, tails + (size_t)row * stride, holes + (size_t)row * stride,
               inf.x, ru, lane_id_x(), 256, wg_id_x(), parts);
}

// lens[b] -= E of sequence b (the selection made the moves itself).
__global__ __launch_bounds__(256) void evict_lens_kernel(int* lens, int B, int cap, int w, int n_keep) {
    const int b = wg_id_x() * 256 + lane_id_x();
    if (b < B) lens[b] -= row_plan(lens[b], cap, w, n_keep, 0).E;
}

// Moves of one row, at most: the evicted tokens, and the kept ones.
int evict_max_moves(int cap, int w, int n_keep) {
    const long long over = (long long)cap - w - n_keep;
    if (over <= 0) return 0;
    const long long kept = (long long)n_keep + (w > 0 ? w - 1 : 0);
    return (int)(over < kept ? over : kept);
}

template <typename U>
static hipError_t launch_evict_u(const uint32_t* scores, uint32_t* scores_out, U* k_lat, U* v_lat,
                                 void* ws, int B, int Hkv, int ru, int w, int cap, int len, int n_keep,
                                 int n_fixed, const LatRows& lat, int* lens, hipStream_t st) {
    const int rows = B * Hkv;
    const int stride = evict_max_moves(cap, w, n_keep);
    int2* info = (int2*)ws;
    int* holes = (int*)(info + rows);
    int* tails = holes + (size_t)rows * stride;
    // candidates of the longest row, and the lists that then fit LDS
    const int most = (lens ? cap : len) - w - (n_fixed & ~3);
    const int room = (most <= kKeysShort ? kKeysShort * 4 : most <= kKeysLong ? kKeysLong * 4 : kStreamPool) / 8;
    // The selecting workgroups make the moves themselves where the lists fit and
    // either the moves are few or every row of a full chip has as many (dense): one
    // launch less, and no list goes through memory. (Sequences of 2K to 32K tokens
    // cut to 8K: 84 us with the move kernel, 92 without, the longest rows last.)
    const bool fused = stride <= room && ((rows >= 256 && !lens) || stride <= 2048);
#define DAR_SELECT(K_, F_)                                                                         \
    hipLaunchKernelGGL((evict_select_kernel<K_, F_, U>), dim3(rows), dim3(kSelThreads), 0, st,     \
                       scores, scores_out, info, holes, tails, stride, Hkv, w, cap, len, lens,     \
                       n_keep, n_fixed, k_lat, v_lat, ru, lat)
#define DAR_SELECT_F(K_)              \
    if (fused) DAR_SELECT(K_, true);  \
    else DAR_SELECT(K_, false);
    if (most <= kKeysShort) { DAR_SELECT_F(kKeysShort) }
    else if (most <= kKeysLong) { DAR_SELECT_F(kKeysLong) }
    else { DAR_SELECT_F(0) }
#undef DAR_SELECT_F
#undef DAR_SELECT
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (fused) {
        if (lens) {
            hipLaunchKernelGGL(evict_lens_kernel, dim3((B + 255) / 256), dim3(256), 0, st, lens, B, cap,
                               w, n_keep);
            e = hipGetLastError();
        }
        return e;
    }
    long long nb = ((long long)stride * 2 * ru + 2047) / 2048;
    const long long fill = (16 * 256 + rows - 1) / rows;  // about 16 workgroups a compute unit
    nb = nb > fill ? fill : nb;
    hipLaunchKernelGGL((evict_move_kernel<U>), dim3((unsigned)nb, rows), dim3(256), 0, st, k_lat, v_lat,
                       info, holes, tails, stride, Hkv, ru, lat, lens, (int)nb);
    return hipGetLastError();
}

hipError_t launch_evict(const float* scores, float* scores_out, void* k_lat, void* v_lat, void* ws,
                        int B, int Hkv, int row_bytes, int esize, int w, int cap, int len,
                        int n_keep, int n_fixed, const PagedArgs* pg, int* lens, hipStream_t st) {
    const LatRows lat{pg ? pg->bt : nullptr, pg ? pg->maxb : 0, pg ? pg->n_pages : 0,
                      pg ? pg->ps_shift : 0, cap, Hkv};
    const uint32_t* in = (const uint32_t*)scores;
    uint32_t* out = (uint32_t*)scores_out;
    if (row_bytes % 16 == 0)
        return launch_evict_u(in, out, (eu32x4*)k_lat, (eu32x4*)v_lat, ws, B, Hkv, row_bytes / 16, w, cap,
                              len, n_keep, n_fixed, lat, lens, st);
    if (esize == 4)
        return launch_evict_u(in, out, (uint32_t*)k_lat, (uint32_t*)v_lat, ws, B, Hkv, row_bytes / 4, w,
                              cap, len, n_keep, n_fixed, lat, lens, st);
    return launch_evict_u(in, out, (uint16_t*)k_lat, (uint16_t*)v_lat, ws, B, Hkv, row_bytes / 2, w, cap,
                          len, n_keep, n_fixed, lat, lens, st);
}

}  // namespace dar
