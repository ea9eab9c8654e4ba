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
// evict_select_kernel: one workgroup per row of up to 34816 candidates. Scores
//   become integer keys whose order is the scores' order, read once and kept in
//   LDS. The K-th largest key is found by histograms over ever narrower key
//   ranges: 4096 bins of the range that holds it, at most three levels of 32-bit
//   keys (a bin whose keys all stay ends the search). Then a bit per token says
//   whether it stays, 64 tokens a word, first for the slots below `left`, then for
//   the others: a prefix sum of the words' counts gives every hole and tail its
//   rank, and a thread walks its word's holes or tails. (Ranks by ballots in
//   unrolled code over keys in registers took 19000 cycles of 116000 at 33999
//   tokens, its instructions missing the cache; here 16 waves run loops of a few
//   instructions a key.) Lists that fit LDS are followed by the same workgroup,
//   else by
// evict_move_kernel on the whole chip.
// Longer rows: the same steps as launches of several workgroups a row, each with
//   a share of its tokens. evict_count_kernel three times (the workgroups'
//   histograms are added up in memory, in integers, so in any order alike; every
//   workgroup finds the range for itself), evict_words_kernel (the bits, and each
//   share's counts), evict_lists_kernel (the ranks go on from the shares before),
//   the moves with their scores, and evict_shift_kernel for what lies past `left`.
//   They begin where LDS ends; before it they are no faster: 24000 tokens cut to
//   half, one workgroup a row and several, 8 rows 33.9 and 37.1 us, 64 rows 57.8 and
//   70.3, 256 rows 139 and 183; 34500 tokens 40.3 and 39.8, 75.4 and 84.2, 196 and
//   243. Then several: 35600 tokens 40.5, 84.9 and 251 us.
#include "../../include/dar_serving.h"
#include "dar_common.hpp"
#include "dar_kernels.hpp"

namespace dar {

namespace {

typedef unsigned int eu32x4 __attribute__((ext_vector_type(4)));

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kBinBits = 12, kBins = 1 << kBinBits;
constexpr int kKeysShort = 8192, kKeysLong = 34816;  // candidates whose keys LDS holds
constexpr int kSplitThreads = 512, kSplitWaves = kSplitThreads / 64;
constexpr int kMaxParts = 64;    // workgroups of a row, at most
constexpr int kMinPart = 4096;   // tokens of a workgroup, at least

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

// Exclusive prefix and total of a count over a workgroup of WAVES wavefronts.
template <int WAVES>
__device__ __forceinline__ uint32_t group_scan(uint32_t v, uint32_t& total, uint32_t* wsum, int lane,
                                               int wave) {
    static_assert(WAVES <= 16, "a row of lanes holds the wavefronts' sums");
    const uint32_t inc = wave_prefix(v);
    if (lane == 63) wsum[wave] = inc;
    __syncthreads();
    const uint32_t sums = wave_prefix(lane < WAVES ? wsum[lane] : 0);
    total = __builtin_amdgcn_readlane(sums, WAVES - 1);
    const uint32_t before = wave > 0 ? __builtin_amdgcn_readlane(sums, imax(wave - 1, 0)) : 0;
    __syncthreads();  // wsum is used again
    return before + inc - v;
}

// The bin that holds the want-th key from the top, of THREADS * BPT bins: its
// number, the keys above it and those in it into pick (a barrier follows).
// Thread t has BPT bins from the top (bins_of), thread 0 the highest.
template <int THREADS, int BPT>
__device__ __forceinline__ void bins_of(const uint32_t* hist, int tid, uint32_t (&c)[BPT]) {
    static_assert(BPT % 4 == 0, "read by fours");
    const int b0 = THREADS * BPT - BPT * (tid + 1);
#pragma unroll
    for (int i = 0; i < BPT / 4; ++i) {
        const uint4 u = *reinterpret_cast<const uint4*>(hist + b0 + 4 * i);
        c[4 * i] = u.x;
        c[4 * i + 1] = u.y;
        c[4 * i + 2] = u.z;
        c[4 * i + 3] = u.w;
    }
}
template <int THREADS, int BPT>
__device__ __forceinline__ void find_bin(const uint32_t (&c)[BPT], uint32_t want, uint32_t* pick,
                                         uint32_t* wsum, int tid, int lane, int wave) {
    const int b0 = THREADS * BPT - BPT * (tid + 1);
    uint32_t total, mine = 0;
#pragma unroll
    for (int i = 0; i < BPT; ++i) mine += c[i];
    uint32_t above = group_scan<THREADS / 64>(mine, total, wsum, lane, wave);
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
}

// The tokens whose bits are set in `todo`, a word of 64 a thread, into `list` from
// place r on; e0: the wavefront's first word's first token. A full word by the
// wavefront's lanes, a thin one by its thread.
__device__ __forceinline__ void write_list(int* list, uint64_t todo, int r, int e0, int lane) {
    const uint64_t full = __builtin_amdgcn_ballot_w64(__builtin_popcountll(todo) > 8);
    for (uint64_t f = full; f; f &= f - 1) {
        const int src = __builtin_ctzll(f);
        const uint64_t bits = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(todo >> 32), src) << 32) |
                              (uint32_t)__builtin_amdgcn_readlane((int)todo, src);
        const int at = __builtin_amdgcn_readlane(r, src) +
                       (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0));
        if (bits >> lane & 1) list[at] = e0 + 64 * src + lane;
    }
    if (!(full >> lane & 1))
        for (; todo; todo &= todo - 1) list[r++] = e0 + 64 * lane + __builtin_ctzll(todo);
}

// A row's scores by groups of four.
struct RowScores {
    const uint32_t* in;
    uint32_t* out;
    bool vec;  // rows of scores start on 16 bytes
    int n_fixed, D, left;
    __device__ __forceinline__ uint4 fetch(int e) const {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (vec) {
            if (e < D) u = *reinterpret_cast<const uint4*>(in + e);
        } else {
            if (e < D) u.x = in[e];
            if (e + 1 < D) u.y = in[e + 1];
            if (e + 2 < D) u.z = in[e + 2];
            if (e + 3 < D) u.w = in[e + 3];
        }
        return u;
    }
    __device__ __forceinline__ uint4 keys_of(int e, const uint4& u) const {
        uint4 k = make_uint4(score_key(u.x), score_key(u.y), score_key(u.z), score_key(u.w));
        if (e < n_fixed || e + 3 >= D) {  // an end of the row
            k.x = e >= n_fixed && e < D ? k.x : 0;
            k.y = e + 1 >= n_fixed && e + 1 < D ? k.y : 0;
            k.z = e + 2 >= n_fixed && e + 2 < D ? k.z : 0;
            k.w = e + 3 >= n_fixed && e + 3 < D ? k.w : 0;
        }
        return k;
    }
    // scores below `left` to their places (holes are filled later)
    __device__ __forceinline__ void pass_on(int e, const uint4& u) const {
        if (e >= left) return;
        if (vec && e >= n_fixed && e + 3 < left) {
            *reinterpret_cast<uint4*>(out + e) = u;
        } else {
            const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e + j >= n_fixed && e + j < left) out[e + j] = x[j];
        }
    }
};

// Scores of the moves r = first, first + step, ... below n.
__device__ __forceinline__ void move_scores(const uint32_t* in, uint32_t* out, const int* from,
                                            const int* to, int n, int first, int step) {
    constexpr int kGather = 4;
    for (int r0 = first; r0 < n; r0 += kGather * step) {
        uint32_t z[kGather];
#pragma unroll
        for (int i = 0; i < kGather; ++i) {
            const int r = r0 + i * step;
            z[i] = r < n ? in[from[r]] : 0;
        }
#pragma unroll
        for (int i = 0; i < kGather; ++i) {
            const int r = r0 + i * step;
            if (r < n) out[to[r]] = z[i];
        }
    }
}

// What lies past `left`, entries left + first, left + first + step, ...: the
// window's entries move down by E >= w, to a range that does not meet their own;
// entries len - E .. len - 1 become zero, each of those in the window's old range
// by the thread that has read it.
__device__ __forceinline__ void shift_scores(const uint32_t* in, uint32_t* out, const RowPlan& p,
                                             int first, int step) {
    for (int e = p.left + first; e < p.len; e += step) {
        if (e >= p.D) out[e - p.E] = in[e];
        if (e >= p.len - p.E) out[e] = 0;
    }
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
// d_down32, 131072 tokens cut to half: 34 us of the call). Bound by the scatter: rows of
// 2 dd bytes in lines of 128, 32500 of which for each of 64 heads take 158 us, 3.4 TB/s
// of what they name.
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
// KEYS: candidates that LDS holds the keys of.
template <int KEYS, bool FUSED, typename U>
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(
    const uint32_t* scores, uint32_t* scores_out, int2* __restrict__ info, int* holes, int* tails,
    int stride, int Hkv, int w, int cap, int len_arg, const int* __restrict__ lens, int n_keep,
    int n_fixed, U* k_lat, U* v_lat, int ru, LatRows lat) {
    constexpr int POOL = KEYS * 4;  // bytes: the keys, then the lists
    constexpr int BPT = kBins / kSelThreads;  // bins of a thread
    constexpr int WORDS = (KEYS / 64 + 3) & ~3;  // (made four at a time)
    static_assert(WORDS <= kSelThreads, "a thread a word");
    __shared__ __attribute__((aligned(16))) uint32_t pool[POOL / 4];
    __shared__ __attribute__((aligned(16))) uint32_t hist[kBins];  // then the words
    __shared__ uint32_t wsum[kSelWaves];
    __shared__ uint32_t pick[3];  // bin, keys above it, keys in it
    const int row = wg_id_x(), b = row / Hkv, g = row - b * Hkv;
    const int tid = lane_id_x(), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const RowPlan p = row_plan(lens ? lens[b] : len_arg, cap, w, n_keep, n_fixed);
    const uint32_t* in = scores + (size_t)row * cap;
    uint32_t* out = scores_out + (size_t)row * cap;
    const bool copy = scores != scores_out;
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

    auto scan = [&](uint32_t v, uint32_t& total) { return group_scan<kSelWaves>(v, total, wsum, lane, wave); };
    int moves = 0;
    if (p.K > 0) {
        const int a0 = n_fixed & ~3, ngrp = (p.D - a0 + 3) >> 2;  // groups of four from a0 on
        const RowScores rs{in, out, (cap & 3) == 0, n_fixed, p.D, p.left};
        auto clear = [&]() {
#pragma unroll
            for (int i = 0; i < BPT / 4; ++i)
                reinterpret_cast<uint4*>(hist)[tid + i * kSelThreads] = make_uint4(0, 0, 0, 0);
            __syncthreads();
        };
        // ---- the K-th largest key (it lies in lo .. lo + span) and its rank from
        // the top among the keys there
        uint32_t lo = 1, span = 0xfffffffeu, want = (uint32_t)p.K;
        int sh = 32 - kBinBits;
        bool ties;  // of the keys equal to lo only `want` stay
        auto count = [&](const uint4& k) {
            if (k.x - lo <= span) atomicAdd(&hist[(k.x - lo) >> sh], 1u);
            if (k.y - lo <= span) atomicAdd(&hist[(k.y - lo) >> sh], 1u);
            if (k.z - lo <= span) atomicAdd(&hist[(k.z - lo) >> sh], 1u);
            if (k.w - lo <= span) atomicAdd(&hist[(k.w - lo) >> sh], 1u);
        };
        clear();
        constexpr int kAhead = 4;  // loads in flight a thread
        bool first = true;
        for (;;) {
            if (first) {
                for (int i0 = tid; i0 < ngrp; i0 += kAhead * kSelThreads) {
                    uint4 u[kAhead];
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) u[i] = rs.fetch(a0 + 4 * (i0 + i * kSelThreads));
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const int gi = i0 + i * kSelThreads, e = a0 + 4 * gi;
                        if (gi < ngrp) {
                            if (copy) rs.pass_on(e, u[i]);
                            const uint4 k = rs.keys_of(e, u[i]);
                            reinterpret_cast<uint4*>(pool)[gi] = k;
                            count(k);
                        }
                    }
                }
            } else {
                for (int gi = tid; gi < ngrp; gi += kSelThreads) count(reinterpret_cast<const uint4*>(pool)[gi]);
            }
            first = false;
            __syncthreads();
            uint32_t c[BPT];
            bins_of<kSelThreads, BPT>(hist, tid, c);
            find_bin<kSelThreads, BPT>(c, want, pick, wsum, tid, lane, wave);
            lo += pick[0] << sh;
            span = (1u << sh) - 1u;
            want -= pick[1];
            ties = want != pick[2];
            if (sh == 0 || !ties) break;
            sh = sh > kBinBits ? sh - kBinBits : 0;
            clear();
        }
        const uint32_t T = lo, least = ties ? T + 1 : T;  // (T is below the keys' last value)
        // ---- ranks. Without ties every key >= T stays; else those above T, and of
        // the keys equal to it the first `want`.
        uint32_t kept = 0, equal = 0;
        static_assert(2 * WORDS * sizeof(uint64_t) <= sizeof(hist), "the words take the histogram's place");
        uint64_t* const above_bits = reinterpret_cast<uint64_t*>(hist);
        uint64_t* const equal_bits = above_bits + WORDS;
        __syncthreads();
        auto rank_region = [&](int c0, int c1, bool low, uint32_t kept_low) {
            const int nwords = (c1 - c0 + 63) >> 6;
            constexpr int kWide = 4;  // words in flight a wavefront
            for (int w0 = wave * kWide; w0 < nwords; w0 += kWide * kSelWaves) {
                uint32_t k[kWide];
#pragma unroll
                for (int i = 0; i < kWide; ++i) {
                    const int e = c0 + 64 * (w0 + i) + lane;
                    k[i] = e < c1 ? pool[e - a0] : 0;
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
            const int r = low ? e0 - n_fixed - (int)kb : (int)(kb - kept_low);
            write_list(low ? lh : lt, todo, r, c0 + 64 * 64 * wave, lane);
            __syncthreads();  // the words are used again
        };
        // (FUSED: the lists lie where the keys were. The holes' list is no longer than
        // the low region, whose words are made; the tails' follows the high region's.)
        rank_region(n_fixed, p.left, true, 0);
        const uint32_t kept_low = kept;
        moves = p.K - (int)kept_low;
        rank_region(p.left, p.D, false, kept_low);
    }
    __syncthreads();  // the lists are complete, and `out` below `left` but for the holes
    move_scores(in, out, lt, lh, moves, tid, kSelThreads);
    if constexpr (FUSED)
        move_share(k_lat, v_lat, lat, b, g, lt, lh, moves, ru, tid, kSelThreads, 0, 1);
    __syncthreads();  // tails are read before entries past `left` change
    shift_scores(in, out, p, tid, kSelThreads);
    if (!FUSED && tid == 0) info[row] = make_int2(moves, p.E);
}

// ---- rows with more candidates than LDS holds: `parts` workgroups a row, grid
// (parts, rows). Bound by latency: 64 rows of 131072 tokens take 5 us to clear, 13,
// 11 and 9 to count, 17 for the words, 15 for the lists, 7 to shift (one workgroup
// a row took 142), before and after moves of 158 us.

// A row's share of the workspace: histograms of the three levels [3][kBins], counts
// of the parts [kMaxParts] (staying and tied tokens below `left`, the same past it), words
// of staying and of tied tokens [2][words], words = ceil(cap / 64).
struct SplitWs {
    uint32_t* hist;
    uint4* counts;
    uint64_t* bits;
    int words;
};

// Tokens [from, to) of a part, whole words of the row.
__device__ __forceinline__ void part_range(const RowPlan& p, int n_fixed, int part, int parts, int& from,
                                           int& to) {
    const int a0 = n_fixed & ~63, chunk = ((p.D - a0 + parts - 1) / parts + 63) & ~63;
    const long long f = a0 + (long long)chunk * part;
    from = (int)(f < p.D ? f : p.D);
    to = p.D - from < chunk ? p.D : from + chunk;
}

// The K-th largest key from `levels` levels of histograms: it lies in key ..
// key + 2^sh - 1, the want-th from the top of the keys there, not all of which
// stay (ties). Bits of a level: 12, 12, 8.
struct Pivot {
    uint32_t key, want;
    int sh;
    bool ties;
};
constexpr int kSplitBpt = kBins / kSplitThreads;
// The histograms of all levels are requested at once, then searched one by one.
struct LevelBins {
    uint32_t c[3][kSplitBpt];
    __device__ __forceinline__ LevelBins(const uint32_t* hist, int levels, int tid) {
#pragma unroll
        for (int l = 0; l < 3; ++l)
            if (l < levels) bins_of<kSplitThreads, kSplitBpt>(hist + l * kBins, tid, c[l]);
    }
    __device__ __forceinline__ Pivot find(int levels, int K, uint32_t* pick, uint32_t* wsum, int tid,
                                          int lane, int wave) const {
        Pivot v{0, (uint32_t)K, 32, true};
#pragma unroll
        for (int l = 0; l < 3; ++l) {
            if (l >= levels || !v.ties) continue;
            v.sh = imax(v.sh - kBinBits, 0);
            find_bin<kSplitThreads, kSplitBpt>(c[l], v.want, pick, wsum, tid, lane, wave);
            v.key += pick[0] << v.sh;
            v.want -= pick[1];
            v.ties = v.want != pick[2];
            __syncthreads();  // pick is used again
        }
        return v;
    }
};

__global__ __launch_bounds__(256) void evict_clear_kernel(uint4* __restrict__ hist, int n) {
    const int i = wg_id_x() * 256 + lane_id_x();
    if (i < n) hist[i] = make_uint4(0, 0, 0, 0);
}

__global__ __launch_bounds__(kSplitThreads) void evict_count_kernel(
    const uint32_t* scores, uint32_t* scores_out, SplitWs ws, int Hkv, int w, int cap, int len_arg,
    const int* __restrict__ lens, int n_keep, int n_fixed, int level, int parts) {
    __shared__ __attribute__((aligned(16))) uint32_t hist[kBins];
    __shared__ uint32_t wsum[kSplitWaves];
    __shared__ uint32_t pick[3];
    const int part = wg_id_x(), row = wg_id_y(), b = row / Hkv;
    const int tid = lane_id_x(), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const RowPlan p = row_plan(lens ? lens[b] : len_arg, cap, w, n_keep, n_fixed);
    const uint32_t* in = scores + (size_t)row * cap;
    uint32_t* out = scores_out + (size_t)row * cap;
    const bool copy = scores != scores_out && level == 0;
    if (copy) {  // what stays in its place for certain
        const int n = p.E == 0 ? p.len : n_fixed;
        for (int e = part * kSplitThreads + tid; e < n; e += parts * kSplitThreads) out[e] = in[e];
    }
    if (p.E == 0 || p.K <= 0) return;
    uint32_t* const rhist = ws.hist + (size_t)row * 3 * kBins;
    const Pivot v = LevelBins(rhist, level, tid).find(level, p.K, pick, wsum, tid, lane, wave);
    if (!v.ties) return;
    const RowScores rs{in, out, (cap & 3) == 0, n_fixed, p.D, p.left};
    int from, to;
    part_range(p, n_fixed, part, parts, from, to);
    constexpr int kAhead = 4;
    for (int i = tid; i < kBins / 4; i += kSplitThreads) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    const int sh = imax(v.sh - kBinBits, 0);
    // the range's keys (0: no candidate, not counted)
    const uint32_t lo = v.key ? v.key : 1;
    const uint32_t span = (level == 0 ? ~0u : (1u << v.sh) - 1u) - (lo - v.key);
    auto count = [&](uint32_t k) {
        if (k - lo <= span) atomicAdd(&hist[(k - v.key) >> sh], 1u);
    };
    for (int e0 = from + 4 * tid; e0 < to; e0 += 4 * kAhead * kSplitThreads) {
        uint4 u[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) u[i] = rs.fetch(e0 + 4 * i * kSplitThreads);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int e = e0 + 4 * i * kSplitThreads;
            if (e < to) {
                if (copy) rs.pass_on(e, u[i]);
                const uint4 k = rs.keys_of(e, u[i]);
                count(k.x);
                count(k.y);
                count(k.z);
                count(k.w);
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < kBins; i += kSplitThreads)
        if (hist[i]) atomicAdd(&rhist[level * kBins + i], hist[i]);
}

__global__ __launch_bounds__(kSplitThreads) void evict_words_kernel(
    const uint32_t* scores, SplitWs ws, int Hkv, int w, int cap, int len_arg,
    const int* __restrict__ lens, int n_keep, int n_fixed, int parts) {
    __shared__ uint32_t wsum[kSplitWaves];
    __shared__ uint32_t pick[3];
    __shared__ uint4 sums[kSplitWaves];
    const int part = wg_id_x(), row = wg_id_y(), b = row / Hkv;
    const int tid = lane_id_x(), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const RowPlan p = row_plan(lens ? lens[b] : len_arg, cap, w, n_keep, n_fixed);
    if (p.E == 0 || p.K <= 0) return;
    const uint32_t* in = scores + (size_t)row * cap;
    const Pivot v = LevelBins(ws.hist + (size_t)row * 3 * kBins, 3, tid).find(3, p.K, pick, wsum, tid, lane, wave);
    const uint32_t T = v.key, least = v.ties ? T + 1 : T;  // (T is below the keys' last value)
    uint64_t* const above = ws.bits + (size_t)row * 2 * ws.words;
    uint64_t* const equal = above + ws.words;
    int from, to;
    part_range(p, n_fixed, part, parts, from, to);
    uint4 n = make_uint4(0, 0, 0, 0);
    constexpr int kWide = 8;  // words in flight a wavefront
    for (int e0 = from + 64 * kWide * wave; e0 < to; e0 += 64 * kWide * kSplitWaves) {
        uint32_t k[kWide];
#pragma unroll
        for (int i = 0; i < kWide; ++i) k[i] = in[imin(e0 + 64 * i + lane, p.D - 1)];
#pragma unroll
        for (int i = 0; i < kWide; ++i) {
            const int e = e0 + 64 * i + lane;
            k[i] = e >= n_fixed && e < to ? score_key(k[i]) : 0;
        }
#pragma unroll
        for (int i = 0; i < kWide; ++i) {
            const int e = e0 + 64 * i;
            const uint64_t ma = __builtin_amdgcn_ballot_w64(k[i] >= least);
            const uint64_t me = v.ties ? __builtin_amdgcn_ballot_w64(k[i] == T) : 0;
            if (lane == 0 && e < to) {
                above[e >> 6] = ma;
                equal[e >> 6] = me;
            }
            const int nl = imin(imax(p.left - e, 0), 64);  // tokens of the word below `left`
            const uint64_t low = nl == 64 ? ~0ull : (1ull << nl) - 1;
            n.x += __builtin_popcountll(ma & low);
            n.y += __builtin_popcountll(me & low);
            n.z += __builtin_popcountll(ma & ~low);
            n.w += __builtin_popcountll(me & ~low);
        }
    }
    if (lane == 0) sums[wave] = n;
    __syncthreads();
    if (tid == 0) {
        uint4 t = make_uint4(0, 0, 0, 0);
        for (int i = 0; i < kSplitWaves; ++i) {
            t.x += sums[i].x;
            t.y += sums[i].y;
            t.z += sums[i].z;
            t.w += sums[i].w;
        }
        ws.counts[(size_t)row * kMaxParts + part] = t;
    }
}

__global__ __launch_bounds__(kSplitThreads) void evict_lists_kernel(
    SplitWs ws, int2* __restrict__ info, int* holes, int* tails, int stride, int Hkv, int w, int cap,
    int len_arg, const int* __restrict__ lens, int n_keep, int n_fixed, int parts) {
    __shared__ uint32_t wsum[kSplitWaves];
    __shared__ uint32_t pick[3];
    const int part = wg_id_x(), row = wg_id_y(), b = row / Hkv;
    const int tid = lane_id_x(), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const RowPlan p = row_plan(lens ? lens[b] : len_arg, cap, w, n_keep, n_fixed);
    if (p.E == 0 || p.K <= 0) {
        if (part == 0 && tid == 0) info[row] = make_int2(0, p.E);
        return;
    }
    const uint4 none = make_uint4(0, 0, 0, 0);
    const uint4 c = lane < parts ? ws.counts[(size_t)row * kMaxParts + lane] : none;
    const Pivot v = LevelBins(ws.hist + (size_t)row * 3 * kBins, 3, tid).find(3, p.K, pick, wsum, tid, lane, wave);
    const uint32_t take = v.ties ? v.want : 0;  // tied tokens that stay: the first so many
    // sums over the wavefront's lanes, the parts
    auto total = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)wave_prefix(x), 63); };
    const bool in_front = lane < part;
    const uint32_t tied_low = total(c.y);
    const uint32_t kept_low = total(c.x) + (tied_low < take ? tied_low : take);
    uint32_t equal = total(in_front ? c.y + c.w : 0);
    uint32_t kept = total(in_front ? c.x + c.z : 0) + (equal < take ? equal : take);
    if (part == 0 && tid == 0) info[row] = make_int2(p.K - (int)kept_low, p.E);
    const uint64_t* const above_bits = ws.bits + (size_t)row * 2 * ws.words;
    const uint64_t* const equal_bits = above_bits + ws.words;
    int from, to;
    part_range(p, n_fixed, part, parts, from, to);
    // a thread a word, the words spread evenly over the wavefronts
    const int words = (to - from + 63) >> 6;
    const int per = imin((words + kSplitWaves - 1) / kSplitWaves, 64);
    for (int c0 = from; c0 < to; c0 += 64 * per * kSplitWaves) {
        const int w0 = c0 + 64 * per * wave, e0 = w0 + 64 * lane;
        const bool on = lane < per && e0 < to;
        uint64_t mine = on ? above_bits[e0 >> 6] : 0;
        uint32_t sum;
        if (take > 0) {
            uint64_t me = on ? equal_bits[e0 >> 6] : 0;
            const uint32_t before = equal + group_scan<kSplitWaves>(__builtin_popcountll(me), sum, wsum, lane, wave);
            equal += sum;
            for (uint32_t t = before < take ? take - before : 0; t > 0 && me; --t) {
                mine |= me & -me;
                me &= me - 1;
            }
        }
        const uint32_t kb = kept + group_scan<kSplitWaves>(__builtin_popcountll(mine), sum, wsum, lane, wave);
        kept += sum;
        // bits of a word's tokens before token x
        auto below = [&](int x) -> uint64_t {
            const int n = imin(imax(x - e0, 0), 64);
            return n == 64 ? ~0ull : (1ull << n) - 1;
        };
        const uint64_t low = below(p.left);
        write_list(holes + (size_t)row * stride, on ? ~mine & low & ~below(n_fixed) : 0,
                   imax(e0 - n_fixed, 0) - (int)kb, w0, lane);
        write_list(tails + (size_t)row * stride, on ? mine & ~low : 0,
                   e0 >= p.left ? (int)(kb - kept_low) : 0, w0, lane);
    }
}

// Entries past `left`, after the moves (which have taken E off lens).
__global__ __launch_bounds__(kSplitThreads) void evict_shift_kernel(
    const uint32_t* scores, uint32_t* scores_out, const int2* __restrict__ info, int Hkv, int w, int cap,
    int len_arg, const int* __restrict__ lens, int n_keep, int n_fixed, int parts) {
    const int row = wg_id_y(), b = row / Hkv, E = info[row].y;
    if (E == 0) return;
    const RowPlan p = row_plan(lens ? lens[b] + E : len_arg, cap, w, n_keep, n_fixed);
    shift_scores(scores + (size_t)row * cap, scores_out + (size_t)row * cap, p,
                 wg_id_x() * kSplitThreads + lane_id_x(), parts * kSplitThreads);
}

// The moves of one row, parts of them spread over the grid's x; scores (NULL:
// already moved) with them.
template <typename U>
__global__ __launch_bounds__(256) void evict_move_kernel(U* k_lat, U* v_lat,
                                                         const int2* __restrict__ info,
                                                         const int* __restrict__ holes,
                                                         const int* __restrict__ tails, int stride,
                                                         int Hkv, int ru, LatRows lat, int* lens,
                                                         const uint32_t* scores, uint32_t* scores_out,
                                                         int cap, int parts) {
    const int row = wg_id_y(), b = row / Hkv, g = row - b * Hkv;
    const int2 inf = info[row];
    // the sequence's length: nothing in this launch reads it
    if (lens && g == 0 && wg_id_x() == 0 && lane_id_x() == 0 && inf.y > 0) lens[b] -= inf.y;
    const int *from = tails + (size_t)row * stride, *to = holes + (size_t)row * stride;
    if (scores)
        move_scores(scores + (size_t)row * cap, scores_out + (size_t)row * cap, from, to, inf.x,
                    wg_id_x() * 256 + lane_id_x(), parts * 256);
    move_share(k_lat, v_lat, lat, b, g, from, to, inf.x, ru, lane_id_x(), 256, wg_id_x(), parts);
}

// lens[b] -= E of sequence b (the selection made the moves itself).
__global__ __launch_bounds__(256) void evict_lens_kernel(int* lens, int B, int cap, int w, int n_keep) {
    const int b = wg_id_x() * 256 + lane_id_x();
    if (b < B) lens[b] -= row_plan(lens[b], cap, w, n_keep, 0).E;
}

// Moves of one row, at most: the evicted tokens, and the kept ones.
static int evict_max_moves(int cap, int w, int n_keep) {
    const long long over = (long long)cap - w - n_keep;
    if (over <= 0) return 0;
    const long long kept = (long long)n_keep + (w > 0 ? w - 1 : 0);
    return (int)(over < kept ? over : kept);
}

// Words of the tokens of a cache that may hold rows too long for LDS (0: none).
static int split_words(int cap, int w) { return cap - w > kKeysLong ? (cap + 63) / 64 : 0; }

// The workspace: for long rows the parts' counts, the words and the histograms;
// the results, the lists.
size_t evict_workspace(int B, int Hkv, int cap, int w, int n_keep) {
    const size_t rows = (size_t)B * Hkv, words = split_words(cap, w);
    const size_t split = words ? kMaxParts * sizeof(uint4) + 2 * words * sizeof(uint64_t) + 3 * kBins * sizeof(uint32_t) : 0;
    return rows * (split + sizeof(int2) + 2 * sizeof(int) * (size_t)evict_max_moves(cap, w, n_keep));
}

template <typename U>
static hipError_t launch_evict_u(const uint32_t* scores, uint32_t* scores_out, U* k_lat, U* v_lat,
                                 void* ws, int B, int Hkv, int ru, int w, int cap, int len, int n_keep,
                                 int n_fixed, const LatRows& lat, int* lens, hipStream_t st) {
    const int rows = B * Hkv;
    const int stride = evict_max_moves(cap, w, n_keep);
    SplitWs sw{};
    char* at = (char*)ws;
    if (const int words = split_words(cap, w)) {
        sw.words = words;
        sw.counts = (uint4*)at;
        at += (size_t)rows * kMaxParts * sizeof(uint4);
        sw.hist = (uint32_t*)at;
        at += (size_t)rows * 3 * kBins * sizeof(uint32_t);
        sw.bits = (uint64_t*)at;
        at += (size_t)rows * 2 * words * sizeof(uint64_t);
    }
    int2* info = (int2*)at;
    int* holes = (int*)(info + rows);
    int* tails = holes + (size_t)rows * stride;
    // candidates of the longest row, and the lists that then fit LDS
    const int most = (lens ? cap : len) - w - (n_fixed & ~3);
    const bool split = most > kKeysLong;
    const int room = (most <= kKeysShort ? kKeysShort * 4 : kKeysLong * 4) / 8;
    // The selecting workgroups make the moves themselves where the lists fit and
    // either the moves are few or the rows alike (dense) and at least half as many
    // as compute units: one launch less, and no list goes through memory. Us a
    // call, moves by the selection and by the move kernel, d_down 16 bf16:
    //   2 x 8 rows, 20000 tokens, lists of 1500 slots 19.1 and 23.3, of 2600 27.6 and
    //   29.2, of 5000 36.5 and 34.5; paged 25.5 and 26.6, 39.7 and 33.7, 50.9 and 38.2;
    //   dense, 16384 tokens cut to half: 16 rows 36.7 and 31.7, 64 45.6 and 46.4, 128
    //   58.1 and 68.2, 248 91.9 and 102, 512 173 and 193; 30000 tokens: 64 rows 73.3
    //   and 68.4, 256 169 and 175;
    //   paged, all of 16384 tokens: 64 rows 59 and 49, 128 72 and 71, 256 106 and 109;
    //   2K to 32K tokens cut to 8K: 93 and 79, the longest rows last.
    const bool fused = !split && stride <= room && ((rows >= 128 && !lens) || stride <= 2048);
#define DAR_SELECT(K_, F_)                                                                         \
    hipLaunchKernelGGL((evict_select_kernel<K_, F_, U>), dim3(rows), dim3(kSelThreads), 0, st,     \
                       scores, scores_out, info, holes, tails, stride, Hkv, w, cap, len, lens,     \
                       n_keep, n_fixed, k_lat, v_lat, ru, lat)
#define DAR_SELECT_F(K_)              \
    if (fused) DAR_SELECT(K_, true);  \
    else DAR_SELECT(K_, false);
    // workgroups of a long row: about four a compute unit in all, which run at once
    // (64 rows of 131072 tokens: 2, 4 and 8 gave 238, 234 and 253 us a call)
    const int longest = lens ? cap : len;
    int parts = (1024 + rows - 1) / rows;
    if (parts > longest / kMinPart) parts = longest / kMinPart;
    parts = parts > kMaxParts ? kMaxParts : parts < 1 ? 1 : parts;
    if (split) {
        const dim3 grid(parts, rows), block(kSplitThreads);
        const int n4 = rows * (3 * kBins / 4);
        hipLaunchKernelGGL(evict_clear_kernel, dim3((n4 + 255) / 256), dim3(256), 0, st, (uint4*)sw.hist, n4);
        for (int level = 0; level < 3; ++level)
            hipLaunchKernelGGL(evict_count_kernel, grid, block, 0, st, scores, scores_out, sw, Hkv, w, cap,
                               len, lens, n_keep, n_fixed, level, parts);
        hipLaunchKernelGGL(evict_words_kernel, grid, block, 0, st, scores, sw, Hkv, w, cap, len, lens,
                           n_keep, n_fixed, parts);
        hipLaunchKernelGGL(evict_lists_kernel, grid, block, 0, st, sw, info, holes, tails, stride, Hkv, w,
                           cap, len, lens, n_keep, n_fixed, parts);
    } else if (most <= kKeysShort) { DAR_SELECT_F(kKeysShort) }
    else { DAR_SELECT_F(kKeysLong) }
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
    nb = nb > fill ? fill : nb < 1 ? 1 : nb;
    hipLaunchKernelGGL((evict_move_kernel<U>), dim3((unsigned)nb, rows), dim3(256), 0, st, k_lat, v_lat,
                       info, holes, tails, stride, Hkv, ru, lat, lens, split ? scores : nullptr,
                       scores_out, cap, (int)nb);
    if (split)
        hipLaunchKernelGGL(evict_shift_kernel, dim3(parts, rows), dim3(kSplitThreads), 0, st, scores,
                           scores_out, info, Hkv, w, cap, len, lens, n_keep, n_fixed, parts);
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
