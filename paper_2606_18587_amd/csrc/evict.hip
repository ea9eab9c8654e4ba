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
//   order is the scores' order; the K-th largest key is found by histograms
//   over ever narrower key ranges (2048 bins of the range that holds it, at
//   most three levels of 32-bit keys). A last pass in slot order counts kept
//   tokens in front of each token, which gives every hole and tail its rank:
//   with kb(e) kept candidates below slot e, hole e has rank e - n_fixed -
//   kb(e) and tail e has rank kb(e) - kb(left). It writes the lists and the
//   scores.
// evict_move_kernel: copies the latents along the lists.
#include "../../include/dar_serving.h"
#include "dar_common.hpp"
#include "dar_kernels.hpp"

namespace dar {

namespace {

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kBinBits = 11, kBins = 1 << kBinBits;

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

// Keys in the order of the scores: NaN 0, then -inf .. -0 = 0 .. inf.
// (On the bits: the build assumes that floating-point values are no NaN.)
__device__ __forceinline__ uint32_t score_key(uint32_t u) {
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
    if (u == 0x80000000u) u = 0;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

}  // namespace

// Moves and per-row results in the workspace: info[row] = {moves, E}, then the
// lists holes[row * stride + r], tails[row * stride + r].
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(
    const uint32_t* scores, uint32_t* scores_out, int2* __restrict__ info, int* __restrict__ holes,
    int* __restrict__ tails, int stride, int Hkv, int w, int cap, int len_arg,
    const int* __restrict__ lens, int n_keep, int n_fixed) {
    __shared__ uint32_t hist[kBins];
    __shared__ uint32_t wsum[kSelWaves];
    __shared__ uint32_t pick[4];          // bin, keys above it, keys in it
    __shared__ uint32_t cnt[4][kSelWaves];  // kept-above and equal: all, below `left`
    const int row = wg_id_x(), b = row / Hkv;
    const int tid = lane_id_x(), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const RowPlan p = row_plan(lens ? lens[b] : len_arg, cap, w, n_keep, n_fixed);
    const uint32_t* in = scores + (size_t)row * cap;
    uint32_t* out = scores_out + (size_t)row * cap;
    const bool copy = scores != scores_out;
    if (p.E == 0) {
        if (tid == 0) info[row] = make_int2(0, 0);
        if (copy)
            for (int e = tid; e < p.len; e += kSelThreads) out[e] = in[e];
        return;
    }
    int moves = 0;
    if (p.K > 0) {
        // ---- the K-th largest key, and how many tokens equal to it stay
        uint32_t lo = 0, hi = 0xffffffffu;  // it lies in [lo, hi]
        uint32_t want = (uint32_t)p.K;      // its rank from the top among the keys in [lo, hi]
        uint32_t equal = 0;                 // keys in [lo, hi]
        for (;;) {
            const uint32_t span = hi - lo;
            const int bits = span ? 32 - __builtin_clz(span) : 0;
            const int sh = bits > kBinBits ? bits - kBinBits : 0;
            for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
            __syncthreads();
            for (int e = n_fixed + tid; e < p.D; e += kSelThreads) {
                const uint32_t k = score_key(in[e]);
                if (k >= lo && k <= hi) atomicAdd(&hist[(k - lo) >> sh], 1u);
            }
            __syncthreads();
            // thread t: bins 2 t' and 2 t' + 1 from the top, t' = kSelThreads - 1 - t
            const int b1 = kBins - 1 - 2 * tid, b0 = b1 - 1;
            const uint32_t c1 = hist[b1], c0 = hist[b0];
            uint32_t inc = c1 + c0;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const uint32_t t = __shfl_up(inc, off, 64);
                if (lane >= off) inc += t;
            }
            if (lane == 63) wsum[wave] = inc;
            __syncthreads();
            uint32_t above = inc - (c1 + c0);
            for (int v = 0; v < wave; ++v) above += wsum[v];
            if (want > above && want <= above + c1) {
                pick[0] = b1;
                pick[1] = above;
                pick[2] = c1;
            } else if (want > above + c1 && want <= above + c1 + c0) {
                pick[0] = b0;
                pick[1] = above + c1;
                pick[2] = c0;
            }
            __syncthreads();
            lo += pick[0] << sh;
            hi = lo + ((1u << sh) - 1u);
            want -= pick[1];
            equal = pick[2];
            __syncthreads();
            if (sh == 0) break;
        }
        const uint32_t T = lo;  // want of the `equal` keys equal to T stay
        (void)equal;
        // ---- kept tokens in slot order: wave v takes a contiguous share
        const int n = p.D - n_fixed;
        const int share = ((n + kSelWaves - 1) / kSelWaves + 63) & ~63;
        const int e0 = n_fixed + wave * share, e1 = imin(e0 + share, p.D);
        uint32_t gt = 0, eq = 0, gt_low = 0, eq_low = 0;
        for (int eb = e0; eb < e1; eb += 64) {
            const int e = eb + lane;
            const uint32_t k = e < e1 ? score_key(in[e]) : 0;
            const uint64_t mg = __builtin_amdgcn_ballot_w64(e < e1 && k > T);
            const uint64_t me = __builtin_amdgcn_ballot_w64(e < e1 && k == T);
            const uint64_t ml = __builtin_amdgcn_ballot_w64(e < p.left);
            gt += __builtin_popcountll(mg);
            eq += __builtin_popcountll(me);
            gt_low += __builtin_popcountll(mg & ml);
            eq_low += __builtin_popcountll(me & ml);
        }
        if (lane == 0) {
            cnt[0][wave] = gt;
            cnt[1][wave] = eq;
            cnt[2][wave] = gt_low;
            cnt[3][wave] = eq_low;
        }
        __syncthreads();
        uint32_t gt_b = 0, eq_b = 0, gl = 0, el = 0;
        for (int v = 0; v < kSelWaves; ++v) {
            if (v < wave) {
                gt_b += cnt[0][v];
                eq_b += cnt[1][v];
            }
            gl += cnt[2][v];
            el += cnt[3][v];
        }
        const uint32_t kept_low = gl + (el < want ? el : want);  // kb(left)
        moves = p.K - (int)kept_low;
        const size_t lbase = (size_t)row * stride;
        for (int eb = e0; eb < e1; eb += 64) {
            const int e = eb + lane;
            const bool in_r = e < e1;
            const uint32_t u = in_r ? in[e] : 0;
            const uint32_t k = score_key(u);
            const uint64_t mg = __builtin_amdgcn_ballot_w64(in_r && k > T);
            const uint64_t me = __builtin_amdgcn_ballot_w64(in_r && k == T);
            const uint64_t below = (1ull << lane) - 1;
            const uint32_t g_here = gt_b + __builtin_popcountll(mg & below);
            const uint32_t e_here = eq_b + __builtin_popcountll(me & below);
            const int kb = (int)(g_here + (e_here < want ? e_here : want));
            const bool kept = k > T || (k == T && e_here < want);
            if (in_r) {
                if (e < p.left) {
                    if (!kept) holes[lbase + (e - n_fixed - kb)] = e;
                    else if (copy) out[e] = u;
                } else if (kept) {
                    tails[lbase + (kb - (int)kept_low)] = e;
                }
            }
            gt_b += __builtin_popcountll(mg);
            eq_b += __builtin_popcountll(me);
        }
    }
    if (copy)
        for (int e = tid; e < n_fixed; e += kSelThreads) out[e] = in[e];
    __syncthreads();  // the lists are complete (one workgroup: visible to it)
    const size_t lbase = (size_t)row * stride;
    for (int r = tid; r < moves; r += kSelThreads) out[holes[lbase + r]] = in[tails[lbase + r]];
    __syncthreads();  // tails are read before entries past `left` change
    // E >= w: the window's entries move to a range that does not meet their own
    const int near = p.len - p.D;
    for (int i = tid; i < near; i += kSelThreads) out[p.left + i] = in[p.D + i];
    __syncthreads();
    for (int e = p.len - p.E + tid; e < p.len; e += kSelThreads) out[e] = 0;
    if (tid == 0) info[row] = make_int2(moves, p.E);
}

// Piece t of a row's moves: one U-sized part of the key or value latent of one
// move. ru: such parts in a latent row.
template <typename U>
__global__ __launch_bounds__(256) void evict_move_kernel(U* k_lat, U* v_lat,
                                                         const int2* __restrict__ info,
                                                         const int* __restrict__ holes,
                                                         const int* __restrict__ tails, int stride,
                                                         int Hkv, int cap, int ru,
                                                         const int* __restrict__ bt, int maxb,
                                                         int n_pages, int ps_shift, int* lens) {
    const int row = wg_id_y(), b = row / Hkv, g = row - b * Hkv;
    const int2 inf = info[row];
    // the sequence's length: nothing in this launch reads it
    if (lens && g == 0 && wg_id_x() == 0 && lane_id_x() == 0 && inf.y > 0) lens[b] -= inf.y;
    const size_t lbase = (size_t)row * stride;
    const long long n = (long long)inf.x * 2 * ru;
    const int nthr = (int)__builtin_amdgcn_grid_size_x();
    for (long long t = (long long)wg_id_x() * 256 + lane_id_x(); t < n; t += nthr) {
        const int r = (int)(t / (2 * ru)), part = (int)(t - (long long)r * (2 * ru));
        const int from = tails[lbase + r], to = holes[lbase + r];
        U* lat = part < ru ? k_lat : v_lat;
        const int c = part < ru ? part : part - ru;
        if (bt == nullptr) {
            lat[((size_t)row * cap + to) * ru + c] = lat[((size_t)row * cap + from) * ru + c];
        } else {
            const int* btb = bt + (size_t)b * maxb;
            const int ps = 1 << ps_shift;
            const int pf = btb[from >> ps_shift], pt = btb[to >> ps_shift];
            if (pt < 0 || pt >= n_pages) continue;
            U x{};
            if (pf >= 0 && pf < n_pages)
                x = lat[(((size_t)pf * Hkv + g) * ps + (from & (ps - 1))) * ru + c];
            lat[(((size_t)pt * Hkv + g) * ps + (to & (ps - 1))) * ru + c] = x;
        }
    }
}

// Moves of one row, at most: the evicted tokens, and the kept ones.
int evict_max_moves(int cap, int w, int n_keep) {
    const long long over = (long long)cap - w - n_keep;
    if (over <= 0) return 0;
    const long long kept = (long long)n_keep + (w > 0 ? w - 1 : 0);
    return (int)(over < kept ? over : kept);
}

hipError_t launch_evict(const float* scores, float* scores_out, void* k_lat, void* v_lat, void* ws,
                        int B, int Hkv, int row_bytes, int esize, int w, int cap, int len,
                        int n_keep, int n_fixed, const PagedArgs* pg, int* lens, hipStream_t st) {
    const int rows = B * Hkv;
    const int stride = evict_max_moves(cap, w, n_keep);
    int2* info = (int2*)ws;
    int* holes = (int*)(info + rows);
    int* tails = holes + (size_t)rows * stride;
    hipLaunchKernelGGL(evict_select_kernel, dim3(rows), dim3(kSelThreads), 0, st,
                       (const uint32_t*)scores, (uint32_t*)scores_out, info, holes, tails, stride,
                       Hkv, w, cap, len, pg ? (const int*)lens : nullptr, n_keep, n_fixed);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int us = row_bytes % 16 == 0 ? 16 : esize;
    const int ru = row_bytes / us;
    const long long work = (long long)stride * 2 * ru;
    long long nb = (work + 255) / 256;
    const long long most = (16 * 256 + rows - 1) / rows;  // about 16 workgroups a compute unit
    nb = nb > most ? most : nb;
    nb = nb < 1 ? 1 : nb;
#define DAR_EVICT_MOVE(U_)                                                                       \
    hipLaunchKernelGGL((evict_move_kernel<U_>), dim3((unsigned)nb, rows), dim3(256), 0, st,      \
                       (U_*)k_lat, (U_*)v_lat, info, holes, tails, stride, Hkv, cap, ru,         \
                       pg ? pg->bt : nullptr, pg ? pg->maxb : 0, pg ? pg->n_pages : 0,           \
                       pg ? pg->ps_shift : 0, pg ? lens : nullptr)
    if (us == 16) DAR_EVICT_MOVE(uint4);
    else if (us == 4) DAR_EVICT_MOVE(uint32_t);
    else DAR_EVICT_MOVE(uint16_t);
#undef DAR_EVICT_MOVE
    return hipGetLastError();
}

}  // namespace dar
