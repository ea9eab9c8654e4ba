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
//   order is the scores' order, read once into registers (rows longer than
//   kMaxIter 16-byte loads a thread are read again, from the caches, at each
//   pass). The K-th largest key is found by histograms over ever narrower key
//   ranges: 8192 bins of the range that holds it, at most three levels of
//   32-bit keys, usually two (a bin whose keys all stay ends the search). A last
//   pass in slot order counts kept tokens in front of each token, which gives
//   every hole and tail its rank: with kb(e) kept candidates below slot e, hole
//   e has rank e - n_fixed - kb(e) and tail e has rank kb(e) - kb(left).
//   Few moves (kListLds at most) are made by the same workgroup from lists in
//   LDS; else it leaves the lists in the workspace for
// evict_move_kernel, which copies the latents along them on the whole chip.
#include "../../include/dar_serving.h"
#include "dar_common.hpp"
#include "dar_kernels.hpp"

namespace dar {

namespace {

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kBinBits = 13, kBins = 1 << kBinBits;
constexpr int kBinsPer = kBins / kSelThreads;
constexpr int kListLds = kBins / 2;  // moves whose lists take the histogram's place
constexpr int kMaxIter = 16;         // 16-byte loads of keys a thread keeps (64 registers)

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

// Part c of the latent rows (each of ru parts) of one move, key and value.
template <typename U>
__device__ __forceinline__ void move_part(U* lat, const LatRows& rows, int b, int g, int from, int to,
                                          int c, int ru) {
    const long long rf = rows.at(b, g, from), rt = rows.at(b, g, to);
    U x{};
    if (rf >= 0) x = lat[rf * ru + c];
    if (rt >= 0) lat[rt * ru + c] = x;
}

// info[row] = {moves, E}; lists holes[row * stride + r], tails[row * stride + r]
// (FUSED: not written; the moves are made here, U-sized parts, ru a latent row).
// ITER: 16-byte loads that hold a thread's share of the row (0: not held).
template <int ITER, bool FUSED, typename U>
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(
    const uint32_t* scores, uint32_t* scores_out, int2* __restrict__ info, int* holes, int* tails,
    int stride, int Hkv, int w, int cap, int len_arg, const int* __restrict__ lens, int n_keep,
    int n_fixed, U* k_lat, U* v_lat, int ru, LatRows lat) {
    __shared__ __attribute__((aligned(16))) uint32_t hist[kBins];
    __shared__ uint32_t wsum[kSelWaves];
    __shared__ uint32_t pick[3];            // bin, keys above it, keys in it
    __shared__ uint32_t cnt[4][kSelWaves];  // above T and equal to it: all, below `left`
    const int row = wg_id_x(), b = row / Hkv;
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
    int* const lh = FUSED ? (int*)hist : holes + (size_t)row * stride;
    int* const lt = FUSED ? (int*)hist + kListLds : tails + (size_t)row * stride;
    int moves = 0;
    if (p.K > 0) {
        // Candidates n_fixed..D-1 in groups of four; wave v takes `per` times 64
        // consecutive groups, so that ranks need one exchange between waves.
        const int a0 = n_fixed & ~3, n = p.D - n_fixed;
        const int per = (((p.D - a0 + 3) >> 2) + kSelThreads - 1) / kSelThreads;
        const int e_lane = a0 + ((wave * per) << 8) + (lane << 2);  // + 256 it
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
        auto candidate = [&](int e) -> bool { return (uint32_t)(e - n_fixed) < (uint32_t)n; };
        uint4 key[ITER > 0 ? ITER : 1];
        // f(e, four keys) for every group of this lane, in slot order
        auto visit = [&](auto&& f) {
            if constexpr (ITER > 0) {
#pragma unroll
                for (int it = 0; it < ITER; ++it)
                    if (it < per) f(e_lane + 256 * it, key[it]);
            } else {
                for (int i0 = 0; i0 < per; i0 += 4) {
                    uint4 u[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) u[i] = i0 + i < per ? fetch(e_lane + 256 * (i0 + i)) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i0 + i < per)
                            f(e_lane + 256 * (i0 + i), make_uint4(score_key(u[i].x), score_key(u[i].y),
                                                                  score_key(u[i].z), score_key(u[i].w)));
                }
            }
        };
        // scores below `left` to their places (holes are filled below)
        auto pass_on = [&](int e, const uint4& u) {
            if (!copy || e >= p.left) return;
            if (vec && e >= n_fixed && e + 3 < p.left) {
                *reinterpret_cast<uint4*>(out + e) = u;
            } else {
                const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (e + j >= n_fixed && e + j < p.left) out[e + j] = x[j];
            }
        };
        if constexpr (ITER > 0) {
#pragma unroll
            for (int it = 0; it < ITER; ++it) key[it] = it < per ? fetch(e_lane + 256 * it) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int it = 0; it < ITER; ++it) {
                if (it < per) pass_on(e_lane + 256 * it, key[it]);
                key[it] = make_uint4(score_key(key[it].x), score_key(key[it].y), score_key(key[it].z),
                                     score_key(key[it].w));
            }
        } else if (copy) {
            for (int i0 = 0; i0 < per; i0 += 4) {
                uint4 u[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = i0 + i < per ? fetch(e_lane + 256 * (i0 + i)) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i0 + i < per) pass_on(e_lane + 256 * (i0 + i), u[i]);
            }
        }
        // ---- the K-th largest key, and how many tokens equal to it stay
        uint32_t lo = 0, hi = 0xffffffffu;  // it lies in [lo, hi]
        uint32_t want = (uint32_t)p.K;      // its rank from the top among the keys in [lo, hi]
        bool ties;                          // of the keys equal to lo only `want` stay
        for (;;) {
            const uint32_t span = hi - lo;
            const int bits = span ? 32 - __builtin_clz(span) : 0;
            const int sh = bits > kBinBits ? bits - kBinBits : 0;
#pragma unroll
            for (int i = 0; i < kBinsPer / 4; ++i)
                reinterpret_cast<uint4*>(hist)[tid + kSelThreads * i] = make_uint4(0, 0, 0, 0);
            __syncthreads();
            visit([&](int e, const uint4& k) {
                const uint32_t x[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (candidate(e + j) && x[j] - lo <= span) atomicAdd(&hist[(x[j] - lo) >> sh], 1u);
            });
            __syncthreads();
            // thread t: kBinsPer bins from the top, thread 0 the highest
            uint32_t c[kBinsPer];
            const int b0 = kBins - kBinsPer * (tid + 1);
            uint32_t inc = 0;
#pragma unroll
            for (int i = 0; i < kBinsPer / 4; ++i) {
                const uint4 u = *reinterpret_cast<const uint4*>(hist + b0 + 4 * i);
                c[4 * i] = u.x; c[4 * i + 1] = u.y; c[4 * i + 2] = u.z; c[4 * i + 3] = u.w;
                inc += u.x + u.y + u.z + u.w;
            }
            const uint32_t mine = inc;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const uint32_t t = __shfl_up(inc, off, 64);
                if (lane >= off) inc += t;
            }
            if (lane == 63) wsum[wave] = inc;
            __syncthreads();
            uint32_t above = inc - mine;
            for (int v = 0; v < wave; ++v) above += wsum[v];
            if (want > above && want <= above + mine) {
#pragma unroll
                for (int i = kBinsPer - 1; i >= 0; --i) {
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
            hi = lo + ((1u << sh) - 1u);
            want -= pick[1];
            ties = want != pick[2];
            __syncthreads();
            if (sh == 0 || !ties) break;
        }
        const uint32_t T = lo;
        // ---- kept tokens in slot order. Without ties every key >= T stays; else
        // of the keys equal to T the first `want`.
        uint32_t gt = 0, eq = 0, gt_low = 0, eq_low = 0;
        visit([&](int e, const uint4& k) {
            const uint32_t x[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in_r = candidate(e + j), low = e + j < p.left;
                const bool a = in_r && (ties ? x[j] > T : x[j] >= T);
                gt += a;
                gt_low += a && low;
                if (ties) {
                    const bool q = in_r && x[j] == T;
                    eq += q;
                    eq_low += q && low;
                }
            }
        });
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) {
            gt += __shfl_xor(gt, off, 64);
            gt_low += __shfl_xor(gt_low, off, 64);
            if (ties) {
                eq += __shfl_xor(eq, off, 64);
                eq_low += __shfl_xor(eq_low, off, 64);
            }
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
        visit([&](int e, const uint4& k) {
            const uint32_t x[4] = {k.x, k.y, k.z, k.w};
            uint32_t g_here = gt_b, e_here = eq_b;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint64_t mg = __builtin_amdgcn_ballot_w64(candidate(e + j) && (ties ? x[j] > T : x[j] >= T));
                g_here += __builtin_amdgcn_mbcnt_hi((uint32_t)(mg >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mg, 0));
                gt_b += __builtin_popcountll(mg);
                if (ties) {
                    const uint64_t me = __builtin_amdgcn_ballot_w64(candidate(e + j) && x[j] == T);
                    e_here += __builtin_amdgcn_mbcnt_hi((uint32_t)(me >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)me, 0));
                    eq_b += __builtin_popcountll(me);
                }
            }
            // (g_here, e_here: before this lane's group; its own follow in order)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool a = ties ? x[j] > T : x[j] >= T;
                const bool q = ties && x[j] == T;
                const bool kept = a || (q && e_here < want);
                const int kb = (int)(g_here + (e_here < want ? e_here : want));
                if (candidate(e + j)) {
                    if (e + j < p.left) {
                        if (!kept) lh[e + j - n_fixed - kb] = e + j;
                    } else if (kept) {
                        lt[kb - (int)kept_low] = e + j;
                    }
                    g_here += a;
                    e_here += q;
                }
            }
        });
    }
    __syncthreads();  // the lists are complete, and `out` below `left` but for the holes
    for (int r = tid; r < moves; r += kSelThreads) out[lh[r]] = in[lt[r]];
    if constexpr (FUSED) {
        const int g = row - b * Hkv, parts = moves * 2 * ru;
        for (int t = tid; t < parts; t += kSelThreads) {
            const int r = t / (2 * ru), c = t - r * (2 * ru);
            move_part(c < ru ? k_lat : v_lat, lat, b, g, lt[r], lh[r], c < ru ? c : c - ru, ru);
        }
    }
    __syncthreads();  // tails are read before entries past `left` change
    // E >= w: the window's entries move to a range that does not meet their own
    const int near = p.len - p.D;
    for (int i = tid; i < near; i += kSelThreads) out[p.left + i] = in[p.D + i];
    __syncthreads();
    for (int e = p.len - p.E + tid; e < p.len; e += kSelThreads) out[e] = 0;
    if (!FUSED && tid == 0) info[row] = make_int2(moves, p.E);
}

// The moves of one row, parts of them spread over the grid's x.
template <typename U>
__global__ __launch_bounds__(256) void evict_move_kernel(U* k_lat, U* v_lat,
                                                         const int2* __restrict__ info,
                                                         const int* __restrict__ holes,
                                                         const int* __restrict__ tails, int stride,
                                                         int Hkv, int ru, LatRows lat, int* lens) {
    const int row = wg_id_y(), b = row / Hkv, g = row - b * Hkv;
    const int2 inf = info[row];
    // the sequence's length: nothing in this launch reads it
    if (lens && g == 0 && wg_id_x() == 0 && lane_id_x() == 0 && inf.y > 0) lens[b] -= inf.y;
    const int* lh = holes + (size_t)row * stride;
    const int* lt = tails + (size_t)row * stride;
    const int lanes = 2 * ru, per = 256 / lanes;  // moves of a workgroup at a time
    if (per == 0) {                               // (rows of more than 128 parts)
        for (int r = wg_id_x(); r < inf.x; r += (int)(__builtin_amdgcn_grid_size_x() >> 8))
            for (int c = lane_id_x(); c < lanes; c += 256)
                move_part(c < ru ? k_lat : v_lat, lat, b, g, lt[r], lh[r], c < ru ? c : c - ru, ru);
        return;
    }
    const int sub = lane_id_x() / lanes, c = lane_id_x() - sub * lanes;
    if (sub >= per) return;
    U* a = c < ru ? k_lat : v_lat;
    const int cc = c < ru ? c : c - ru;
    const int step = per * (int)(__builtin_amdgcn_grid_size_x() >> 8);
    constexpr int kFlight = 4;  // moves in flight a thread
    for (int r0 = wg_id_x() * per + sub; r0 < inf.x; r0 += kFlight * step) {
        long long rt[kFlight];
        U x[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int r = r0 + i * step;
            rt[i] = -1;
            x[i] = U{};
            if (r < inf.x) {
                const long long rf = lat.at(b, g, lt[r]);
                rt[i] = lat.at(b, g, lh[r]);
                if (rf >= 0) x[i] = a[rf * ru + cc];
            }
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
            if (rt[i] >= 0) a[rt[i] * ru + cc] = x[i];
    }
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
    const bool fused = stride <= kListLds;
    // candidates of the longest row, in groups a thread
    const int most = (lens ? cap : len) - w - (n_fixed & ~3);
    const int per = most <= 0 ? 1 : (((most + 3) >> 2) + kSelThreads - 1) / kSelThreads;
#define DAR_SELECT(IT_, F_)                                                                        \
    hipLaunchKernelGGL((evict_select_kernel<IT_, F_, U>), dim3(rows), dim3(kSelThreads), 0, st,    \
                       scores, scores_out, info, holes, tails, stride, Hkv, w, cap, len, lens,     \
                       n_keep, n_fixed, k_lat, v_lat, ru, lat)
#define DAR_SELECT_F(IT_)              \
    if (fused) DAR_SELECT(IT_, true);  \
    else DAR_SELECT(IT_, false);
    if (per <= 2) { DAR_SELECT_F(2) }
    else if (per <= 5) { DAR_SELECT_F(5) }
    else if (per <= 9) { DAR_SELECT_F(9) }
    else if (per <= kMaxIter) { DAR_SELECT_F(kMaxIter) }
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
    long long nb = ((long long)stride * 2 * ru + 1023) / 1024;
    const long long fill = (32 * 256 + rows - 1) / rows;  // about 32 workgroups a compute unit
    nb = nb > fill ? fill : nb;
    hipLaunchKernelGGL((evict_move_kernel<U>), dim3((unsigned)nb, rows), dim3(256), 0, st, k_lat, v_lat,
                       info, holes, tails, stride, Hkv, ru, lat, lens);
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
        return launch_evict_u(in, out, (uint4*)k_lat, (uint4*)v_lat, ws, B, Hkv, row_bytes / 16, w, cap,
                              len, n_keep, n_fixed, lat, lens, st);
    if (esize == 4)
        return launch_evict_u(in, out, (uint32_t*)k_lat, (uint32_t*)v_lat, ws, B, Hkv, row_bytes / 4, w,
                              cap, len, n_keep, n_fixed, lat, lens, st);
    return launch_evict_u(in, out, (uint16_t*)k_lat, (uint16_t*)v_lat, ws, B, Hkv, row_bytes / 2, w, cap,
                          len, n_keep, n_fixed, lat, lens, st);
}

}  // namespace dar
