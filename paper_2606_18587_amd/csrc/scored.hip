// Decode steps that score the cached tokens by the attention weight they
// receive (dar_attn_decode_scored, dar_attn_decode_paged_scored), and the
// merge of partial records that they share with the shared-prefix decode.
//
//   1. partial records of every part of the cache (decode_mfma.hip in its records
//      mode, scored_split_kernel for the shapes it does not take);
//   2. their merge under one maximum into the output, and the weights. These
//      need the softmax denominator, which is known after the last key, so every
//      key is met a second time: p = exp2(s - lse2), summed over the query heads
//      of the KV head and added to the token's score. Of the cache that reads the
//      key latents and the ring's keys, half of what step 1 reads. On the matrix
//      cores (decode_finish_kernel) both run in one launch; else
//      (records_join_kernel, decode_weights_kernel) one after the other.
#include "../../include/dar_serving.h"
#include "dar_common.hpp"
#include "dar_kernels.hpp"
#include "mfma_common.hpp"

namespace dar {

// Merge for any shape: records {m, l, acc_lat[dd], acc_win[d]} of (sequence,
// query head) bh at part + (bh * S + s) * (2 + dd + d).
// A wavefront per head. Its loads come in three groups, each independent within
// itself: the records' {m, l} and the first W_up rows, the records' sums, the
// rest of W_up; as many records side by side as their latent sums leave lanes
// for. NR: output columns per lane (d <= 64 NR).
constexpr int kJoinMax = 1024;  // records of a head, at most
constexpr int kJoinRegs = 32;        // W_up rows requested before the records

template <typename T, int NR>
__global__ __launch_bounds__(64) void records_join_kernel(
    const float* __restrict__ part, int n, const T* __restrict__ wd, const T* __restrict__ wu,
    T* __restrict__ o, float* __restrict__ lse2, int Hq, int Hkv, int d, int dd) {
    __shared__ float wsh[kJoinMax];  // the records' weights
    __shared__ float lsh[256];       // the merged latent sum
    const int bh = wg_id_x(), lane = lane_id_x();
    const int g = bh % Hq / (Hq / Hkv);
    const T* wdg = wd + (size_t)g * d * dd;
    const T* wug = wu ? wu + (size_t)g * dd * d : nullptr;
    auto up = [&](int c, int e) -> float {  // W_up[c][e]
        return wug ? elem<T>::load(wug + (size_t)c * d + e) : elem<T>::load(wdg + (size_t)e * dd + c);
    };
    float wcol[NR][kJoinRegs];
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int c = 0; c < kJoinRegs; ++c) wcol[r][c] = up(imin(c, dd - 1), imin(lane + 64 * r, d - 1));
    const int stride = 2 + dd + d;
    const float* own = part + (size_t)bh * n * stride;
    auto rec = [&](int s) { return own + (size_t)s * stride; };

    // weights w_s = 2^(m_s - M); two records a lane at once
    const float2 none = make_float2(-INFINITY, 0.f);
    auto ml = [&](int s) { const float* r = rec(s); return make_float2(r[0], r[1]); };
    const float2 r0 = lane < n ? ml(lane) : none, r1 = lane + 64 < n ? ml(lane + 64) : none;
    float M = fmaxf(r0.x, r1.x);
    for (int s = lane + 128; s < n; s += 64) M = fmaxf(M, rec(s)[0]);
    M = wave_max(M);
    float L = 0.f;
    auto weigh = [&](int s, float2 x) {
        const float ws = x.x == -INFINITY ? 0.f : exp2f(x.x - M);
        wsh[s] = ws;
        L = __builtin_fmaf(ws, x.y, L);
    };
    if (lane < n) weigh(lane, r0);
    if (lane + 64 < n) weigh(lane + 64, r1);
    for (int s = lane + 128; s < n; s += 64) weigh(s, ml(s));
    L = wave_sum(L);
    if (lane == 0) lse2[bh] = M + log2f(L);
    __syncthreads();

    // window sums: a lane owns columns lane + 64 r
    constexpr int kAhead = 8;
    float acc[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) acc[r] = 0.f;
    for (int s0 = 0; s0 < n; s0 += kAhead) {
        float x[kAhead][NR];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
#pragma unroll
            for (int r = 0; r < NR; ++r)
                x[j][r] = own[(size_t)imin(s0 + j, n - 1) * stride + 2 + dd + imin(lane + 64 * r, d - 1)];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const float ws = s0 + j < n ? wsh[s0 + j] : 0.f;
#pragma unroll
            for (int r = 0; r < NR; ++r) acc[r] = __builtin_fmaf(ws, x[j][r], acc[r]);
        }
    }
    // latent sums: lpr lanes a record, 64 / lpr records side by side
    for (int c0 = 0; c0 < dd; c0 += 64) {
        const int width = imin(dd - c0, 64);
        int lpr = 1;
        while (lpr < width) lpr <<= 1;
        const int c = lane & (lpr - 1), side = 64 / lpr;
        const int cc = c0 + imin(c, width - 1);
        float lat = 0.f;
        for (int s0 = lane / lpr; s0 < n; s0 += side * kAhead) {
            float x[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) x[j] = rec(imin(s0 + j * side, n - 1))[2 + cc];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                lat = __builtin_fmaf(s0 + j * side < n ? wsh[s0 + j * side] : 0.f, x[j], lat);
        }
        for (int off = lpr; off < 64; off <<= 1) lat += __shfl_xor(lat, off, 64);
        if (lane < width) lsh[c0 + lane] = lat;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < NR; ++r) {
#pragma unroll
        for (int c = 0; c < kJoinRegs; ++c)
            if (c < dd) acc[r] = __builtin_fmaf(lsh[c], wcol[r][c], acc[r]);
        const int e = lane + 64 * r;
        for (int c = kJoinRegs; c < dd; ++c) acc[r] = __builtin_fmaf(lsh[c], up(c, imin(e, d - 1)), acc[r]);
        if (e < d) o[(size_t)bh * d + e] = elem<T>::from_f32(acc[r] / L);
    }
}

namespace {

constexpr int kWThreads = 256, kWWaves = kWThreads / 64;
constexpr int kFinMaxGroup = 8;   // query heads per KV head on the matrix-core path
constexpr int kFinMaxRec = 320;   // records of a head: own (256 at most) and shared-prefix ones
constexpr int kRawWord3 = 0x00020000;  // raw buffer, 32-bit data: reads past its size are zero
typedef unsigned int wu32x4 __attribute__((ext_vector_type(4)));

// p rounded by nothing: the absorbed query as three bf16 operands (24 bits)
__device__ __forceinline__ void split3(const float* src, bool on, bf16x8_t (&p)[3]) {
    float v[8];
    const float4 a = *reinterpret_cast<const float4*>(src), c = *reinterpret_cast<const float4*>(src + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = c.x; v[5] = c.y; v[6] = c.z; v[7] = c.w;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = on ? v[j] : 0.f;
#pragma unroll
    for (int t = 0; t < 3; ++t) {
        uint32_t h[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            h[j] = pack2(v[2 * j], v[2 * j + 1]);
            v[2 * j] -= __uint_as_float(h[j] << 16);
            v[2 * j + 1] -= __uint_as_float(h[j] & 0xffff0000u);
        }
        p[t] = __builtin_bit_cast(bf16x8_t, make_uint4(h[0], h[1], h[2], h[3]));
    }
}

}  // namespace

// Second stage on the matrix cores (bf16, d in {64, 128}, d_down in {16, 32}) of
// one (sequence, KV head) y: the merge of its records (the first workgroups x), and, if
// scores are asked for, the weights (the others, dealt groups of 64 tokens).
// Both begin with the records' {m, l}: the denominators of the pair's heads.
//
// Merge: W_up passes through LDS, once for the G heads (2-byte loads of its
// columns by every head's wavefront took 7 of 13 us at 2048 heads).
//
// Weights: S = Q~ C^T with the query heads as rows and 32 tokens as columns, so
// that a lane holds all heads of one token and the sum over them stays in it.
// Rows 0..3 and 4..7 (lane halves) hold heads 0..3 twice, or (G8) heads 0..3 and
// 4..7; two subtiles at a time, so that lane l finishes token l of the 64. Bound
// by memory: 2 dd bytes of key latent and 8 of scores a token; the next group's
// loads are in flight under this one's products, through descriptors that end
// with the rows (no load on a branch).
template <int D, int DD, bool G8, bool PAGED>
__global__ __launch_bounds__(kWThreads) void decode_finish_kernel(
    const bf16_t* __restrict__ q, const bf16_t* __restrict__ wd, const bf16_t* __restrict__ wu,
    const float* __restrict__ part, int S_all, const float* __restrict__ ppart, int NS,
    const float* __restrict__ qt, const bf16_t* __restrict__ k_win,
    const bf16_t* __restrict__ k_lat, bf16_t* __restrict__ o, const float* scores,
    float* scores_out, int Hq, int Hkv, int w, int cap, int len_arg, PagedArgs pg, float qscale,
    int gw) {
    constexpr int KS = D / 16, DS = DD / 16, NR = D / 64;
    constexpr int stride = 2 + DD + D, pstride = 2 + DD;
    constexpr int kPer = 8;    // records side by side in the merge
    __shared__ float lse[kFinMaxGroup];
    __shared__ float wsh[kFinMaxGroup][kFinMaxRec];  // the records' weights, normalised
    __shared__ bf16_t ush[DD][D + 2];
    __shared__ float lsh[kWWaves][DD];
    const int bg = wg_id_y(), b = bg / Hkv, g = bg - b * Hkv;
    const int tid = lane_id_x(), lane = tid & 63, col = lane & 31, hg = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = Hq / Hkv;
    const size_t bh0 = (size_t)b * Hq + (size_t)g * G;
    const int nm = (G + kWWaves - 1) / kWWaves;  // workgroups of the merge, a wavefront a head
    const bool merge = wg_id_x() < nm;
    if (merge) {
        const bf16_t* src = wu ? wu + (size_t)g * DD * D : wd + (size_t)g * D * DD;
        for (int i = tid * 8; i < DD * D; i += kWThreads * 8) {
            const bf16x8_t x = load_bf16x8(src + i);
            const uint4 u = __builtin_bit_cast(uint4, x);
            const uint32_t w4[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bf16_t e = (bf16_t)(w4[j >> 1] >> (16 * (j & 1)));
                if (wu) ush[(i + j) / D][(i + j) & (D - 1)] = e;
                else ush[(i + j) & (DD - 1)][(i + j) / DD] = e;
            }
        }
    }
    int len = len_arg, S = S_all;
    if constexpr (PAGED) {
        len = pg.lens[b];
        if (len < 1) {  // empty or overflowed: no query position, NaN
            if (wg_id_x() == 0)
                for (int e = tid; e < G * D; e += kWThreads) o[bh0 * D + e] = 0x7fc0;
            return;
        }
        len = imin(len, cap);
        // (a sequence all of whose tokens are the prefix's has no part of its own, and
        // no count)
        S = w == 0 && (len + 31) / 32 <= pg.pre ? 0 : imin(S_all, pg.counts[bg]);
    }
    const int n = S + NS;
    auto rec = [&](int h, int s) {
        return s < S ? part + ((bh0 + h) * S_all + s) * stride : ppart + ((bh0 + h) * NS + s - S) * pstride;
    };
    // the denominators, a wavefront a head; the first 64 records stay in registers
    for (int h = wave; h < G; h += kWWaves) {
        if (merge && h / kWWaves != wg_id_x()) continue;
        const float* r = rec(h, imin(lane, n - 1));
        const float m0 = lane < n ? r[0] : -INFINITY, l0 = r[1];
        float M = m0;
        for (int s = lane + 64; s < n; s += 64) M = fmaxf(M, rec(h, s)[0]);
        M = wave_max(M);
        float L = m0 == -INFINITY ? 0.f : exp2f(m0 - M) * l0;
        for (int s = lane + 64; s < n; s += 64) {
            const float m = rec(h, s)[0];
            if (m != -INFINITY) L = __builtin_fmaf(exp2f(m - M), rec(h, s)[1], L);
        }
        L = wave_sum(L);
        const float lg = M + log2f(L);
        if (lane == 0) lse[h] = lg;
        if (merge) {
            const float inv = 1.f / L;
            if (lane < n) wsh[h][lane] = m0 == -INFINITY ? 0.f : exp2f(m0 - M) * inv;
            for (int s = lane + 64; s < n; s += 64) {
                const float m = rec(h, s)[0];
                wsh[h][s] = m == -INFINITY ? 0.f : exp2f(m - M) * inv;
            }
        }
    }
    __syncthreads();

    if (merge) {
        const int h = wg_id_x() * kWWaves + wave;
        if (h < G) {
            float acc[NR];
#pragma unroll
            for (int r = 0; r < NR; ++r) acc[r] = 0.f;
            for (int s0 = 0; s0 < S; s0 += kPer) {
                float x[kPer][NR];
#pragma unroll
                for (int j = 0; j < kPer; ++j)
#pragma unroll
                    for (int r = 0; r < NR; ++r) x[j][r] = rec(h, imin(s0 + j, S - 1))[2 + DD + lane + 64 * r];
#pragma unroll
                for (int j = 0; j < kPer; ++j)
#pragma unroll
                    for (int r = 0; r < NR; ++r)
                        acc[r] = __builtin_fmaf(s0 + j < S ? wsh[h][s0 + j] : 0.f, x[j][r], acc[r]);
            }
            // latent sums, 64 / DD records side by side
            constexpr int side = 64 / DD;
            const int c = lane & (DD - 1);
            float lat = 0.f;
            for (int s0 = lane / DD; s0 < n; s0 += side * kPer) {
                float x[kPer];
#pragma unroll
                for (int j = 0; j < kPer; ++j) x[j] = rec(h, imin(s0 + j * side, n - 1))[2 + c];
#pragma unroll
                for (int j = 0; j < kPer; ++j)
                    lat = __builtin_fmaf(s0 + j * side < n ? wsh[h][s0 + j * side] : 0.f, x[j], lat);
            }
#pragma unroll
            for (int off = DD; off < 64; off <<= 1) lat += __shfl_xor(lat, off, 64);
            if (lane < DD) lsh[wave][lane] = lat;
            wave_lds_order();
#pragma unroll
            for (int r = 0; r < NR; ++r) {
#pragma unroll
                for (int k = 0; k < DD; ++k)
                    acc[r] = __builtin_fmaf(lsh[wave][k], bf16_to_f32(ush[k][lane + 64 * r]), acc[r]);
                o[(bh0 + h) * D + lane + 64 * r] = f32_to_bf16(acc[r]);
            }
        }
        return;
    }

    // ---- the weights
    const int first = PAGED ? pg.first : 0;
    const int n_lat = imax(len - w, 0);
    const int ngl = (imax(n_lat - first, 0) + 63) >> 6, ngw = (len - n_lat + 63) >> 6;
    // (the grid's size is an argument: read from the dispatch packet, in host memory,
    // it takes microseconds to come)
    const int nw = gw * kWWaves;  // wavefronts of the weights
    const int idx0 = (wg_id_x() - nm) * kWWaves + wave;
    if (idx0 >= ngl + ngw) return;

    const int head = G8 ? col : (col & 3);  // A-operand row col
    const bool hval = col < 8 && head < G;
    float nl[4];  // -lse of the head in accumulator register r
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int h = G8 ? 4 * hg + r : r;
        nl[r] = -lse[h < G ? h : 0];
    }
    float* out = scores_out + (size_t)bg * cap;
    const float* in = scores + (size_t)bg * cap;
    // the weight of this lane's token from the scores of both subtiles
    auto weight = [&](const f32x16_t& xa, const f32x16_t& xb, float f) -> float {
        float sa = 0.f, sb = 0.f;
        if constexpr (G8) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                sa += __builtin_amdgcn_exp2f(__builtin_fmaf(xa[r], f, nl[r]));
                sb += __builtin_amdgcn_exp2f(__builtin_fmaf(xb[r], f, nl[r]));
            }
            auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(sa), __float_as_uint(sb), false, false);
            return __uint_as_float(x[0]) + __uint_as_float(x[1]);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = hg ? xb[r] : xa[r];
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x, f, nl[r]));
                sa += r < G ? p : 0.f;
            }
            return sa;
        }
    };
    if (idx0 < ngl) {
        const int koff = col * DD * 2 + hg * 16;
        const int* btb = PAGED ? pg.bt + (size_t)b * pg.maxb : nullptr;
        auto page_of = [&](int t) {
            return *(const __attribute__((address_space(4))) int*)(btb + imin(t >> pg.ps_shift, pg.maxb - 1));
        };
        // the two subtiles of group i and this lane's old score
        int page[2] = {0, 0};
        auto pages = [&](int i) {
            if constexpr (PAGED) {
                page[0] = page_of(first + 64 * i);
                page[1] = page_of(first + 64 * i + 32);
            }
        };
        auto fetch = [&](int i, wu32x4 (&c)[2][DS], float& old) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int tj = first + 64 * i + 32 * j;
                bool ok = tj < n_lat;
                size_t row = (size_t)bg * cap + tj;
                if constexpr (PAGED) {
                    ok = ok && page[j] >= 0 && page[j] < pg.n_pages;
                    row = ((size_t)(ok ? page[j] : 0) * Hkv + g) * pg.ps + (tj & (pg.ps - 1));
                }
                const int nb = ok ? imin(n_lat - tj, 32) * DD * 2 : 0;
                const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc((void*)(k_lat + (ok ? row : 0) * DD), (short)0, nb, kRawWord3);
#pragma unroll
                for (int k = 0; k < DS; ++k) c[j][k] = __builtin_amdgcn_raw_buffer_load_b128(rk, koff + 32 * k, 0, 0);
            }
            old = in[imin(first + 64 * i + lane, n_lat - 1)];
        };
        wu32x4 c[2][DS];
        float old;
        pages(idx0);
        fetch(idx0, c, old);
        pages(idx0 + nw);
        bf16x8_t qa[DS][3];
#pragma unroll
        for (int k = 0; k < DS; ++k) split3(qt + (bh0 + (hval ? head : 0)) * DD + 16 * k + 8 * hg, hval, qa[k]);
        for (int i = idx0; i < ngl; i += nw) {
            wu32x4 cn[2][DS];
            float oldn;
            fetch(i + nw, cn, oldn);
            pages(i + 2 * nw);
            f32x16_t x[2] = {splat16(0.f), splat16(0.f)};
#pragma unroll
            for (int k = 0; k < DS; ++k)
#pragma unroll
                for (int t = 2; t >= 0; --t)
#pragma unroll
                    for (int j = 0; j < 2; ++j) x[j] = mfma(qa[k][t], __builtin_bit_cast(bf16x8_t, c[j][k]), x[j]);
            const float p = weight(x[0], x[1], 1.f);
            const int e = first + 64 * i + lane;
            if (e < n_lat) out[e] = old + p;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < DS; ++k) c[j][k] = cn[j][k];
            old = oldn;
        }
    }
    // (the first of this wavefront's groups past the latents)
    int i0 = idx0;
    if (i0 < ngl) i0 += (ngl - i0 + nw - 1) / nw * nw;
    if (i0 >= ngl + ngw) return;
    bf16x8_t qw[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k)
        qw[k] = hval ? load_bf16x8(q + (bh0 + head) * D + 16 * k + 8 * hg) : zero_bf16x8();
    const bf16_t* kw = k_win + (size_t)bg * w * D;
    for (int i = i0 - ngl; i < ngw; i += nw) {
        const int t0 = n_lat + 64 * i;
        const int e = t0 + lane;
        const float old = in[imin(e, len - 1)];
        f32x16_t x[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bf16_t* row = kw + (size_t)(imin(t0 + 32 * j + col, len - 1) % w) * D;
            x[j] = splat16(0.f);
#pragma unroll
            for (int k = 0; k < KS; ++k) x[j] = mfma(qw[k], load_bf16x8(row + 16 * k + 8 * hg), x[j]);
        }
        const float p = weight(x[0], x[1], qscale);
        if (e < len && e >= first) out[e] = old + p;
    }
}

// ---- any shape of the dense decode, on the vector ALU ------------------------
//
// Lanes share a token's row, eight elements each. A batch is kBatch such tokens
// of every group of lanes: its keys and values are requested together, so that a
// workgroup of one batch (most caches) waits for memory once.

namespace {

// (4 against 2: B4 Hq16 Hkv4 d64 d_down16 4001 tokens 35.6 and 34.0 us, B8 Hq32 Hkv8 d80
// d_down20 8192 tokens 114.6 and 93.8; the other way round at most
// 4%, B8 Hkv8 G1 d80 d_down16 4000 tokens)
constexpr int kBatch = 2;
constexpr int kVThreads = 256;

struct VecSplits {
    int chunk_lat, chunk_win, n_lat, n_win;  // tokens a workgroup, workgroups of either region
};

__host__ __device__ inline int lanes_of(int dim) {
    int l = 1;
    while (l * 8 < dim) l <<= 1;
    return l;
}

// Workgroups of a region: one batch each, or several batches where that would
// be more than about four workgroups a compute unit.
VecSplits vec_splits(int B, int Hkv, int len, int w, int d, int dd) {
    VecSplits v{};
    const int far = len > w ? len - w : 0, near = len - far;
    const int most = vec_split_most(B, Hkv);
    auto cut = [&](int n, int dim, int& chunk, int& parts) {
        const int batch = kBatch * kVThreads / lanes_of(dim);
        const int nb = (n + batch - 1) / batch, per = (nb + most - 1) / most;
        chunk = batch * (per > 0 ? per : 1);
        parts = (n + chunk - 1) / chunk;
    };
    cut(far, dd, v.chunk_lat, v.n_lat);
    cut(near, d, v.chunk_win, v.n_win);
    return v;
}

template <typename T>
__device__ __forceinline__ void row8(const T* row, int off, int dim, bool vec, float (&x)[8]) {
    if (vec) {
        if constexpr (sizeof(T) == 2) {
            const uint4 u = *reinterpret_cast<const uint4*>(row + off);
            const uint32_t w4[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[2 * j] = __uint_as_float(w4[j] << 16);
                x[2 * j + 1] = __uint_as_float(w4[j] & 0xffff0000u);
            }
        } else {
            const float4 a = *reinterpret_cast<const float4*>(row + off);
            const float4 c = *reinterpret_cast<const float4*>(row + off + 4);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
            x[4] = c.x; x[5] = c.y; x[6] = c.z; x[7] = c.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = off + j < dim ? elem<T>::load(row + off + j) : 0.f;
    }
}

}  // namespace

int vec_split_most(int B, int Hkv) {
    const int most = 1024 / (B * Hkv);
    return most < 1 ? 1 : most > 256 ? 256 : most;
}

// Records of a dense decode, one workgroup per (split, sequence and KV head):
// {m, l, acc_lat[dd], acc_win[d]}, one region's part zero. qt [B * Hq][dd]: the
// absorbed, scaled queries (from the first split).
template <typename T, int G>
__global__ __launch_bounds__(kVThreads) void scored_split_kernel(
    const T* __restrict__ q, const T* __restrict__ wd, const T* __restrict__ wu,
    const T* __restrict__ k_win, const T* __restrict__ v_win, const T* __restrict__ k_lat,
    const T* __restrict__ v_lat, float* __restrict__ part, float* __restrict__ qt, int Hq, int Hkv,
    int d, int dd, int w, int cap, int len, VecSplits sp, float qscale) {
    __shared__ float qsh[G][256];
    __shared__ float red[4 * G * 256];  // partial absorbed queries, then the wavefronts' sums
    __shared__ float mred[4][G], lred[4][G];
    const int s = wg_id_x(), bg = wg_id_y(), b = bg / Hkv, g = bg - b * Hkv;
    const int tid = lane_id_x(), lane = tid & 63, wave = tid >> 6;
    const int far = imax(len - w, 0);
    const bool latent = s < sp.n_lat;
    const int dim = latent ? dd : d;
    const int t_begin = latent ? s * sp.chunk_lat : far + (s - sp.n_lat) * sp.chunk_win;
    const int t_end = latent ? imin(t_begin + sp.chunk_lat, far) : imin(t_begin + sp.chunk_win, len);
    const size_t bh0 = (size_t)b * Hq + (size_t)g * G;

    const int lpt = lanes_of(dim), sub = tid & (lpt - 1), off = sub * 8, tpi = kVThreads / lpt;
    const bool vec = (dim & 7) == 0 && off < dim;
    auto row = [&](bool keys, int t) -> const T* {
        const int c = imin(t, t_end - 1);
        return latent ? (keys ? k_lat : v_lat) + ((size_t)bg * cap + c) * dd
                      : (keys ? k_win : v_win) + ((size_t)bg * w + c % w) * d;
    };
    float k[kBatch][8], v[kBatch][8];
    auto request = [&](int t0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) row8(row(true, t0 + i * tpi + tid / lpt), off, dim, vec, k[i]);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) row8(row(false, t0 + i * tpi + tid / lpt), off, dim, vec, v[i]);
    };
    request(t_begin);

    // ---- the query, or q W_up^T: each element of W_up is read once a workgroup
    for (int i = tid; i < G * d; i += kVThreads) red[i] = elem<T>::load(q + bh0 * d + i);
    __syncthreads();
    if (latent) {
        int dp = 1;  // threads a share of the sum: one per latent column
        while (dp < dd) dp <<= 1;
        const int c = tid & (dp - 1), share = tid / dp, shares = kVThreads / dp;
        float acc[G];
#pragma unroll
        for (int h = 0; h < G; ++h) acc[h] = 0.f;
        if (c < dd)
            for (int e = share; e < d; e += shares) {
                const float u = wu ? elem<T>::load(wu + ((size_t)g * dd + c) * d + e)
                                   : elem<T>::load(wd + ((size_t)g * d + e) * dd + c);
#pragma unroll
                for (int h = 0; h < G; ++h) acc[h] = __builtin_fmaf(red[h * d + e], u, acc[h]);
            }
        __syncthreads();  // red is reused
#pragma unroll
        for (int h = 0; h < G; ++h) red[h * kVThreads + tid] = acc[h];
        __syncthreads();
        for (int i = tid; i < G * dd; i += kVThreads) {
            const int h = i / dd, c2 = i - h * dd;
            float a = 0.f;
            for (int j = 0; j < shares; ++j) a += red[h * kVThreads + j * dp + c2];
            qsh[h][c2] = a * qscale;
            if (s == 0) qt[(bh0 + h) * dd + c2] = a * qscale;
        }
    } else {
        for (int i = tid; i < G * d; i += kVThreads) qsh[i / d][i % d] = red[i] * qscale;
    }
    __syncthreads();

    float qreg[G][8], m[G], l[G], acc[G][8];
#pragma unroll
    for (int h = 0; h < G; ++h) {
        m[h] = -INFINITY;
        l[h] = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            qreg[h][j] = off + j < dim ? qsh[h][off + j] : 0.f;
            acc[h][j] = 0.f;
        }
    }
    for (int t0 = t_begin; t0 < t_end; t0 += kBatch * tpi) {
        if (t0 > t_begin) request(t0);
#pragma unroll
        for (int h = 0; h < G; ++h) {
            float x[kBatch], top = m[h];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                float a = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) a = __builtin_fmaf(qreg[h][j], k[i][j], a);
                for (int o2 = 1; o2 < lpt; o2 <<= 1) a += __shfl_xor(a, o2, 64);
                x[i] = t0 + i * tpi + tid / lpt < t_end ? a : -INFINITY;
                top = fmaxf(top, x[i]);
            }
            // (a lane's own running maximum: the lanes of a token share it)
            const float f = m[h] == -INFINITY ? 0.f : exp2f(m[h] - top);
            m[h] = top;
            l[h] *= f;
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[h][j] *= f;
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const float p = x[i] == -INFINITY ? 0.f : exp2f(x[i] - top);
                l[h] += p;
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[h][j] = __builtin_fmaf(p, v[i][j], acc[h][j]);
            }
        }
    }
    // one maximum for the workgroup, then the sums over its token groups
#pragma unroll
    for (int h = 0; h < G; ++h) {
        const float mw = wave_max(m[h]);
        if (lane == 0) mred[wave][h] = mw;
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < G; ++h) {
        const float M = fmaxf(fmaxf(mred[0][h], mred[1][h]), fmaxf(mred[2][h], mred[3][h]));
        const float f = m[h] == -INFINITY ? 0.f : exp2f(m[h] - M);
        const float lw = wave_sum(sub == 0 ? l[h] * f : 0.f);
        if (lane == 0) lred[wave][h] = lw;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float a = acc[h][j] * f;
            for (int o2 = lpt; o2 < 64; o2 <<= 1) a += __shfl_xor(a, o2, 64);
            if (lane < lpt && off + j < dim) red[(wave * G + h) * 256 + off + j] = a;
        }
    }
    __syncthreads();
    const int stride = 2 + dd + d, lo = latent ? 2 : 2 + dd, S = sp.n_lat + sp.n_win;
    for (int i = tid; i < G * stride; i += kVThreads) {
        const int h = i / stride, f = i - h * stride;
        float x = 0.f;
        if (f == 0) x = fmaxf(fmaxf(mred[0][h], mred[1][h]), fmaxf(mred[2][h], mred[3][h]));
        else if (f == 1) x = lred[0][h] + lred[1][h] + lred[2][h] + lred[3][h];
        else if (f >= lo && f < lo + dim)
            x = red[h * 256 + f - lo] + red[(G + h) * 256 + f - lo] + red[(2 * G + h) * 256 + f - lo] +
                red[(3 * G + h) * 256 + f - lo];
        part[((bh0 + h) * S + s) * stride + f] = x;
    }
}

// The weights, over the same splits.
template <typename T, int G>
__global__ __launch_bounds__(kVThreads) void decode_weights_kernel(
    const T* __restrict__ q, const float* __restrict__ qt, const float* __restrict__ lse2,
    const T* __restrict__ k_win, const T* __restrict__ k_lat, const float* scores, float* scores_out,
    int Hq, int Hkv, int d, int dd, int w, int cap, int len, VecSplits sp, float qscale) {
    const int s = wg_id_x(), bg = wg_id_y(), b = bg / Hkv, g = bg - b * Hkv;
    const int tid = lane_id_x();
    const int far = imax(len - w, 0);
    const bool latent = s < sp.n_lat;
    const int dim = latent ? dd : d;
    const int t_begin = latent ? s * sp.chunk_lat : far + (s - sp.n_lat) * sp.chunk_win;
    const int t_end = latent ? imin(t_begin + sp.chunk_lat, far) : imin(t_begin + sp.chunk_win, len);
    const size_t bh0 = (size_t)b * Hq + (size_t)g * G;
    const int lpt = lanes_of(dim), sub = tid & (lpt - 1), off = sub * 8, tpi = kVThreads / lpt;
    const bool vec = (dim & 7) == 0 && off < dim;
    float* out = scores_out + (size_t)bg * cap;
    const float* in = scores + (size_t)bg * cap;
    float k[kBatch][8], old[kBatch];
    auto request = [&](int t0) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int c = imin(t0 + i * tpi + tid / lpt, t_end - 1);
            row8(latent ? k_lat + ((size_t)bg * cap + c) * dd : k_win + ((size_t)bg * w + c % w) * d, off, dim,
                 vec, k[i]);
            old[i] = in[c];
        }
    };
    request(t_begin);
    float qreg[G][8], nl[G];
#pragma unroll
    for (int h = 0; h < G; ++h) {
        nl[h] = -lse2[bh0 + h];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = imin(off + j, dim - 1);
            const float x = latent ? qt[(bh0 + h) * dd + c] : elem<T>::load(q + (bh0 + h) * d + c) * qscale;
            qreg[h][j] = off + j < dim ? x : 0.f;
        }
    }
    for (int t0 = t_begin; t0 < t_end; t0 += kBatch * tpi) {
        if (t0 > t_begin) request(t0);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            float p = 0.f;
#pragma unroll
            for (int h = 0; h < G; ++h) {
                float a = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) a = __builtin_fmaf(qreg[h][j], k[i][j], a);
                for (int o2 = 1; o2 < lpt; o2 <<= 1) a += __shfl_xor(a, o2, 64);
                p += exp2f(a + nl[h]);
            }
            const int t = t0 + i * tpi + tid / lpt;
            if (sub == 0 && t < t_end) out[t] = old[i] + p;
        }
    }
}

hipError_t launch_decode_finish(const bf16_t* q, const bf16_t* wd, const bf16_t* wu,
                                const float* part, int S, const float* ppart, int NS,
                                const float* qt, const bf16_t* k_win, const bf16_t* k_lat, bf16_t* o,
                                const float* scores, float* scores_out, int B, int Hq, int Hkv, int d,
                                int dd, int w, int cap, int len, const PagedArgs* pg_in,
                                hipStream_t st) {
    const float qscale = 1.4426950408889634f / sqrtf((float)d);
    const PagedArgs pg = pg_in ? *pg_in : PagedArgs{};
    long long gx = 0;  // workgroups of the weights
    if (scores) {
        const long long groups = ((pg_in ? cap : len) + 63) / 64 + 1;
        // about 4 a compute unit (6 and 8: up to 3% more at 32 x 8 pairs of 32K tokens)
        const long long most = (4 * 256 + B * Hkv - 1) / (B * Hkv);
        gx = (groups + kWWaves - 1) / kWWaves;
        gx = gx > most ? most : gx;
    }
    const dim3 grid((unsigned)(gx + (Hq / Hkv + kWWaves - 1) / kWWaves), B * Hkv);
#define DAR_FINISH(D_, DD_, G8_, P_)                                                               \
    hipLaunchKernelGGL((decode_finish_kernel<D_, DD_, G8_, P_>), grid, dim3(kWThreads), 0, st, q, wd, \
                       wu, part, S, ppart, NS, qt, k_win, k_lat, o, scores, scores_out, Hq, Hkv, w,  \
                       cap, len, pg, qscale, (int)gx)
#define DAR_FINISH_G(D_, DD_)                                   \
    if (Hq / Hkv > 4) {                                         \
        if (pg_in) DAR_FINISH(D_, DD_, true, true);             \
        else DAR_FINISH(D_, DD_, true, false);                  \
    } else {                                                    \
        if (pg_in) DAR_FINISH(D_, DD_, false, true);            \
        else DAR_FINISH(D_, DD_, false, false);                 \
    }
    if (d == 64 && dd == 16) { DAR_FINISH_G(64, 16) }
    else if (d == 64 && dd == 32) { DAR_FINISH_G(64, 32) }
    else if (d == 128 && dd == 16) { DAR_FINISH_G(128, 16) }
    else { DAR_FINISH_G(128, 32) }
#undef DAR_FINISH_G
#undef DAR_FINISH
    return hipGetLastError();
}

template <typename T>
hipError_t launch_scored_vec(const T* q, const T* wd, const T* wu, const T* k_win, const T* v_win,
                             const T* k_lat, const T* v_lat, T* o, float* part, float* qt, float* lse2,
                             const float* scores, float* scores_out, int B, int Hq, int Hkv, int d,
                             int dd, int w, int cap, int len, hipStream_t st) {
    const float qscale = 1.4426950408889634f / sqrtf((float)d);
    const VecSplits sp = vec_splits(B, Hkv, len, w, d, dd);
    const int S = sp.n_lat + sp.n_win;
    const dim3 grid(S, B * Hkv), block(kVThreads);
#define DAR_BY_GROUP(X_)                    \
    switch (Hq / Hkv) {                     \
        case 1: X_(1); break;               \
        case 2: X_(2); break;               \
        case 4: X_(4); break;               \
        case 8: X_(8); break;               \
        default: return hipErrorInvalidValue; \
    }
#define DAR_SPLIT(G_)                                                                              \
    hipLaunchKernelGGL((scored_split_kernel<T, G_>), grid, block, 0, st, q, wd, wu, k_win, v_win,  \
                       k_lat, v_lat, part, qt, Hq, Hkv, d, dd, w, cap, len, sp, qscale)
    DAR_BY_GROUP(DAR_SPLIT)
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
#define DAR_JOIN(NR_)                                                                              \
    hipLaunchKernelGGL((records_join_kernel<T, NR_>), dim3(B * Hq), dim3(64), 0, st, part, S, wd, wu, \
                       o, lse2, Hq, Hkv, d, dd)
    if (d <= 64) DAR_JOIN(1);
    else if (d <= 128) DAR_JOIN(2);
    else DAR_JOIN(4);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
#define DAR_WEIGHTS(G_)                                                                            \
    hipLaunchKernelGGL((decode_weights_kernel<T, G_>), grid, block, 0, st, q, qt, lse2, k_win, k_lat, \
                       scores, scores_out, Hq, Hkv, d, dd, w, cap, len, sp, qscale)
    DAR_BY_GROUP(DAR_WEIGHTS)
#undef DAR_WEIGHTS
#undef DAR_JOIN
#undef DAR_SPLIT
#undef DAR_BY_GROUP
    return hipGetLastError();
}
template hipError_t launch_scored_vec<float>(const float*, const float*, const float*, const float*,
                                             const float*, const float*, const float*, float*, float*,
                                             float*, float*, const float*, float*, int, int, int, int,
                                             int, int, int, int, hipStream_t);
template hipError_t launch_scored_vec<bf16_t>(const bf16_t*, const bf16_t*, const bf16_t*,
                                              const bf16_t*, const bf16_t*, const bf16_t*,
                                              const bf16_t*, bf16_t*, float*, float*, float*,
                                              const float*, float*, int, int, int, int, int, int, int,
                                              int, hipStream_t);

}  // namespace dar
