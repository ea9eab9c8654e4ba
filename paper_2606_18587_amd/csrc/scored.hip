// Decode steps that score the cached tokens by the attention weight they
// receive (dar_attn_decode_scored, dar_attn_decode_paged_scored), and the
// merge of partial records that they share with the shared-prefix decode.
//
//   1. partial records of every part of the cache: the split decode kernels
//      (decode.hip, or decode_mfma.hip in its records mode);
//   2. records_join_kernel: one wavefront per (sequence, query head) merges
//      them under one maximum, writes the output and the logarithm of the
//      softmax denominator;
//   3. decode_weights_*_kernel: the weights themselves. They need the
//      denominator, which is known after the last key, so every key is met a
//      second time: p = exp2(s - lse2), summed over the query heads of the KV
//      head and added to the token's score. Of the cache it reads the key
//      latents and the ring's keys, half of what step 1 reads.
#include "../../include/dar_serving.h"
#include "dar_common.hpp"
#include "dar_kernels.hpp"
#include "mfma_common.hpp"

namespace dar {

// Own records {m, l, acc_lat[dd], acc_win[d]} of (sequence, query head) bh at
// part + (bh * S_all + s) * (2 + dd + d): all S_all of them, or (paged) the
// count that the decode kernel left for the pair. Shared-prefix records
// {m, l, acc_lat[dd]} at ppart + (bh * NS + s) * (2 + dd).
// A wavefront per head. Its loads come in three groups, each independent within
// itself: the records' {m, l} and the first W_up rows, the records' sums, the
// rest of W_up; as many records side by side as their latent sums leave lanes
// for. (One record after the other, each waiting for the last: 20 to 30 us at
// 1024 to 2048 heads.) NR: output columns per lane (d <= 64 NR).
constexpr int kJoinMax = 1024 + 64;  // own records and shared-prefix records, at most
constexpr int kJoinRegs = 32;        // W_up rows requested before the records

template <typename T, int NR>
__global__ __launch_bounds__(64) void records_join_kernel(
    const float* __restrict__ part, int S_all, const float* __restrict__ ppart, int NS,
    const T* __restrict__ wd, const T* __restrict__ wu, T* __restrict__ o, float* __restrict__ lse2,
    int Hq, int Hkv, int d, int dd, int w, const int* __restrict__ lens,
    const int* __restrict__ counts, int pre) {
    __shared__ float wsh[kJoinMax];  // the records' weights
    __shared__ float lsh[256];       // the merged latent sum
    const int bh = wg_id_x(), lane = lane_id_x();
    const int b = bh / Hq, g = (bh - b * Hq) / (Hq / Hkv);
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
    int S = S_all;
    if (lens) {
        const int len = lens[b];
        if (len < 1) {  // empty or overflowed: no query position, NaN
            for (int e = lane; e < d; e += 64) {
                if (sizeof(T) == 2) reinterpret_cast<uint16_t*>(o)[(size_t)bh * d + e] = 0x7fc0;
                else reinterpret_cast<uint32_t*>(o)[(size_t)bh * d + e] = 0x7fc00000u;
            }
            return;
        }
        // (a sequence all of whose tokens are the prefix's has no part of its own)
        S = w == 0 && (len + 31) / 32 <= pre ? 0 : imin(S_all, counts[b * Hkv + g]);
    }
    const int stride = 2 + dd + d, pstride = 2 + dd, n = S + NS;
    const float* own = part + (size_t)bh * S_all * stride;
    const float* pfx = ppart + (size_t)bh * NS * pstride;
    auto rec = [&](int s) { return s < S ? own + (size_t)s * stride : pfx + (size_t)(s - S) * pstride; };

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
    if (lse2 && lane == 0) lse2[bh] = M + log2f(L);
    __syncthreads();

    // window sums: a lane owns columns lane + 64 r
    constexpr int kAhead = 8;
    float acc[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) acc[r] = 0.f;
    for (int s0 = 0; s0 < S; s0 += kAhead) {
        float x[kAhead][NR];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
#pragma unroll
            for (int r = 0; r < NR; ++r)
                x[j][r] = own[(size_t)imin(s0 + j, S - 1) * stride + 2 + dd + imin(lane + 64 * r, d - 1)];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const float ws = s0 + j < S ? wsh[s0 + j] : 0.f;
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

template <typename T>
hipError_t launch_records_join(const float* part, int S, const float* ppart, int NS, const T* wd,
                               const T* wu, T* o, float* lse2, int B, int Hq, int Hkv, int d, int dd,
                               int w, const int* lens, const int* counts, int pre, hipStream_t st) {
#define DAR_JOIN(NR_)                                                                              \
    hipLaunchKernelGGL((records_join_kernel<T, NR_>), dim3(B * Hq), dim3(64), 0, st, part, S, ppart, \
                       NS, wd, wu, o, lse2, Hq, Hkv, d, dd, w, lens, counts, pre)
    if (d <= 64) DAR_JOIN(1);
    else if (d <= 128) DAR_JOIN(2);
    else DAR_JOIN(4);
#undef DAR_JOIN
    return hipGetLastError();
}
template hipError_t launch_records_join<float>(const float*, int, const float*, int, const float*,
                                               const float*, float*, float*, int, int, int, int, int,
                                               int, const int*, const int*, int, hipStream_t);
template hipError_t launch_records_join<bf16_t>(const float*, int, const float*, int, const bf16_t*,
                                                const bf16_t*, bf16_t*, float*, int, int, int, int,
                                                int, int, const int*, const int*, int, hipStream_t);

namespace {

constexpr int kWThreads = 256, kWWaves = kWThreads / 64;

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

// Weights on the matrix cores (bf16, d in {64, 128}, d_down in {16, 32}):
// S = Q~ C^T with the query heads as rows and 32 tokens as columns, so that a
// lane holds all heads of one token and the sum over them stays in it. Rows 0..3
// and 4..7 (lane halves) hold heads 0..3 twice, or (G8) heads 0..3 and 4..7;
// two subtiles at a time, so that lane l finishes token l of the 64.
template <int D, int DD, bool G8, bool PAGED>
__global__ __launch_bounds__(kWThreads) void decode_weights_mfma_kernel(
    const bf16_t* __restrict__ q, const float* __restrict__ qt, const float* __restrict__ lse2,
    const bf16_t* __restrict__ k_win, const bf16_t* __restrict__ k_lat, const float* scores,
    float* scores_out, int Hq, int Hkv, int w, int cap, int len_arg, PagedArgs pg, float qscale) {
    constexpr int KS = D / 16, DS = DD / 16;
    const int bg = wg_id_y(), b = bg / Hkv, g = bg - b * Hkv;
    const int tid = lane_id_x(), lane = tid & 63, col = lane & 31, hg = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = Hq / Hkv;
    int len = len_arg;
    if constexpr (PAGED) len = imin(pg.lens[b], cap);
    if (len < 1) return;
    const int first = PAGED ? 32 * pg.pre : 0;
    const int n_lat = imax(len - w, 0);
    const int ngl = (imax(n_lat - first, 0) + 63) >> 6, ngw = (len - n_lat + 63) >> 6;
    const int nw = (int)(__builtin_amdgcn_grid_size_x() >> 6);
    const int idx0 = wg_id_x() * kWWaves + wave;
    if (idx0 >= ngl + ngw) return;

    const int head = G8 ? col : (col & 3);  // A-operand row col
    const bool hval = col < 8 && head < G;
    const size_t bh0 = (size_t)b * Hq + (size_t)g * G;
    float nl[4];  // -lse2 of the head in accumulator register r
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int h = G8 ? 4 * hg + r : r;
        nl[r] = -lse2[bh0 + (h < G ? h : 0)];
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
        bf16x8_t qa[DS][3];
#pragma unroll
        for (int k = 0; k < DS; ++k) split3(qt + (bh0 + (hval ? head : 0)) * DD + 16 * k + 8 * hg, hval, qa[k]);
        const bf16_t* kl = k_lat + (size_t)bg * cap * DD;
        for (int i = idx0; i < ngl; i += nw) {
            const int t0 = first + 64 * i;
            const int e = t0 + lane;
            const float old = e < n_lat ? in[e] : 0.f;
            bf16x8_t c[2][DS];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int tj = t0 + 32 * j;
                const bf16_t* row;
                bool ok = tj < n_lat;  // (uniform)
                if constexpr (PAGED) {
                    const int blk = imin(tj >> pg.ps_shift, pg.maxb - 1);
                    const int page = pg.bt[(size_t)b * pg.maxb + blk];
                    ok = ok && page >= 0 && page < pg.n_pages;
                    row = k_lat + (((size_t)(ok ? page : 0) * Hkv + g) * pg.ps +
                                   (imin(tj + col, n_lat - 1) & (pg.ps - 1))) * DD;
                } else {
                    row = kl + (size_t)imin(tj + col, n_lat - 1) * DD;
                }
#pragma unroll
                for (int k = 0; k < DS; ++k) c[j][k] = ok ? load_bf16x8(row + 16 * k + 8 * hg) : zero_bf16x8();
            }
            f32x16_t x[2] = {splat16(0.f), splat16(0.f)};
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < DS; ++k)
#pragma unroll
                    for (int t = 2; t >= 0; --t) x[j] = mfma(qa[k][t], c[j][k], x[j]);
            const float p = weight(x[0], x[1], 1.f);
            if (e < n_lat) out[e] = old + p;
        }
    }
    bf16x8_t qw[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k)
        qw[k] = hval ? load_bf16x8(q + (bh0 + head) * D + 16 * k + 8 * hg) : zero_bf16x8();
    const bf16_t* kw = k_win + (size_t)bg * w * D;
    // (the first of this wavefront's groups past the latents)
    int i0 = idx0;
    if (i0 < ngl) i0 += (ngl - i0 + nw - 1) / nw * nw;
    for (int i = i0 - ngl; i < ngw; i += nw) {
        const int t0 = n_lat + 64 * i;
        const int e = t0 + lane;
        f32x16_t x[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bf16_t* row = kw + (size_t)(imin(t0 + 32 * j + col, len - 1) % w) * D;
            x[j] = splat16(0.f);
#pragma unroll
            for (int k = 0; k < KS; ++k) x[j] = mfma(qw[k], load_bf16x8(row + 16 * k + 8 * hg), x[j]);
        }
        const float p = weight(x[0], x[1], qscale);
        if (e < len && e >= first) out[e] = in[e] + p;
    }
}

// Weights on the vector ALU, any shape of the dense decode: lanes share a
// token's row as in the split kernel.
template <typename T, int G>
__global__ __launch_bounds__(kWThreads) void decode_weights_kernel(
    const T* __restrict__ q, const T* __restrict__ wd, const T* __restrict__ wu,
    const float* __restrict__ lse2, const T* __restrict__ k_win, const T* __restrict__ k_lat,
    const float* scores, float* scores_out, int Hq, int Hkv, int d, int dd, int w, int cap, int len,
    int chunk, int n_lat_chunk, float qscale) {
    __shared__ float qsh[G][256];
    const int s = wg_id_x(), bg = wg_id_y(), b = bg / Hkv, g = bg - b * Hkv;
    const int tid = lane_id_x();
    const int n_lat = imax(len - w, 0);
    const bool latent = s < n_lat_chunk;
    const int dim = latent ? dd : d;
    const int t_begin = latent ? s * chunk : n_lat + (s - n_lat_chunk) * chunk;
    const int t_end = imin(t_begin + chunk, latent ? n_lat : len);
    const size_t bh0 = (size_t)b * Hq + (size_t)g * G;
    for (int idx = tid; idx < G * dim; idx += kWThreads) {
        const int hh = idx / dim, c = idx - hh * dim;
        const T* qrow = q + (bh0 + hh) * d;
        float acc;
        if (latent) {
            acc = 0.f;
            for (int e = 0; e < d; ++e) {
                const float u = wu ? elem<T>::load(wu + ((size_t)g * dd + c) * d + e)
                                   : elem<T>::load(wd + ((size_t)g * d + e) * dd + c);
                acc = __builtin_fmaf(elem<T>::load(qrow + e), u, acc);
            }
        } else {
            acc = elem<T>::load(qrow + c);
        }
        qsh[hh][c] = acc * qscale;
    }
    __syncthreads();
    int lpt = 1;  // lanes per token, eight elements each
    while (lpt * 8 < dim) lpt <<= 1;
    const int sub = tid & (lpt - 1), off = sub * 8;
    float qreg[G][8], nl[G];
#pragma unroll
    for (int hh = 0; hh < G; ++hh) {
        nl[hh] = -lse2[bh0 + hh];
#pragma unroll
        for (int j = 0; j < 8; ++j) qreg[hh][j] = off + j < dim ? qsh[hh][off + j] : 0.f;
    }
    for (int t0 = t_begin; t0 < t_end; t0 += kWThreads / lpt) {
        const int t = t0 + tid / lpt;
        float x[8];
        const T* row = latent ? k_lat + ((size_t)bg * cap + imin(t, t_end - 1)) * dd
                              : k_win + ((size_t)bg * w + imin(t, t_end - 1) % w) * d;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = off + j < dim ? elem<T>::load(row + off + j) : 0.f;
        float p = 0.f;
#pragma unroll
        for (int hh = 0; hh < G; ++hh) {
            float a = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) a = __builtin_fmaf(qreg[hh][j], x[j], a);
            for (int o2 = 1; o2 < lpt; o2 <<= 1) a += __shfl_xor(a, o2, 64);
            p += exp2f(a + nl[hh]);
        }
        if (sub == 0 && t < t_end) scores_out[(size_t)bg * cap + t] = scores[(size_t)bg * cap + t] + p;
    }
}

hipError_t launch_decode_weights_mfma(const bf16_t* q, const float* qt, const float* lse2,
                                      const bf16_t* k_win, const bf16_t* k_lat, const float* scores,
                                      float* scores_out, int B, int Hq, int Hkv, int d, int dd, int w,
                                      int cap, int len, const PagedArgs* pg_in, hipStream_t st) {
    const float qscale = 1.4426950408889634f / sqrtf((float)d);
    const PagedArgs pg = pg_in ? *pg_in : PagedArgs{};
    const long long groups = ((pg_in ? cap : len) + 63) / 64 + 1;
    long long gx = (groups + kWWaves - 1) / kWWaves;
    const long long most = (8 * 256 + B * Hkv - 1) / (B * Hkv);  // about 8 workgroups a compute unit
    gx = gx > most ? most : gx;
    const dim3 grid((unsigned)gx, B * Hkv);
#define DAR_WEIGHTS(D_, DD_, G8_, P_)                                                              \
    hipLaunchKernelGGL((decode_weights_mfma_kernel<D_, DD_, G8_, P_>), grid, dim3(kWThreads), 0, st, \
                       q, qt, lse2, k_win, k_lat, scores, scores_out, Hq, Hkv, w, cap, len, pg, qscale)
#define DAR_WEIGHTS_G(D_, DD_)                                   \
    if (Hq / Hkv > 4) {                                          \
        if (pg_in) DAR_WEIGHTS(D_, DD_, true, true);             \
        else DAR_WEIGHTS(D_, DD_, true, false);                  \
    } else {                                                     \
        if (pg_in) DAR_WEIGHTS(D_, DD_, false, true);            \
        else DAR_WEIGHTS(D_, DD_, false, false);                 \
    }
    if (d == 64 && dd == 16) { DAR_WEIGHTS_G(64, 16) }
    else if (d == 64 && dd == 32) { DAR_WEIGHTS_G(64, 32) }
    else if (d == 128 && dd == 16) { DAR_WEIGHTS_G(128, 16) }
    else { DAR_WEIGHTS_G(128, 32) }
#undef DAR_WEIGHTS_G
#undef DAR_WEIGHTS
    return hipGetLastError();
}

template <typename T>
hipError_t launch_decode_weights(const T* q, const T* wd, const T* wu, const float* lse2,
                                 const T* k_win, const T* k_lat, const float* scores,
                                 float* scores_out, int B, int Hq, int Hkv, int d, int dd, int w,
                                 int cap, int len, hipStream_t st) {
    const float qscale = 1.4426950408889634f / sqrtf((float)d);
    const int n_lat = len > w ? len - w : 0;
    const int chunk = 1024;
    const int ncl = (n_lat + chunk - 1) / chunk, ncw = (len - n_lat + chunk - 1) / chunk;
#define DAR_WEIGHTS(G_)                                                                            \
    hipLaunchKernelGGL((decode_weights_kernel<T, G_>), dim3(ncl + ncw, B * Hkv), dim3(kWThreads), 0, \
                       st, q, wd, wu, lse2, k_win, k_lat, scores, scores_out, Hq, Hkv, d, dd, w, cap, \
                       len, chunk, ncl, qscale)
    switch (Hq / Hkv) {
        case 1: DAR_WEIGHTS(1); break;
        case 2: DAR_WEIGHTS(2); break;
        case 4: DAR_WEIGHTS(4); break;
        case 8: DAR_WEIGHTS(8); break;
        default: return hipErrorInvalidValue;
    }
#undef DAR_WEIGHTS
    return hipGetLastError();
}
template hipError_t launch_decode_weights<float>(const float*, const float*, const float*,
                                                 const float*, const float*, const float*,
                                                 const float*, float*, int, int, int, int, int, int,
                                                 int, int, hipStream_t);
template hipError_t launch_decode_weights<bf16_t>(const bf16_t*, const bf16_t*, const bf16_t*,
                                                  const float*, const bf16_t*, const bf16_t*,
                                                  const float*, float*, int, int, int, int, int, int,
                                                  int, int, hipStream_t);

}  // namespace dar
