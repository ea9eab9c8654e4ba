// Decode over a cache whose distant latents are held in 4 bits
// (include/dar_q4.h): Eq. 3-4 for one query a sequence, the distant tokens as
// they stand in the cache, the window at full dimension, one softmax over both.
//
// Work split. Every (sequence, KV head, tile of query heads) pair has two regions,
// its distant tokens in blocks of 128 and its window in steps of 32 tokens. Laid
// end to end in units of about the same bytes (kWinUnits a window step, one a
// block) all regions of the batch form one line, which the wavefronts of the
// launch share evenly, wherever the cuts fall; the line is computed on the
// device from the sequences' lengths, so ragged batches are balanced as dense
// ones are. A wavefront's piece of a region is a segment: it leaves one record
// {m, l, acc} per query head, with m the reference of its exponentials (log2
// units), l their sum and acc the weighted sum of values (of latents where
// distant). q4_merge_kernel joins the records of a query head and lifts the
// latent part once, o = (acc_win + acc_lat W_up) / l.
#include "mfma_common.hpp"
#include "q4.hpp"

namespace dar {

namespace {

constexpr int kBlock = 128;     // distant tokens a unit
constexpr int kStep = 32;       // window tokens a step
constexpr int kWinUnits = 4;    // units a window step counts for (64 x 32 x 4 B against 128 x 18)
constexpr int kMinUnits = 4;    // units a wavefront takes at least
constexpr int kWaves = 4096;    // wavefronts of the largest launch
constexpr int kMaxTile = 8;     // query heads of a tile, at most

// --- the line of units ---------------------------------------------------------

struct Plan {
    const int* lens;  // NULL: every sequence holds len
    int len, cap, w, B;
    int pairs;  // (KV head, tile) pairs a sequence
    int waves;
};

__host__ __device__ inline int held(int len, int cap) { return len < 0 ? 0 : (len > cap ? cap : len); }
__host__ __device__ inline int lat_units(int L, int w) { return L > w ? (int)(((long long)L - w + kBlock - 1) / kBlock) : 0; }
__host__ __device__ inline int win_units(int L, int w) { return ((L < w ? L : w) + kStep - 1) / kStep * kWinUnits; }
__host__ __device__ inline int seq_units(int L, int w) { return lat_units(L, w) + win_units(L, w); }
// units of a wavefront
__host__ __device__ inline long long share_of(long long total, int waves) {
    const long long cu = (total + waves - 1) / waves;
    return cu > kMinUnits ? cu : kMinUnits;
}

__device__ __forceinline__ int plan_len(const Plan& p, int b) { return p.lens ? held(p.lens[b], p.cap) : p.len; }

__device__ __forceinline__ long long wave_sum64(long long x) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
    return x;
}

// All units of the batch.
__device__ __forceinline__ long long plan_total(const Plan& p, int lane) {
    if (!p.lens) return (long long)p.B * p.pairs * seq_units(p.len, p.w);
    long long t = 0;
    for (int b = lane; b < p.B; b += 64) t += seq_units(plan_len(p, b), p.w);
    return wave_sum64(t) * p.pairs;
}

// The sequence that unit u (< total) lies in, and its first unit.
__device__ __forceinline__ int plan_find(const Plan& p, long long u, int lane, long long& base) {
    if (!p.lens) {
        const long long per = (long long)p.pairs * seq_units(p.len, p.w);
        const int b = (int)(u / per);
        base = b * per;
        return b;
    }
    long long before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        long long x = b0 + lane < p.B ? (long long)p.pairs * seq_units(plan_len(p, b0 + lane), p.w) : 0;
        const long long mine = x;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const long long y = __shfl_up(x, off, 64);
            if (lane >= off) x += y;
        }
        const unsigned long long past = __builtin_amdgcn_ballot_w64(before + x > u);
        if (past) {
            const int at = __builtin_ctzll(past);
            base = before + __shfl(x - mine, at, 64);
            return b0 + at;
        }
        before += __shfl(x, 63, 64);
    }
    base = before;
    return p.B;  // not reached for u < total
}

// First unit of sequence b.
__device__ __forceinline__ long long plan_base(const Plan& p, int b, int lane) {
    if (!p.lens) return (long long)b * p.pairs * seq_units(p.len, p.w);
    long long t = 0;
    for (int i = lane; i < b; i += 64) t += seq_units(plan_len(p, i), p.w);
    return wave_sum64(t) * p.pairs;
}

// Records. A segment's number grows along the line, by the wavefront and by the
// region: 2 pair + (window) + wavefront is unique.
__host__ __device__ inline size_t record_floats(int tile, int d) { return (size_t)tile * (2 + d); }
__device__ __forceinline__ float* record(float* part, long long wave, long long pair, int win, int tile, int d) {
    return part + (size_t)(wave + 2 * pair + win) * record_floats(tile, d);
}

struct DecodeArgs {
    const void *q, *wd, *wu, *k_win, *v_win;
    const uint8_t *codes[2], *exps[2];
    float* part;
    void* o;
    Q4Rows rows;
    Plan plan;
    int Hq, Hkv, d, dd, w, tiles;
    float qscale;
};

// Walks the segments of wavefront `wave`: seg(b, x, L, win, lo, hi) for units [lo,
// hi) of region `win` of pair x of sequence b, which holds L tokens.
template <typename F>
__device__ __forceinline__ void walk(const Plan& p, long long wave, int lane, F&& seg) {
    const long long total = plan_total(p, lane), cu = share_of(total, p.waves);
    long long u = wave * cu;
    const long long end = u + cu < total ? u + cu : total;
    if (u >= end) return;
    long long base;
    int b = plan_find(p, u, lane, base);
    while (u < end && b < p.B) {
        const int L = __builtin_amdgcn_readfirstlane(plan_len(p, b));
        const int nl = lat_units(L, p.w), nu = nl + win_units(L, p.w);
        if (nu == 0 || u - base >= (long long)nu * p.pairs) {
            base += (long long)nu * p.pairs;
            ++b;
            continue;
        }
        const int x = (int)((u - base) / nu), off = (int)((u - base) - (long long)x * nu);
        const int win = off >= nl;
        const int lo = win ? off - nl : off;
        const int size = win ? nu - nl : nl;
        const int hi = (int)(end - u < size - lo ? lo + (end - u) : size);
        seg(b, x, L, win, lo, hi);
        u += hi - lo;
    }
}

// --- any shape, on the vector ALU ----------------------------------------------
//
// A lane a token for the scores (64 tokens at a time), a lane a column for the
// values; the weights pass through LDS. Reached where the matrix cores are not:
// fp32, other head sizes and bottlenecks.

constexpr int kVecTile = 4;

template <typename T>
__global__ __launch_bounds__(256) void q4_vec_kernel(DecodeArgs a) {
    __shared__ float qsh[4][kVecTile][256];
    __shared__ float psh[4][64][kVecTile];
    const int lane = lane_id_x() & 63;
    const int wv = __builtin_amdgcn_readfirstlane(lane_id_x() >> 6);
    const long long wave = (long long)wg_id_x() * 4 + wv;
    const int G = a.Hq / a.Hkv, d = a.d, dd = a.dd;
    const int rb = q4_row_bytes(dd), ng = q4_groups(dd);
    float(*qs)[256] = qsh[wv];
    float(*ps)[kVecTile] = psh[wv];

    walk(a.plan, wave, lane, [&](int b, int x, int L, int win, int lo, int hi) {
        const int g = x / a.tiles, h0 = (x - g * a.tiles) * kVecTile;
        const int nh = imin(kVecTile, G - h0);
        const int bg = b * a.Hkv + g;
        const int n_lat = L > a.w ? L - a.w : 0;
        const int width = win ? d : dd;
        const T* wdg = (const T*)a.wd + (size_t)g * d * dd;
        const T* wug = a.wu ? (const T*)a.wu + (size_t)g * dd * d : nullptr;
        // queries, absorbed for distant tokens, in log2 units
        wave_lds_order();
        for (int h = 0; h < kVecTile; ++h) {
            const T* q = (const T*)a.q + ((size_t)b * a.Hq + (size_t)g * G + h0 + imin(h, nh - 1)) * d;
            for (int c = lane; c < 256; c += 64) {
                float s = 0.f;
                if (h < nh && c < width) {
                    if (win) {
                        s = elem<T>::load(q + c);
                    } else {
                        for (int e = 0; e < d; ++e)
                            s = __builtin_fmaf(elem<T>::load(q + e),
                                               elem<T>::load(wug ? wug + (size_t)c * d + e : wdg + (size_t)e * dd + c), s);
                    }
                }
                qs[h][c] = s * a.qscale;
            }
        }
        wave_lds_order();

        // tokens [t0, t1) of the sequence
        const int t0 = win ? n_lat + (lo + kWinUnits - 1) / kWinUnits * kStep : lo * kBlock;
        const int t1 = win ? imin(L, n_lat + (hi + kWinUnits - 1) / kWinUnits * kStep)
                           : (int)(hi * (long long)kBlock < n_lat ? hi * kBlock : n_lat);
        const T* kw = (const T*)a.k_win + (size_t)bg * a.w * d;
        const T* vw = (const T*)a.v_win + (size_t)bg * a.w * d;
        // value lanes: a column each, groups of lanes taking turns at the tokens
        const int cw = width <= 16 ? 16 : (width <= 32 ? 32 : 64);
        const int tg = lane / cw, ntg = 64 / cw, col = lane - tg * cw;
        float m[kVecTile], l[kVecTile], acc[kVecTile][4];
#pragma unroll
        for (int h = 0; h < kVecTile; ++h) {
            m[h] = -INFINITY;
            l[h] = 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[h][r] = 0.f;
        }
        for (int tb = t0; tb < t1; tb += 64) {
            const int t = tb + lane;
            const bool live = t < t1;
            float s[kVecTile] = {0.f, 0.f, 0.f, 0.f};
            if (live && win) {
                const T* k = kw + (size_t)(t % a.w) * d;
                for (int e = 0; e < d; ++e) {
                    const float kv = elem<T>::load(k + e);
#pragma unroll
                    for (int h = 0; h < kVecTile; ++h) s[h] = __builtin_fmaf(kv, qs[h][e], s[h]);
                }
            } else if (live) {
                const long long row = q4_row(a.rows, b, g, a.Hkv, t);
                if (row >= 0)
                    for (int k = 0; k < rb / 4; ++k) {
                        float v[8];
                        q4_values_f32(((const uint32_t*)a.codes[0])[row * (rb / 4) + k],
                                      q4_scale(a.exps[0][row * ng + (k >> 2)]), v);
#pragma unroll
                        for (int h = 0; h < kVecTile; ++h)
#pragma unroll
                            for (int c = 0; c < 8; ++c) s[h] = __builtin_fmaf(v[c], qs[h][8 * k + c], s[h]);
                    }
            }
            wave_lds_order();
#pragma unroll
            for (int h = 0; h < kVecTile; ++h) {
                const float mx = fmaxf(m[h], wave_max(live ? s[h] : -INFINITY));
                // (mx is -inf only where every score is; NaN scores stay NaN)
                const float ref = mx == -INFINITY ? 0.f : mx;
                const float f = m[h] == -INFINITY ? 0.f : exp2f(m[h] - ref);
                const float p = live ? exp2f(s[h] - ref) : 0.f;
                l[h] = l[h] * f + p;
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[h][r] *= f;
                m[h] = mx;
                ps[lane][h] = p;
            }
            wave_lds_order();
            const int nt = imin(64, t1 - tb);
            for (int i = tg; i < nt; i += ntg) {
                const float4 p4 = *reinterpret_cast<const float4*>(ps[i]);
                const float pv[4] = {p4.x, p4.y, p4.z, p4.w};
                const T* v = vw;
                long long row = 0;
                if (win) v = vw + (size_t)((tb + i) % a.w) * d;
                else row = q4_row(a.rows, b, g, a.Hkv, tb + i);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int c = col + 64 * r;
                    if (c >= width || row < 0) continue;
                    float val;
                    if (win) {
                        val = elem<T>::load(v + c);
                    } else {
                        const uint32_t w = ((const uint32_t*)a.codes[1])[row * (rb / 4) + (c >> 3)];
                        val = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w >> (4 * (c & 7)), q4_scale(a.exps[1][row * ng + (c >> 5)]), 0)[0];
                    }
#pragma unroll
                    for (int h = 0; h < kVecTile; ++h) acc[h][r] = __builtin_fmaf(pv[h], val, acc[h][r]);
                }
            }
        }
        float* rec = record(a.part, wave, (long long)b * a.plan.pairs + x, win, kVecTile, d);
#pragma unroll
        for (int h = 0; h < kVecTile; ++h) {
            const float ls = wave_sum(l[h]);
            float* r = rec + h * (2 + d);
            if (lane == 0) {
                r[0] = t0 < t1 ? m[h] : -INFINITY;
                r[1] = ls;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float v = acc[h][k];
                for (int off = cw; off < 64; off <<= 1) v += __shfl_xor(v, off, 64);
                const int c = col + 64 * k;
                if (tg == 0 && c < width) r[2 + c] = v;
            }
        }
    });
}

// --- merge ---------------------------------------------------------------------
//
// One workgroup a query head. Records of its two regions: those of the wavefronts
// whose shares meet them. A sequence without a query position gets NaN.
template <typename T>
__global__ __launch_bounds__(256) void q4_merge_kernel(DecodeArgs a, int tile) {
    constexpr int kMost = 512;  // records whose weights are kept in LDS at a time
    __shared__ float wt[kMost], red[4], sum[2][256], out[256];
    const int tid = lane_id_x(), lane = tid & 63, wv = tid >> 6;
    const int bh = wg_id_x(), b = bh / a.Hq, h = bh - b * a.Hq;
    const int G = a.Hq / a.Hkv, g = h / G, hg = h - g * G;
    const int d = a.d, dd = a.dd;
    T* o = (T*)a.o + (size_t)bh * d;
    if (a.plan.lens && a.plan.lens[b] < 1) {
        for (int e = tid; e < d; e += 256) {
            if (sizeof(T) == 2) reinterpret_cast<uint16_t*>(o)[e] = 0x7fc0;
            else reinterpret_cast<uint32_t*>(o)[e] = 0x7fc00000u;
        }
        return;
    }
    const long long cu = share_of(plan_total(a.plan, lane), a.plan.waves);
    const int L = plan_len(a.plan, b);
    const int nl = lat_units(L, a.w), nw = win_units(L, a.w);
    const int x = g * a.tiles + hg / tile;
    const long long pair = (long long)b * a.plan.pairs + x;
    const long long a0 = plan_base(a.plan, b, lane) + (long long)x * (nl + nw), a1 = a0 + nl, a2 = a1 + nw;
    const long long il = a0 / cu, iw = a1 / cu;
    const int cl = nl ? (int)((a1 - 1) / cu - il) + 1 : 0, cw = nw ? (int)((a2 - 1) / cu - iw) + 1 : 0;
    const int n = cl + cw, hr = (hg % tile) * (2 + d);
    auto rec = [&](int i) {
        return (i < cl ? record(a.part, il + i, pair, 0, tile, d) : record(a.part, iw + (i - cl), pair, 1, tile, d)) + hr;
    };
    float M = -INFINITY;
    for (int i = tid; i < n; i += 256) M = fmaxf(M, rec(i)[0]);
    M = wave_max(M);
    if (lane == 0) red[wv] = M;
    __syncthreads();
    M = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    __syncthreads();
    float l = 0.f;
    // columns: threads of a group of cwid take a column each, the groups take turns
    // at the records
    float lat = 0.f, win = 0.f;
    const int cwid = d <= 64 ? 64 : (d <= 128 ? 128 : 256);
    const int grp = tid / cwid, ngrp = 256 / cwid, col = tid - grp * cwid;
    const int lwid = dd <= 16 ? 16 : (dd <= 32 ? 32 : cwid);
    const int lgrp = tid / lwid, nlgrp = 256 / lwid, lcol = tid - lgrp * lwid;
    for (int i0 = 0; i0 < n; i0 += kMost) {
        const int ni = imin(kMost, n - i0);
        for (int i = tid; i < ni; i += 256) {
            const float* r = rec(i0 + i);
            // (an empty record, by its bits: the build assumes that no comparison
            // meets a NaN, and a reference may be one)
            const bool empty = __float_as_uint(r[0]) == 0xff800000u;
            const float f = empty ? 0.f : exp2f(r[0] - M);
            wt[i] = f;
            if (!empty) l += f * r[1];
        }
        __syncthreads();
        const int ml = imin(imax(cl - i0, 0), ni);
        if (lcol < dd)
            for (int i = lgrp; i < ml; i += nlgrp) {
                const float f = wt[i];
                if (__float_as_uint(f) != 0u) lat = __builtin_fmaf(f, rec(i0 + i)[2 + lcol], lat);
            }
        if (col < d)
            for (int i = ml + grp; i < ni; i += ngrp) {
                const float f = wt[i];
                if (__float_as_uint(f) != 0u) win = __builtin_fmaf(f, rec(i0 + i)[2 + col], win);
            }
        __syncthreads();
    }
    l = wave_sum(l);
    if (lane == 0) red[wv] = l;
    sum[0][tid] = lat;
    sum[1][tid] = win;
    __syncthreads();
    l = red[0] + red[1] + red[2] + red[3];
    if (tid < dd) {
        float s = 0.f;
        for (int k = 0; k < nlgrp; ++k) s += sum[0][k * lwid + tid];
        out[tid] = s;
    }
    __syncthreads();
    if (tid < d) {
        float s = 0.f;
        for (int k = 0; k < ngrp; ++k) s += sum[1][k * cwid + tid];
        if (cl) {
            const T* wdg = (const T*)a.wd + (size_t)g * d * dd + (size_t)tid * dd;
            const T* wug = a.wu ? (const T*)a.wu + (size_t)g * dd * d + tid : nullptr;
            for (int c = 0; c < dd; ++c)
                s = __builtin_fmaf(out[c], elem<T>::load(wug ? wug + (size_t)c * d : wdg + c), s);
        }
        o[tid] = elem<T>::from_f32(s / l);
    }
}

int tile_of(const dar_shape* s) {
    (void)s;
    return kVecTile;
}

template <typename T>
hipError_t launch_decode_q4(const dar_shape* s, DecodeArgs a, hipStream_t st) {
    const int tile = tile_of(s);
    long long waves = kWaves;
    if (!a.plan.lens) {
        const long long total = (long long)s->B * a.plan.pairs * seq_units(a.plan.len, s->w);
        waves = (total + share_of(total, kWaves) - 1) / share_of(total, kWaves);
    }
    const int wgs = (int)((waves + 3) / 4);
    hipLaunchKernelGGL(q4_vec_kernel<T>, dim3(wgs), dim3(256), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(q4_merge_kernel<T>, dim3(s->B * s->Hq), dim3(256), 0, st, a, tile);
    return hipGetLastError();
}

dar_status decode_q4(const dar_shape* s, const Q4Rows& rows, const int* lens, int len, void* const (&arrays)[6],
                     const void* q, const void* w_down, const void* w_up, void* o, void* ws,
                     size_t ws_bytes, hipStream_t stream) {
    if (!q4_dev_ok(q) || !q4_dev_ok(w_down) || !q4_dev_ok(o)) return DAR_E_ARG;
    if (w_up && !q4_dev_ok(w_up)) return DAR_E_ARG;
    const size_t need = dar_decode_q4_workspace_bytes(s, rows.cap);
    if (ws == nullptr || ws_bytes < need) return DAR_E_WORKSPACE;
    if (!q4_dev_ok(ws)) return DAR_E_ARG;
    (void)hipGetLastError();
    const int tile = tile_of(s), tiles = (s->Hq / s->Hkv + tile - 1) / tile;
    DecodeArgs a{q, w_down, w_up, arrays[0], arrays[1],
                 {(const uint8_t*)arrays[2], (const uint8_t*)arrays[3]},
                 {(const uint8_t*)arrays[4], (const uint8_t*)arrays[5]},
                 (float*)ws, o, rows, Plan{lens, len, rows.cap, s->w, s->B, s->Hkv * tiles, kWaves},
                 s->Hq, s->Hkv, s->d, s->d_down, s->w, tiles, 0.f};
    a.qscale = (float)(1.4426950408889634 / __builtin_sqrt((double)s->d));
    const hipError_t e = s->dtype == DAR_BF16 ? launch_decode_q4<bf16_t>(s, a, stream)
                                              : launch_decode_q4<float>(s, a, stream);
    return e == hipSuccess ? DAR_OK : DAR_E_HIP;
}

}  // namespace

}  // namespace dar

using namespace dar;

extern "C" {

size_t dar_decode_q4_workspace_bytes(const dar_shape* s, int cap) {
    if (q4_check_shape(s) != DAR_OK || cap < 1 || cap > kQ4MaxTokens) return 0;
    const int tile = tile_of(s), tiles = (s->Hq / s->Hkv + tile - 1) / tile;
    const size_t segments = (size_t)kWaves + 2 * (size_t)s->B * s->Hkv * tiles;
    return (segments * record_floats(tile, s->d) * sizeof(float) + 255) & ~(size_t)255;
}

dar_status dar_attn_decode_q4(const dar_shape* s, const dar_cache_q4* c, const void* q,
                              const void* w_down, const void* w_up, void* o, void* ws,
                              size_t ws_bytes, hipStream_t stream) {
    dar_status st = q4_check_shape(s);
    if (st != DAR_OK) return st;
    st = q4_check_cache(s, c);
    if (st != DAR_OK) return st;
    if (c->len < 1) return DAR_E_ARG;
    return decode_q4(s, q4_rows(c), nullptr, c->len,
                     {c->k_win, c->v_win, c->k_codes, c->v_codes, c->k_exp, c->v_exp}, q, w_down, w_up,
                     o, ws, ws_bytes, stream);
}

dar_status dar_attn_decode_paged_q4(const dar_shape* s, const dar_paged_cache_q4* c, const void* q,
                                    const void* w_down, const void* w_up, void* o, void* ws,
                                    size_t ws_bytes, hipStream_t stream) {
    dar_status st = q4_check_shape(s);
    if (st != DAR_OK) return st;
    st = q4_check_paged(s, c);
    if (st != DAR_OK) return st;
    return decode_q4(s, q4_rows(c), c->lens, 0,
                     {c->k_win, c->v_win, c->k_codes, c->v_codes, c->k_exp, c->v_exp}, q, w_down, w_up,
                     o, ws, ws_bytes, stream);
}

}  // extern "C"
