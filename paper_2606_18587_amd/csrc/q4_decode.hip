// Decode over a cache whose distant latents are held in 4 bits
// (include/dar_q4.h): Eq. 3-4 for one query a sequence, the distant tokens as
// they stand in the cache, the window at full dimension, one softmax over both.
//
// Work split. Every (sequence, KV head, tile of query heads) pair has two regions,
// its distant tokens in blocks of 128 and its window in steps of 32 tokens. Laid
// end to end in units of about the same bytes (one a block, win_units a step) all
// regions of the batch form one line, which the wavefronts of the launch share
// evenly, wherever the cuts fall; the line is computed on the device from the
// sequences' lengths, so ragged batches are balanced as dense ones are (but for batches
// of few units a pair, which take one workgroup each: launch_decode_q4). A wavefront's
// piece of a region is a segment: it leaves one record {m, l, acc} per query head, with m the reference of its exponentials (log2
// units), l their sum and acc the weighted sum of values (of latents where
// distant). q4_merge_kernel joins the records of a query head and lifts the
// latent part once, o = (acc_win + acc_lat W_up) / l.
#include "mfma_common.hpp"
#include "q4.hpp"

#include <type_traits>

namespace dar {

namespace {

constexpr int kBlock = 128;     // distant tokens a unit
constexpr int kStep = 32;       // window tokens a step
constexpr int kSimds = 1024;
constexpr int kWaves = 3 * kSimds;  // wavefronts that share a batch, at most
constexpr int kMaxTile = 8;     // query heads of a tile, at most

// --- the line of units ---------------------------------------------------------

struct Plan {
    const int* lens;  // NULL: every sequence holds len
    int len, cap, w, B;
    int pairs;      // (KV head, tile) pairs a sequence
    int waves;
    int win_units;  // units a window step counts for
    int least;      // units a wavefront takes at least
};

// Units are numbered in 32 bits (the entry points refuse what does not fit).
__host__ __device__ inline int held(int len, int cap) { return len < 0 ? 0 : (len > cap ? cap : len); }
__host__ __device__ inline uint32_t lat_units(int L, int w) { return L > w ? ((uint32_t)(L - w) + kBlock - 1) / kBlock : 0; }
__host__ __device__ inline uint32_t win_units(int L, const Plan& p) {
    return ((uint32_t)(L < p.w ? L : p.w) + kStep - 1) / kStep * p.win_units;
}
__host__ __device__ inline uint32_t seq_units(int L, const Plan& p) { return lat_units(L, p.w) + win_units(L, p); }
// units of a wavefront
__host__ __device__ inline uint32_t share_of(uint32_t total, const Plan& p) {
    const uint32_t cu = (total + p.waves - 1) / p.waves;
    return cu > (uint32_t)p.least ? cu : (uint32_t)p.least;
}

__device__ __forceinline__ int plan_len(const Plan& p, int b) { return p.lens ? held(p.lens[b], p.cap) : p.len; }

// All units of the batch.
__device__ __forceinline__ uint32_t plan_total(const Plan& p, int lane) {
    if (!p.lens) return (uint32_t)p.B * p.pairs * seq_units(p.len, p);
    uint32_t t = 0;
    for (int b = lane; b < p.B; b += 64) t += seq_units(plan_len(p, b), p);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) t += (uint32_t)__shfl_xor((int)t, off, 64);
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)t) * p.pairs;
}

// The sequence that unit u (< total) lies in, and its first unit.
__device__ __forceinline__ int plan_find(const Plan& p, uint32_t u, int lane, uint32_t& base) {
    if (!p.lens) {
        const uint32_t per = (uint32_t)p.pairs * seq_units(p.len, p);
        const uint32_t b = u / per;
        base = b * per;
        return (int)b;
    }
    uint32_t before = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        uint32_t x = b0 + lane < p.B ? (uint32_t)p.pairs * seq_units(plan_len(p, b0 + lane), p) : 0;
        const uint32_t mine = x;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t y = (uint32_t)__shfl_up((int)x, off, 64);
            if (lane >= off) x += y;
        }
        const unsigned long long past = __builtin_amdgcn_ballot_w64(before + x > u);
        if (past) {
            const int at = __builtin_ctzll(past);
            base = before + (uint32_t)__builtin_amdgcn_readlane((int)(x - mine), at);
            return b0 + at;
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
    }
    base = before;
    return p.B;  // not reached for u < total
}

// The reference that goes into a record. Where every score was NaN none was set, and
// a sum that is NaN is to be met all the same: 0 stands for it. (By its bits: the build
// assumes that no comparison meets a NaN.)
__device__ __forceinline__ float reference_of(float m, float l) {
    return (__float_as_uint(l) & 0x7fffffffu) > 0x7f800000u ? 0.f : m;
}

// Records. A segment's number grows along the line, by the wavefront and by the
// region: 2 pair + (window) + wavefront is unique.
__host__ __device__ inline size_t record_floats(int tile, int d) { return (size_t)tile * (2 + d); }
__device__ __forceinline__ float* record(float* part, uint32_t wave, uint32_t pair, int win, int tile, int d) {
    return part + (size_t)(wave + 2 * pair + win) * record_floats(tile, d);
}

struct DecodeArgs {
    const void *q, *wd, *wu, *k_win, *v_win;
    const uint8_t *codes[2], *exps[2];
    float* part;
    uint32_t* info;  // paged: [0] the units of a wavefront, [1 + b] the first unit of sequence b
    void* o;
    Q4Rows rows;
    Plan plan;
    int Hq, Hkv, d, dd, w, tiles;
    int fuse;  // a workgroup a pair, which finishes it
    float qscale;
};

// Where a head's records lie.
struct Records {
    const float *lat, *win;  // the first of each region
    int n_lat, n_win;
    size_t lat_step, win_step;
};

// False where the sequence has no query position.
__device__ __forceinline__ bool find_records(const DecodeArgs& a, int tile, int b, int h, Records& r) {
    int L = a.plan.len;
    if (a.plan.lens) {
        L = a.plan.lens[b];
        if (L < 1) return false;
        L = imin(L, a.plan.cap);
    }
    const int G = a.Hq / a.Hkv, g = h / G, hg = h - g * G;
    const uint32_t nl = lat_units(L, a.w), nw = win_units(L, a.plan);
    const uint32_t x = g * a.tiles + hg / tile, pair = b * a.plan.pairs + x;
    uint32_t cu, a0;
    if (a.plan.lens) {  // (left by the wavefronts that met them)
        cu = a.info[0];
        a0 = a.info[1 + b] + x * (nl + nw);
    } else {
        cu = share_of((uint32_t)a.plan.B * a.plan.pairs * (nl + nw), a.plan);
        a0 = pair * (nl + nw);
    }
    const uint32_t a1 = a0 + nl, a2 = a1 + nw;
    const uint32_t il = a0 / cu, iw = a1 / cu;
    r.n_lat = nl ? (int)((a1 - 1) / cu - il) + 1 : 0;
    r.n_win = nw ? (int)((a2 - 1) / cu - iw) + 1 : 0;
    r.lat_step = r.win_step = record_floats(tile, a.d);
    r.lat = record(a.part, il, pair, 0, tile, a.d) + (hg % tile) * (2 + a.d);
    r.win = record(a.part, iw, pair, 1, tile, a.d) + (hg % tile) * (2 + a.d);
    return true;
}

template <typename T>
__device__ __forceinline__ void store_nan(T* o, int d, int from, int by) {
    for (int e = from; e < d; e += by) {
        if (sizeof(T) == 2) reinterpret_cast<uint16_t*>(o)[e] = 0x7fc0;
        else reinterpret_cast<uint32_t*>(o)[e] = 0x7fc00000u;
    }
}

// A wavefront's joined records: lane's columns lane, lane + 64, ..
template <int R, int U>
struct Joined {
    float m = -INFINITY, l = 0.f, lat[R] = {}, win[R] = {};

    // records first + i step, i = from, from + by, .. below count, into acc; the lane's
    // columns col, col + 64, ..
    __device__ __forceinline__ void take(const float* first, size_t step, int count, int from, int by, int col,
                                         int width, float (&acc)[R]) {
        for (int i0 = 0; i0 < count; i0 += by * U) {
            float rm[U], rl[U], v[U][R];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float* r = first + (size_t)imin(i0 + from + u * by, count - 1) * step;
                rm[u] = r[0];
                rl[u] = r[1];
#pragma unroll
                for (int k = 0; k < R; ++k) v[u][k] = r[2 + imin(col + 64 * k, width - 1)];
            }
            float M = m;
#pragma unroll
            for (int u = 0; u < U; ++u) M = fmaxf(M, rm[u]);
            const float f = m == -INFINITY ? 0.f : exp2f(m - M);
            m = M;
            l *= f;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                lat[k] *= f;
                win[k] *= f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                // (an empty record by its bits: the build assumes that no comparison meets a
                // NaN, and a reference may be one)
                const bool none = i0 + from + u * by >= count || __float_as_uint(rm[u]) == 0xff800000u;
                const float w = none ? 0.f : exp2f(rm[u] - M);
                l = none ? l : __builtin_fmaf(w, rl[u], l);
#pragma unroll
                for (int k = 0; k < R; ++k) acc[k] = none ? acc[k] : __builtin_fmaf(w, v[u][k], acc[k]);
            }
        }
    }

    // Wavefront wv's share (of nw wavefronts) of a head's records.
    __device__ __forceinline__ void take_all(const Records& r, int d, int dd, int wv, int nw, int lane) {
        // distant records: few columns, so several side by side in a wavefront
        const int lw = dd <= 16 ? 16 : dd <= 32 ? 32 : 64, side = 64 / lw, sub = lane / lw;
        take(r.lat, r.lat_step, r.n_lat, wv * side + sub, nw * side, lane - sub * lw, dd, lat);
        for (int off = lw; off < 64; off <<= 1) {
            const float m2 = __shfl_xor(m, off, 64), l2 = __shfl_xor(l, off, 64), lat2 = __shfl_xor(lat[0], off, 64);
            const float M = fmaxf(m, m2);
            const float f1 = __float_as_uint(m) == 0xff800000u ? 0.f : exp2f(m - M);
            const float f2 = __float_as_uint(m2) == 0xff800000u ? 0.f : exp2f(m2 - M);
            l = f1 * l + f2 * l2;
            lat[0] = f1 * lat[0] + f2 * lat2;
            m = M;
        }
        take(r.win, r.win_step, r.n_win, wv, nw, lane, d, win);
    }
};

// W_up's columns of a lane, the first kAhead rows requested at once; then the lift
// and the output of a wavefront's head. out: d_down floats of LDS.
template <typename T, int R>
struct Lift {
    static constexpr int kAhead = 16;
    const T* from;
    int sc, d, dd;
    float wup[kAhead][R];

    __device__ __forceinline__ float at(int c, int k, int lane) const {
        return elem<T>::load(from + (size_t)c * sc + (size_t)imin(lane + 64 * k, d - 1) * (sc == 1 ? dd : 1));
    }
    __device__ __forceinline__ Lift(const DecodeArgs& a, int g, int lane) : sc(a.wu ? a.d : 1), d(a.d), dd(a.dd) {
        from = a.wu ? (const T*)a.wu + (size_t)g * dd * d : (const T*)a.wd + (size_t)g * d * dd;
#pragma unroll
        for (int c = 0; c < kAhead; ++c)
#pragma unroll
            for (int k = 0; k < R; ++k) wup[c][k] = at(imin(c, dd - 1), k, lane);
    }
    template <int U>
    __device__ __forceinline__ void finish(Joined<R, U>& j, float* out, T* o, int lane) const {
        wave_lds_order();
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (lane + 64 * k < dd) out[lane + 64 * k] = j.lat[k];
        wave_lds_order();
#pragma unroll
        for (int c = 0; c < kAhead; ++c)
#pragma unroll
            for (int k = 0; k < R; ++k)
                if (c < dd) j.win[k] = __builtin_fmaf(out[c], wup[c][k], j.win[k]);
#pragma unroll 8
        for (int c = kAhead; c < dd; ++c)
#pragma unroll
            for (int k = 0; k < R; ++k) j.win[k] = __builtin_fmaf(out[c], at(c, k, lane), j.win[k]);
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (lane + 64 * k < d) o[lane + 64 * k] = elem<T>::from_f32(j.win[k] / j.l);
    }
};

// The end of a fused pair: four wavefronts have left their records in LDS (lat + w
// lat_step, win + w win_step floats for wavefront w; a head's lrow, wrow floats apart),
// and take its heads in turn.
template <typename T, int R>
__device__ __forceinline__ void finish_pair(const DecodeArgs& a, int tile, const float* lat, size_t lat_step, int lrow,
                                            const float* win, size_t win_step, int wrow, float* out, int lane, int wv) {
    const int pair = wg_id_x(), b = pair / a.plan.pairs, x = pair - b * a.plan.pairs;
    const int g = x / a.tiles, h0 = (x - g * a.tiles) * tile, G = a.Hq / a.Hkv;
    const int nh = imin(tile, G - h0);
    const Lift<T, R> lift(a, g, lane);
    __syncthreads();
    for (int h = wv; h < nh; h += 4) {
        T* o = (T*)a.o + ((size_t)b * a.Hq + (size_t)g * G + h0 + h) * a.d;
        if (a.plan.lens && a.plan.lens[b] < 1) {
            store_nan(o, a.d, lane, 64);
            continue;
        }
        const Records r{lat + h * lrow, win + h * wrow, 4, 4, lat_step, win_step};
        Joined<R, 4> j;
        j.take_all(r, a.d, a.dd, 0, 1, lane);
        lift.finish(j, out, o, lane);
    }
}

// Walks the segments of wavefront `wave`: seg(b, x, L, win, lo, hi) for units [lo,
// hi) of region `win` of pair x of sequence b, which holds L tokens. fuse: workgroup i
// has pair i to itself, a quarter of its units a wavefront.
template <typename F>
__device__ __forceinline__ void walk(const Plan& p, uint32_t* info, bool fuse, uint32_t wave, int lane, F&& seg) {
    uint32_t u, end, base;
    int b;
    if (fuse) {
        const uint32_t pair = wave / 4;
        b = (int)(pair / p.pairs);
        const uint32_t nu = seq_units(__builtin_amdgcn_readfirstlane(plan_len(p, b)), p), cu = (nu + 3) / 4;
        base = 0;
        u = (pair - b * p.pairs) * nu;
        end = u + nu;
        u += wave % 4 * cu;
        end = u + cu < end ? u + cu : end;
    } else {
        const uint32_t total = plan_total(p, lane), cu = share_of(total, p);
        if (p.lens && wave == 0 && lane == 0) info[0] = cu;
        if ((unsigned long long)wave * cu >= total) return;
        u = wave * cu;
        end = total - u > cu ? u + cu : total;
        b = plan_find(p, u, lane, base);
    }
    while (u < end && b < p.B) {
        const int L = __builtin_amdgcn_readfirstlane(plan_len(p, b));
        const uint32_t nl = lat_units(L, p.w), nu = nl + win_units(L, p);
        if (nu == 0 || u - base >= nu * p.pairs) {
            base += nu * p.pairs;
            ++b;
            continue;
        }
        if (!fuse && p.lens && u == base && lane == 0) info[1 + b] = base;
        const uint32_t x = (u - base) / nu, off = (u - base) - x * nu;
        const int win = off >= nl;
        const uint32_t lo = win ? off - nl : off, size = win ? nu - nl : nl;
        const uint32_t hi = end - u < size - lo ? lo + (end - u) : size;
        // (the same in every lane: kept in scalar registers)
        seg(__builtin_amdgcn_readfirstlane(b), __builtin_amdgcn_readfirstlane((int)x), L, __builtin_amdgcn_readfirstlane(win),
            __builtin_amdgcn_readfirstlane((int)lo), __builtin_amdgcn_readfirstlane((int)hi));
        u += hi - lo;
    }
}

// --- any shape, on the vector ALU ----------------------------------------------
//
// Reached where the matrix cores are not: fp32, other head sizes and bottlenecks.
// 64 tokens at a time, a lane a token for the scores. The weights pass through
// LDS to the values, which meet them by columns: distant ones a group of 32
// columns at a time, brought to fp32 by the lanes of their tokens (half a
// wavefront then takes half the tokens each), window ones straight from the ring.
// Bounded by the chain of steps of a segment, which in small batches is 128 tokens:
// absorption, dot products, exponentials, products, each waiting for the one before
// (fp32, 4 x 4001 tokens of 4 KV heads, d80 d_down20: 20 us; its 4.4 MB would take one).

constexpr int kVecTile = 4;

// A head's product, summed in four parts: a chain of fp32 sums as long as a row would
// leave more error than the plain forms' (fp32, 4 x 4001 tokens, d80 d_down20, against
// fp64: up to 1.0e-6 in one chain, 3.6e-7 to 5.4e-7 so, plain forms 7.6e-7 to 9.0e-7;
// 17 and 20 us).
struct Parts {
    float p[kVecTile][4] = {};
    __device__ __forceinline__ void add(int h, int i, float a, float b) { p[h][i & 3] = __builtin_fmaf(a, b, p[h][i & 3]); }
    __device__ __forceinline__ float sum(int h) const { return (p[h][0] + p[h][1]) + (p[h][2] + p[h][3]); }
};

// Group j of 32 columns of a lane's token, key and value.
struct VecRow {
    uint32_t k[4], v[4];
    int ke, ve;
};

template <typename T>
__global__ __launch_bounds__(256) void q4_vec_kernel(DecodeArgs a) {
    __shared__ __attribute__((aligned(16))) float qsh[4][kVecTile][256];
    __shared__ __attribute__((aligned(16))) float psh[4][64][kVecTile];
    __shared__ float vsh[4][64][33];
    const int lane = lane_id_x() & 63;
    const int wv = __builtin_amdgcn_readfirstlane(lane_id_x() >> 6);
    const uint32_t wave = (uint32_t)wg_id_x() * 4 + wv;
    const int G = a.Hq / a.Hkv, d = a.d, dd = a.dd;
    const int nw = q4_row_bytes(dd) / 4, ng = q4_groups(dd);
    float(*qs)[256] = qsh[wv];
    float(*ps)[kVecTile] = psh[wv];
    float(*vs)[33] = vsh[wv];

    walk(a.plan, a.info, false, wave, lane, [&](int b, int x, int L, int win, int lo, int hi) {
        const int g = x / a.tiles, h0 = (x - g * a.tiles) * kVecTile;
        const int nh = imin(kVecTile, G - h0);
        const int bg = b * a.Hkv + g;
        const int n_lat = L > a.w ? L - a.w : 0;
        const int wu = a.plan.win_units;
        // tokens [t0, t1) of the sequence
        const int t0 = win ? n_lat + (lo + wu - 1) / wu * kStep : lo * kBlock;
        const int t1 = win ? imin(L, n_lat + (hi + wu - 1) / wu * kStep)
                           : (int)((long long)hi * kBlock < n_lat ? hi * kBlock : n_lat);
        float* rec = record(a.part, wave, (uint32_t)(b * a.plan.pairs + x), win, kVecTile, d);
        if (t0 >= t1) {  // no step of the window begins in this share
            for (int i = lane; i < kVecTile * (2 + d); i += 64) rec[i] = i % (2 + d) ? 0.f : -INFINITY;
            return;
        }
        // group j of the token's row (clamped to the segment; an unmapped page: zeros)
        auto row_of = [&](int i) { return q4_row(a.rows, b, g, a.Hkv, imin(t0 + i, t1 - 1)); };
        auto load = [&](long long row, int j) {
            VecRow r;
            const size_t at = (size_t)(row < 0 ? 0 : row);
            const uint32_t* kc = (const uint32_t*)a.codes[0] + at * nw + 4 * j;
            const uint32_t* vc = (const uint32_t*)a.codes[1] + at * nw + 4 * j;
            const int last = imin(nw - 4 * j, 4) - 1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                r.k[i] = kc[imin(i, last)];
                r.v[i] = vc[imin(i, last)];
            }
            r.ke = a.exps[0][at * ng + j];
            r.ve = a.exps[1][at * ng + j];
            return r;
        };
        long long row = 0;
        VecRow cur{};
        if (!win) {  // (requested ahead of the absorption)
            row = row_of(lane);
            cur = load(row, 0);
        }
        // queries in log2 units: as they are, or absorbed, q W_up^T
        const T* q0 = (const T*)a.q + ((size_t)b * a.Hq + (size_t)g * G + h0) * d;
        wave_lds_order();
        for (int c = lane; c < 256; c += 64)
#pragma unroll
            for (int h = 0; h < kVecTile; ++h)
                qs[h][c] = c < d && h < nh ? elem<T>::load(q0 + h * d + c) * (win ? a.qscale : 1.f) : 0.f;
        wave_lds_order();
        if (!win) {
            const T* wdg = (const T*)a.wd + (size_t)g * d * dd;
            const T* wug = a.wu ? (const T*)a.wu + (size_t)g * dd * d : nullptr;
            float s[4][kVecTile];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int c = imin(lane + 64 * r, dd - 1);
                const T* wp = wug ? wug + (size_t)c * d : wdg + c;
                const int step = wug ? 1 : dd;
                Parts sum;
                if (64 * r < dd) {
                    // (past d: the last element, against zeros)
#pragma unroll 4
                    for (int e = 0; e < d; e += 4)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float up = elem<T>::load(wp + (size_t)imin(e + i, d - 1) * step);
#pragma unroll
                            for (int h = 0; h < kVecTile; ++h) sum.add(h, i, qs[h][e + i], up);
                        }
                }
#pragma unroll
                for (int h = 0; h < kVecTile; ++h) s[r][h] = sum.sum(h);
            }
            wave_lds_order();
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int h = 0; h < kVecTile; ++h) qs[h][lane + 64 * r] = lane + 64 * r < dd ? s[r][h] * a.qscale : 0.f;
            wave_lds_order();
        }
        float m[kVecTile], l[kVecTile];
#pragma unroll
        for (int h = 0; h < kVecTile; ++h) {
            m[h] = -INFINITY;
            l[h] = 0.f;
        }
        // references and weights of 64 scores a head; f: what the sums so far are
        // multiplied with
        auto weights = [&](const float (&s)[kVecTile], bool live, float (&f)[kVecTile]) {
            float p[kVecTile];
#pragma unroll
            for (int h = 0; h < kVecTile; ++h) {
                const float mx = fmaxf(m[h], wave_max(live ? s[h] : -INFINITY));
                const float ref = mx == -INFINITY ? 0.f : mx;  // (every score -inf; NaN scores stay NaN)
                f[h] = m[h] == -INFINITY ? 0.f : exp2f(m[h] - ref);
                p[h] = live ? exp2f(s[h] - ref) : 0.f;
                l[h] = l[h] * f[h] + p[h];
                m[h] = mx;
            }
            wave_lds_order();
            *reinterpret_cast<float4*>(ps[lane]) = make_float4(p[0], p[1], p[2], p[3]);
            wave_lds_order();
        };
        auto store_ml = [&]() {
#pragma unroll
            for (int h = 0; h < kVecTile; ++h) {
                const float ls = wave_sum(l[h]);
                if (lane == 0) {
                    rec[h * (2 + d)] = reference_of(m[h], ls);
                    rec[h * (2 + d) + 1] = ls;
                }
            }
        };

        if (win) {
            const T* kw = (const T*)a.k_win + (size_t)bg * a.w * d;
            const T* vw = (const T*)a.v_win + (size_t)bg * a.w * d;
            const int s0 = t0 % a.w;
            auto slot = [&](int i) {  // of token t0 + i (clamped to the last; i < w, one wrap at most)
                const int s = s0 + imin(i, t1 - 1 - t0);
                return s >= a.w ? s - a.w : s;
            };
            constexpr int VE = 16 / sizeof(T);  // elements of a 16-byte load
            const bool wide = d % VE == 0;
            float acc[kVecTile][4] = {};
            for (int i0 = 0; i0 < t1 - t0; i0 += 64) {
                const T* k = kw + (size_t)slot(i0 + lane) * d;
                Parts sum;
                if (wide) {
#pragma unroll 8
                    for (int e = 0; e < d; e += VE) {
                        const uint4 u = *reinterpret_cast<const uint4*>(k + e);
                        const uint32_t w4[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int i = 0; i < VE; ++i) {
                            const float kv = sizeof(T) == 4 ? __uint_as_float(w4[i % 4])
                                             : __uint_as_float(i & 1 ? w4[i / 2] & 0xffff0000u : w4[i / 2] << 16);
#pragma unroll
                            for (int h = 0; h < kVecTile; ++h) sum.add(h, i, kv, qs[h][e + i]);
                        }
                    }
                } else {
                    // (past d: the last element, against zeros)
#pragma unroll 2
                    for (int e = 0; e < d; e += 4)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float kv = elem<T>::load(k + imin(e + i, d - 1));
#pragma unroll
                            for (int h = 0; h < kVecTile; ++h) sum.add(h, i, kv, qs[h][e + i]);
                        }
                }
                const float s[kVecTile] = {sum.sum(0), sum.sum(1), sum.sum(2), sum.sum(3)};
                float f[kVecTile];
                weights(s, t0 + i0 + lane < t1, f);
#pragma unroll
                for (int h = 0; h < kVecTile; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[h][r] *= f[h];
                const int nt = imin(64, t1 - t0 - i0);
                auto values = [&](auto columns) {  // of the lane: R, 64 apart
                    constexpr int R = decltype(columns)::value;
#pragma unroll 8
                    for (int i = 0; i < nt; ++i) {
                        const float4 p = *reinterpret_cast<const float4*>(ps[i]);
                        const T* row = vw + (size_t)slot(i0 + i) * d;
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            const float v = elem<T>::load(row + imin(lane + 64 * r, d - 1));
                            acc[0][r] = __builtin_fmaf(p.x, v, acc[0][r]);
                            acc[1][r] = __builtin_fmaf(p.y, v, acc[1][r]);
                            acc[2][r] = __builtin_fmaf(p.z, v, acc[2][r]);
                            acc[3][r] = __builtin_fmaf(p.w, v, acc[3][r]);
                        }
                    }
                };
                if (d <= 64) values(std::integral_constant<int, 1>{});
                else if (d <= 128) values(std::integral_constant<int, 2>{});
                else values(std::integral_constant<int, 4>{});
            }
            store_ml();
#pragma unroll
            for (int h = 0; h < kVecTile; ++h)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (lane + 64 * r < d) rec[h * (2 + d) + 2 + lane + 64 * r] = acc[h][r];
            return;
        }

        const int col = lane & 31, half = lane >> 5;
        float acc[kVecTile][8] = {};
        for (int i0 = 0; i0 < t1 - t0; i0 += 64) {
            // the next tokens' first group, while these are worked on
            const long long next_row = row_of(i0 + 64 + lane);
            const VecRow next = load(next_row, 0);
            Parts sum;
            for (int j = 0; j < ng; ++j) {
                const VecRow r = j ? load(row, j) : cur;
                const float sc = row < 0 ? 0.f : q4_scale(r.ke);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (4 * j + i >= nw) break;
                    float v[8];
                    q4_values_f32(row < 0 ? 0u : r.k[i], sc, v);
#pragma unroll
                    for (int h = 0; h < kVecTile; ++h) {
                        const float4 qa = *reinterpret_cast<const float4*>(&qs[h][32 * j + 8 * i]);
                        const float4 qb = *reinterpret_cast<const float4*>(&qs[h][32 * j + 8 * i + 4]);
                        sum.add(h, 0, v[0], qa.x);
                        sum.add(h, 1, v[1], qa.y);
                        sum.add(h, 2, v[2], qa.z);
                        sum.add(h, 3, v[3], qa.w);
                        sum.add(h, 0, v[4], qb.x);
                        sum.add(h, 1, v[5], qb.y);
                        sum.add(h, 2, v[6], qb.z);
                        sum.add(h, 3, v[7], qb.w);
                    }
                }
            }
            const float s[kVecTile] = {sum.sum(0), sum.sum(1), sum.sum(2), sum.sum(3)};
            float f[kVecTile];
            weights(s, t0 + i0 + lane < t1, f);
            const int nt = imin(64, t1 - t0 - i0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= ng) break;
#pragma unroll
                for (int h = 0; h < kVecTile; ++h) acc[h][j] *= f[h];
                const VecRow r = j ? load(row, j) : cur;
                const float sc = row < 0 ? 0.f : q4_scale(r.ve);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (4 * j + i >= nw) break;
                    float v[8];
                    q4_values_f32(row < 0 ? 0u : r.v[i], sc, v);
#pragma unroll
                    for (int c = 0; c < 8; ++c) vs[lane][8 * i + c] = v[c];
                }
                wave_lds_order();
                // (columns past the row's words: what another row left there, not stored)
#pragma unroll 8
                for (int i = half; i < nt; i += 2) {
                    const float4 p = *reinterpret_cast<const float4*>(ps[i]);
                    const float v = vs[i][col];
                    acc[0][j] = __builtin_fmaf(p.x, v, acc[0][j]);
                    acc[1][j] = __builtin_fmaf(p.y, v, acc[1][j]);
                    acc[2][j] = __builtin_fmaf(p.z, v, acc[2][j]);
                    acc[3][j] = __builtin_fmaf(p.w, v, acc[3][j]);
                }
                wave_lds_order();
            }
            row = next_row;
            cur = next;
        }
        store_ml();
#pragma unroll
        for (int h = 0; h < kVecTile; ++h)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = acc[h][j] + __shfl_xor(acc[h][j], 32, 64);
                if (half == 0 && 32 * j + col < dd) rec[h * (2 + d) + 2 + 32 * j + col] = v;
            }
    });
}

// --- bf16, d 64 or 128, d_down 16 or 32: the matrix cores -----------------------
//
// v_mfma_f32_16x16x32_bf16, lane l (n = l % 16, r4 = l / 16): A row n, contraction
// 8 r4 + 0..7; B column n, the same contraction; accumulator rows 4 r4 + 0..3 of
// column n.
//
// Distant tokens, 128 a block, in two sets of 64: lane l brings token l of a set,
// whole rows in 16-byte loads, and turns its codes into bf16 with the row's own
// scale (v_cvt_scalef32_pk_bf16_fp4: exact). The rows a set's lanes hold are the A
// operand as they stand, if the contraction's four parts of 8 are taken for four
// tokens: B then carries octet o of the absorbed query of head h in column 4 j + h,
// part j, and zeros in the other parts, and summed over the octets of a row
// column 4 j + h has the scores of tokens 16 j + 0..15 for head h. So one wavefront's
// exponentials cover four heads and no lane is idle; with one column a head,
// three quarters of them would be.
//   The values meet the weights the other way round: O^T = V^T P^T, the scores'
// registers of the two sets being the B operand (contraction 8 r4 + i: set i / 4,
// token 4 r4 + i % 4 of the column's own part j). A is V^T of part j, from the
// codes in LDS through ds_read_b64_tr_b4 (a lane gets one column of 16 tokens),
// one product for each j, of which column 4 j + h is the one that counts. V's
// scales, different along the contraction, go into the weights.
//   The absorbed query and the scaled weights are pairs of bf16 (16 bits): rounded
// to one, each would add as much error to the output as its own rounding does.
//
// The exponentials' reference of a column moves only when a score exceeds it by
// kTau; it enters the scores as the accumulator's start.
//
// Bounded by HBM in batches: B32 Hq32 Hkv8 32768 tokens, d64 d_down16 w512, 37 us for
// 182 MB, 4.9 TB/s with the microseconds until the first blocks arrive (the 16-bit
// decode, 3.1 times the bytes, streams 6.1); ragged and paged, 1024 to 16384 tokens, d128
// d_down32 w1024, 39 us for 176 MB, 4.5 TB/s. One sequence of 524287 tokens, 4 KV heads
// of 8 query heads, d128 d_down32: 26 us where its 73 MB take 11, by the products and
// vector operations of eight heads a row (two sets of columns) and the absorption, which
// each of 2048 wavefronts does for itself, though a workgroup's four mostly share a pair.

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2_t lds_i32x2_t;
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

constexpr float kTau = 8.f;

__device__ __forceinline__ f32x4_t mma16(bf16x8_t a, bf16x8_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t splat4(float x) { return f32x4_t{x, x, x, x}; }
__device__ __forceinline__ bf16x8_t as_bf16x8(uint4 u) { return __builtin_bit_cast(bf16x8_t, u); }

// Eight fp32 as a bf16 operand, and what the rounding leaves as another.
__device__ __forceinline__ void split8v(const float (&v)[8], bf16x8_t& hi, bf16x8_t& lo) {
    uint32_t h[4], r[4];
    // (the rest of a value in one operation: v - hi as a dot product with the pair; the
    // constants through registers: as literals of the instruction this compiler encodes
    // {-1, 0} as {0, -1})
    uint32_t c0 = 0x0000bf80u, c1 = 0xbf800000u;
    __asm__("" : "+s"(c0), "+s"(c1));
    const bf16x2_t m0 = __builtin_bit_cast(bf16x2_t, c0), m1 = __builtin_bit_cast(bf16x2_t, c1);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        h[k] = pack2(v[2 * k], v[2 * k + 1]);
        const bf16x2_t p = __builtin_bit_cast(bf16x2_t, h[k]);
        r[k] = pack2(__builtin_amdgcn_fdot2_f32_bf16(p, m0, v[2 * k], false),
                     __builtin_amdgcn_fdot2_f32_bf16(p, m1, v[2 * k + 1], false));
    }
    hi = as_bf16x8(make_uint4(h[0], h[1], h[2], h[3]));
    lo = as_bf16x8(make_uint4(r[0], r[1], r[2], r[3]));
}

// The reference, sum and accumulators of a column.
struct Column {
    float m = -INFINITY, l = 0.f;
    float most = -INFINITY;                // scores past this move the reference
    f32x4_t start = {0.f, 0.f, 0.f, 0.f};  // -m (0 where none is set): what a score starts from
};

// Moves the references of the columns whose scores x (relative to the present
// ones, 0 where none is set) exceed them by kTau; wave-uniform and rare.
template <int NX, int NACC>
__device__ __forceinline__ void move_reference(Column& c, float (&x)[NX], f32x4_t (&acc)[NACC]) {
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < NX; ++i) mx = fmaxf(mx, x[i]);
    if (__builtin_amdgcn_ballot_w64(mx > c.most)) {
        __asm__ volatile("");  // (the branch stays one)
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const bool fresh = c.m == -INFINITY, move = mx > c.most;
        const float delta = move ? mx : 0.f;
        const float f = move ? (fresh ? 0.f : exp2f(-mx)) : 1.f;
        c.m = move ? (fresh ? mx : c.m + mx) : c.m;
        c.most = move ? kTau : c.most;
        c.start = splat4(c.m == -INFINITY ? 0.f : -c.m);
        c.l *= f;
#pragma unroll
        for (int i = 0; i < NX; ++i) x[i] -= delta;
#pragma unroll
        for (int k = 0; k < NACC; ++k) acc[k] *= f;
    }
}

// Wavefronts a SIMD that the registers are held to (waves_of launches as many). A
// wavefront has one block in flight beside the one it works on; two and three take the
// third wavefront's registers and gain nothing (compared in an earlier state of this
// kernel, B32 Hkv8 d64 d_down16, 32768 tokens: 35.3 us with one, 36.2 and 36.5 with two
// and three; d128 d_down32 ragged: 40.6, 42.6, 43.5).
template <int D, int DD, int NS>
struct Held {
    static constexpr int waves = NS == 2 && (DD == 32 || D == 128) ? 2 : 3;
};

// One block's rows of a lane: two tokens.
template <int DD>
struct Rows4 {
    static constexpr int N = DD / 16;  // 16-byte loads (DD = 16: two tokens in one)
    u32x4_t k[N], v[N];
    uint32_t ks[N], vs[N];  // scale bytes as loaded (DD = 16: of both tokens)
    bool ok[N];             // paged: the page is mapped
};

template <int D, int DD, int NS, bool PAGED>
__global__ __launch_bounds__(256, (Held<D, DD, NS>::waves)) void q4_mfma_kernel(DecodeArgs a) {
    constexpr int HT = 4 * NS, CT = DD / 16, OC = DD / 8, KS = D / 32, DT = D / 16;
    constexpr int LDW = D + 8;  // padded row of the window's values in LDS
    constexpr int RB = DD / 2;
    constexpr int kStage = 32 * LDW * 2;  // bytes: window values; W_down; codes of 128 values
    static_assert(kStage >= D * DD * 2 && kStage >= 128 * RB + 512, "what else the buffer holds");
    __shared__ __attribute__((aligned(16))) uint8_t lds[4][kStage];
    __shared__ __attribute__((aligned(16))) float qlds[4][HT][DD];
    // fused: the records of the distant tokens; the window's take the wavefront's buffer
    __shared__ __attribute__((aligned(16))) float lrec[4][HT][2 + DD];
    static_assert(kStage >= HT * (2 + D) * 4 && sizeof(qlds[0]) >= DD * sizeof(float), "a record, a head's latents");
    const int lane = lane_id_x() & 63;
    const int wv = __builtin_amdgcn_readfirstlane(lane_id_x() >> 6);
    const uint32_t wave = (uint32_t)wg_id_x() * 4 + wv;
    const int n = lane & 15, r4 = lane >> 4, j4 = (lane >> 2) & 3, h4 = lane & 3;
    const int G = a.Hq / a.Hkv;
    uint8_t* buf = lds[wv];
    bf16_t* vb = reinterpret_cast<bf16_t*>(buf);
    float(*qs)[DD] = qlds[wv];

    bool met_lat = false, met_win = false;
    walk(a.plan, a.info, a.fuse, wave, lane, [&](int b, int x, int L, int win, int lo, int hi) {
        const int g = x / a.tiles, h0 = (x - g * a.tiles) * HT;
        const int nh = imin(HT, G - h0);
        const int bg = b * a.Hkv + g;
        const int n_lat = L > a.w ? L - a.w : 0;
        float* const rec = record(a.part, wave, (uint32_t)(b * a.plan.pairs + x), win, HT, D);
        met_lat = met_lat || !win;
        met_win = met_win || win;
        // query rows as a B operand: column n is head n
        const bf16_t* qrow = (const bf16_t*)a.q + ((size_t)b * a.Hq + (size_t)g * G + h0 + imin(n, nh - 1)) * D;
        bf16x8_t qop[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) qop[s] = load_bf16x8(qrow + 32 * s + 8 * r4);

        if (win) {
            const int wu = a.plan.win_units;
            const int p0 = n_lat + (lo + wu - 1) / wu * kStep;
            const int p1 = imin(L, n_lat + (hi + wu - 1) / wu * kStep);
#pragma unroll
            for (int s = 0; s < KS; ++s)
                if (n >= nh) qop[s] = zero_bf16x8();
            const bf16_t* kw = (const bf16_t*)a.k_win + (size_t)bg * a.w * D;
            const bf16_t* vw = (const bf16_t*)a.v_win + (size_t)bg * a.w * D;
            const int s0 = __builtin_amdgcn_readfirstlane(p0 % a.w);
            // ring slot of position p0 + i (clamped to the last; i < w, one wrap at most)
            auto slot = [&](int i) {
                const int s = s0 + imin(i, p1 - 1 - p0);
                return s >= a.w ? s - a.w : s;
            };
            Column c;
            f32x4_t acc[DT];
#pragma unroll
            for (int t = 0; t < DT; ++t) acc[t] = splat4(0.f);
            // TW tokens at a time: 32, or 16 where the registers of 32 (d = 128: 64 of keys and
            // values) would cost a wavefront a SIMD; half the contraction is then empty
            constexpr int TW = D == 64 ? 32 : 16, NT = TW / 16;
            constexpr int LPR = D / 8, RPL = 64 / LPR, VL = TW / RPL;  // lanes a row, rows a load, loads
            bf16x8_t kr[NT][KS], vr[VL];
            auto load = [&](int i0) {
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const bf16_t* row = kw + (size_t)slot(i0 + 16 * i + n) * D + 8 * r4;
#pragma unroll
                    for (int s = 0; s < KS; ++s) kr[i][s] = load_bf16x8(row + 32 * s);
                }
#pragma unroll
                for (int k = 0; k < VL; ++k)
                    vr[k] = load_bf16x8(vw + (size_t)slot(i0 + RPL * k + lane / LPR) * D + 8 * (lane % LPR));
            };
            if (p0 < p1) load(0);
            for (int i0 = 0; i0 < p1 - p0; i0 += TW) {
                wave_lds_order();
#pragma unroll
                for (int k = 0; k < VL; ++k)
                    *reinterpret_cast<bf16x8_t*>(vb + (RPL * k + lane / LPR) * LDW + 8 * (lane % LPR)) = vr[k];
                float s[4 * NT];
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    f32x4_t t = splat4(0.f);
#pragma unroll
                    for (int k = 0; k < KS; ++k) t = mma16(kr[i][k], qop[k], t);
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[4 * i + r] = __builtin_fmaf(t[r], a.qscale, c.start[0]);
                }
                if (i0 + TW < p1 - p0) {
                    load(i0 + TW);
                } else {
#pragma unroll
                    for (int i = 0; i < 4 * NT; ++i)
                        if (p0 + i0 + 16 * (i >> 2) + 4 * r4 + (i & 3) >= p1) s[i] = -INFINITY;
                }
                move_reference(c, s, acc);
                float p[8] = {};
#pragma unroll
                for (int i = 0; i < 4 * NT; ++i) {
                    p[i] = __builtin_amdgcn_exp2f(s[i]);
                    c.l += p[i];
                }
                bf16x8_t ph, pl;
                split8v(p, ph, pl);
                wave_lds_order();
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    const bf16_t* src = vb + (4 * r4 + (n >> 2)) * LDW + 16 * t + 4 * (n & 3);
                    const s16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)src);
                    const uint2 u0 = __builtin_bit_cast(uint2, v0);
                    uint2 u1 = make_uint2(0, 0);
                    if constexpr (NT == 2)
                        u1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(src + 16 * LDW)));
                    const bf16x8_t vt = as_bf16x8(make_uint4(u0.x, u0.y, u1.x, u1.y));
                    acc[t] = mma16(vt, ph, acc[t]);
                    acc[t] = mma16(vt, pl, acc[t]);
                }
            }
            float l = c.l + __shfl_xor(c.l, 16, 64);
            l += __shfl_xor(l, 32, 64);
            auto put = [&](float* r) {
                if (n >= HT) return;
                r += n * (2 + D);
                if (r4 == 0) *reinterpret_cast<float2*>(r) = make_float2(reference_of(c.m, l), l);
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    float* o = r + 2 + 16 * t + 4 * r4;
                    *reinterpret_cast<float2*>(o) = make_float2(acc[t][0], acc[t][1]);
                    *reinterpret_cast<float2*>(o + 2) = make_float2(acc[t][2], acc[t][3]);
                }
            };
            // (either address space by itself: through one pointer the stores would be flat)
            if (a.fuse) {
                wave_lds_order();  // over the values
                put(reinterpret_cast<float*>(buf));
            } else {
                put(rec);
            }
            return;
        }

        // ---- distant tokens [t0, t1)
        const int t0 = lo * kBlock, t1 = (long long)hi * kBlock < n_lat ? hi * kBlock : n_lat;
        // W_up as the A operand (row: latent column, contraction: e); W_down's rows
        // pass through LDS, which transposes them
        const bf16_t* wup = a.wu ? (const bf16_t*)a.wu + (size_t)g * DD * D : nullptr;
        bf16x8_t wa[CT][KS];
        constexpr int WL = D * DD / 512;  // 16-byte loads of a lane
        if (wup) {
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int s = 0; s < KS; ++s) wa[t][s] = load_bf16x8(wup + (size_t)(16 * t + n) * D + 32 * s + 8 * r4);
        } else {
            const bf16_t* wdn = (const bf16_t*)a.wd + (size_t)g * D * DD;
            static_assert(WL <= CT * KS, "W_down's words fit the operand's registers");
#pragma unroll
            for (int k = 0; k < WL; ++k) wa[k / KS][k % KS] = load_bf16x8(wdn + (lane + 64 * k) * 8);
        }

        using R = Rows4<DD>;
        const size_t head = (size_t)bg * a.rows.cap;
        const int count = t1 - t0;
        const int nb = __builtin_amdgcn_readfirstlane(count * RB), ne = __builtin_amdgcn_readfirstlane((count + 3) & ~3);
        auto rsrc = [&](const uint8_t* p, int bytes) {
            const uint64_t u = (uint64_t)p;
            // (the builtin's result is signed: each half through 32 unsigned bits)
            const uint32_t lo32 = __builtin_amdgcn_readfirstlane((uint32_t)u);
            const uint32_t hi32 = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
            return __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)hi32 << 32 | lo32), (short)0, bytes, 0x00020000);
        };
        // dense: descriptors that end with the segment (what lies past it reads as 0)
        const __amdgpu_buffer_rsrc_t rk = rsrc(PAGED ? a.codes[0] : a.codes[0] + (head + t0) * RB, PAGED ? 0 : nb);
        const __amdgpu_buffer_rsrc_t rv = rsrc(PAGED ? a.codes[1] : a.codes[1] + (head + t0) * RB, PAGED ? 0 : nb);
        const __amdgpu_buffer_rsrc_t rke = rsrc(PAGED ? a.exps[0] : a.exps[0] + head + t0, PAGED ? 0 : ne);
        const __amdgpu_buffer_rsrc_t rve = rsrc(PAGED ? a.exps[1] : a.exps[1] + head + t0, PAGED ? 0 : ne);
        // paged: pages of the four quarters of a block, through the scalar cache (as
        // vector loads they would be waited for behind the rows in flight), and the
        // one of the lane's token k (DD = 16: 2 l, 2 l + 1; DD = 32: l, 64 + l)
        const int* bt = PAGED ? a.rows.bt + (size_t)b * a.rows.maxb : nullptr;
        auto token = [&](int i0, int k) {  // clamped to the segment
            return DD == 16 ? imin(t0 + i0 + 2 * lane, (t1 - 1) & ~1) : imin(t0 + i0 + lane + 64 * k, t1 - 1);
        };
        struct Pages { int a, b, c, d; };
        auto pages = [&](int i0) {
            auto at = [&](int i) {
                return *(const __attribute__((address_space(4))) int*)(bt + (imin(t0 + i, t1 - 1) >> a.rows.shift));
            };
            return Pages{at(i0), at(i0 + 32), at(i0 + 64), at(i0 + 96)};
        };
        auto page_of = [&](Pages pg, int k) {
            const int a = pg.a, b = pg.b, c = pg.c, d = pg.d;  // (values: of references the select is one of addresses)
            if constexpr (DD == 32) {
                const int lo = k ? c : a, hi = k ? d : b;
                return lane < 32 ? lo : hi;
            } else {
                const int lo = lane < 16 ? a : b, hi = lane < 48 ? c : d;
                return lane < 32 ? lo : hi;
            }
        };
        auto load = [&](R& x, int i0, const Pages& pg) {
            if constexpr (PAGED) {
                // (an unmapped page: rows of page 0 are requested, and dropped in block())
#pragma unroll
                for (int k = 0; k < R::N; ++k) {
                    const int page = page_of(pg, k);
                    x.ok[k] = page >= 0 && page < a.rows.n_pages;
                    const size_t row = (((size_t)(x.ok[k] ? page : 0) * a.Hkv + g) << a.rows.shift) +
                                       (token(i0, k) & ((1 << a.rows.shift) - 1));
                    x.k[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(a.codes[0] + row * RB));
                    x.v[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(a.codes[1] + row * RB));
                    if constexpr (DD == 16) {
                        x.ks[k] = *reinterpret_cast<const uint16_t*>(a.exps[0] + row);
                        x.vs[k] = *reinterpret_cast<const uint16_t*>(a.exps[1] + row);
                    } else {
                        x.ks[k] = a.exps[0][row];
                        x.vs[k] = a.exps[1][row];
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < R::N; ++k) {
                    x.k[k] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rk, i0 * RB + lane * 16 + 1024 * k, 0, 2));
                    x.v[k] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rv, i0 * RB + lane * 16 + 1024 * k, 0, 2));
                }
#pragma unroll
                for (int k = 0; k < R::N; ++k) {
                    if constexpr (DD == 16) {
                        x.ks[k] = __builtin_amdgcn_raw_buffer_load_b16(rke, i0 + 2 * lane, 0, 0);
                        x.vs[k] = __builtin_amdgcn_raw_buffer_load_b16(rve, i0 + 2 * lane, 0, 0);
                    } else {
                        x.ks[k] = __builtin_amdgcn_raw_buffer_load_b8(rke, i0 + 64 * k + lane, 0, 0);
                        x.vs[k] = __builtin_amdgcn_raw_buffer_load_b8(rve, i0 + 64 * k + lane, 0, 0);
                    }
                }
            }
        };
        // paged: the page numbers a block ahead of the rows
        R rows;
        Pages pg{};
        if constexpr (PAGED) pg = pages(0);
        load(rows, 0, pg);
        if constexpr (PAGED) pg = pages(kBlock);

        // ---- q~ = W_up q, in log2 units; octet o of head h4 + 4 s for the lanes of part
        // j4 = r4, zeros elsewhere, as bf16 pairs
        if (!wup) {
            wave_lds_order();
#pragma unroll
            for (int k = 0; k < WL; ++k) *reinterpret_cast<bf16x8_t*>(vb + (lane + 64 * k) * 8) = wa[k / KS][k % KS];
            wave_lds_order();
#pragma unroll
            for (int t = 0; t < CT; ++t)
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const bf16_t* src = vb + (32 * s + 8 * r4 + (n >> 2)) * DD + 16 * t + 4 * (n & 3);
                    const s16x4_t v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)src);
                    const s16x4_t v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(src + 4 * DD));
                    const uint2 u0 = __builtin_bit_cast(uint2, v0), u1 = __builtin_bit_cast(uint2, v1);
                    wa[t][s] = as_bf16x8(make_uint4(u0.x, u0.y, u1.x, u1.y));
                }
        }
#pragma unroll
        for (int t = 0; t < CT; ++t) {
            f32x4_t q = splat4(0.f);
#pragma unroll
            for (int s = 0; s < KS; ++s) q = mma16(wa[t][s], qop[s], q);
            if (n < HT)
                *reinterpret_cast<float4*>(&qs[n][16 * t + 4 * r4]) =
                    make_float4(q[0] * a.qscale, q[1] * a.qscale, q[2] * a.qscale, q[3] * a.qscale);
        }
        wave_lds_order();
        bf16x8_t bq[NS][OC][2];
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int o = 0; o < OC; ++o) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const float4 f = *reinterpret_cast<const float4*>(&qs[h4 + 4 * s][8 * o + i]);
                    v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
                }
                split8v(v, bq[s][o][0], bq[s][o][1]);
                if (j4 != r4) bq[s][o][0] = bq[s][o][1] = zero_bf16x8();
            }
        wave_lds_order();

        Column c[NS];
        f32x4_t acc[NS][4 * CT];
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int t = 0; t < 4 * CT; ++t) acc[s][t] = splat4(0.f);
        float* esc = reinterpret_cast<float*>(buf + 128 * RB);  // scales of the values
        // set u of a lane: its u-th token; token 16 j + i of a set lies at this place
        auto place = [&](int u, int i) { return DD == 16 ? 2 * i + u : 64 * u + i; };

        auto block = [&](R& x, int i0, auto&& refill) {
            if constexpr (PAGED) {
                bool all = x.ok[0];
                if constexpr (R::N == 2) all = all && x.ok[1];
                if (__builtin_amdgcn_ballot_w64(!all)) {
                    __asm__ volatile("");
#pragma unroll
                    for (int k = 0; k < R::N; ++k)
                        if (!x.ok[k]) {
                            x.k[k] = x.v[k] = u32x4_t{0, 0, 0, 0};
                            x.ks[k] = x.vs[k] = 0;
                        }
                }
            }
            const bool tail = i0 + kBlock > count;  // wave-uniform
            if (tail) {
                // scale bytes past the end may hold anything; four tokens share a row of
                // the scores' operand, and a NaN would reach all of them
                __asm__ volatile("");
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    if (i0 + place(u, lane) >= count) {
                        if constexpr (DD == 16) x.ks[0] &= u ? 0x00ffu : 0xff00u;
                        else x.ks[u % R::N] = 0;
                    }
            }
            // values to LDS as they are
            wave_lds_order();
#pragma unroll
            for (int k = 0; k < R::N; ++k) *reinterpret_cast<u32x4_t*>(buf + 1024 * k + 16 * lane) = x.v[k];
            // (their scales set by set, so that four consecutive tokens of a set lie
            // together)
            esc[lane] = q4_scale(x.vs[0] & 255);
            esc[64 + lane] = q4_scale(DD == 16 ? x.vs[0] >> 8 : x.vs[R::N - 1]);
            // scores
            float s[NS][8];
            f32x4_t t[NS][2];
#pragma unroll
            for (int h = 0; h < NS; ++h) t[h][0] = t[h][1] = c[h].start;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float ks = q4_scale(DD == 16 ? (x.ks[0] >> (8 * u)) & 255 : x.ks[u % R::N] & 255);
#pragma unroll
                for (int o = 0; o < OC; ++o) {
                    const uint32_t w = DD == 16 ? x.k[0][2 * u + o] : x.k[u % R::N][o];
                    const bf16x8_t ka = as_bf16x8(q4_values_bf16(w, ks));
#pragma unroll
                    for (int h = 0; h < NS; ++h) {
                        t[h][u] = mma16(ka, bq[h][o][0], t[h][u]);
                        t[h][u] = mma16(ka, bq[h][o][1], t[h][u]);
                    }
                }
            }
            refill();  // (the rows' registers are free)
#pragma unroll
            for (int h = 0; h < NS; ++h)
#pragma unroll
                for (int i = 0; i < 8; ++i) s[h][i] = t[h][i >> 2][i & 3];
            if (tail) {
                __asm__ volatile("");
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i0 + place(i >> 2, 16 * j4 + 4 * r4 + (i & 3)) >= count)
#pragma unroll
                        for (int h = 0; h < NS; ++h) s[h][i] = -INFINITY;
            }
            wave_lds_order();
            // scales of the tokens whose weights the lane has
            float vs[8];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float4 y = *reinterpret_cast<const float4*>(esc + 64 * u + 16 * j4 + 4 * r4);
                vs[4 * u] = y.x; vs[4 * u + 1] = y.y; vs[4 * u + 2] = y.z; vs[4 * u + 3] = y.w;
            }
            if (tail) {  // what lies past the end may hold any byte: no product with it
                __asm__ volatile("");
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i0 + place(i >> 2, 16 * j4 + 4 * r4 + (i & 3)) >= count) vs[i] = 0.f;
            }
            bf16x8_t ph[NS], pl[NS];
#pragma unroll
            for (int h = 0; h < NS; ++h) {
                move_reference(c[h], s[h], acc[h]);
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[i] = __builtin_amdgcn_exp2f(s[h][i]);
                    c[h].l += p[i];
                    p[i] *= vs[i];
                }
                split8v(p, ph[h], pl[h]);
            }
            // values: row 4 j + i of a lane group's 16 is token 16 j + 4 r4 + i of the set
            i32x2_t v[2][CT];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint8_t* src = buf + place(u, 16 * (n >> 2) + 4 * r4 + (n & 3)) * RB;
#pragma unroll
                for (int q = 0; q < CT; ++q) v[u][q] = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2_t*)(src + 8 * q));
            }
#pragma unroll
            for (int q = 0; q < CT; ++q) {
                auto part = [&](const int j, const uint32_t w0, const uint32_t w1, const auto half) {
                    constexpr int B0 = decltype(half)::value;
                    const bf16x8_t va = as_bf16x8(make_uint4(
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, 1.f, B0)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, 1.f, B0 + 1)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w1, 1.f, B0)),
                        __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w1, 1.f, B0 + 1))));
#pragma unroll
                    for (int h = 0; h < NS; ++h) {
                        f32x4_t& ac = acc[h][4 * q + j];
                        ac = mma16(va, ph[h], ac);
                        ac = mma16(va, pl[h], ac);
                    }
                };
                part(0, v[0][q][0], v[1][q][0], std::integral_constant<int, 0>{});
                part(1, v[0][q][0], v[1][q][0], std::integral_constant<int, 2>{});
                part(2, v[0][q][1], v[1][q][1], std::integral_constant<int, 0>{});
                part(3, v[0][q][1], v[1][q][1], std::integral_constant<int, 2>{});
            }
        };
        for (int i0 = 0; i0 < count; i0 += kBlock)
            block(rows, i0, [&]() {
                load(rows, i0 + kBlock, pg);
                if constexpr (PAGED) pg = pages(i0 + 2 * kBlock);
            });

        // ---- the record of a head: its four columns joined
        auto put = [&](float* first, const int rs) {  // rs: floats from head to head
#pragma unroll
            for (int h = 0; h < NS; ++h) {
                float l = c[h].l + __shfl_xor(c[h].l, 16, 64);
                l += __shfl_xor(l, 32, 64);
                float M = fmaxf(c[h].m, __shfl_xor(c[h].m, 4, 64));
                M = fmaxf(M, __shfl_xor(M, 8, 64));
                const float f = c[h].m == -INFINITY ? 0.f : exp2f(c[h].m - M);
                l *= f;
                l += __shfl_xor(l, 4, 64);
                l += __shfl_xor(l, 8, 64);
                float* r = first + (h4 + 4 * h) * rs;
                if (lane < 4) *reinterpret_cast<float2*>(r) = make_float2(reference_of(M, l), l);
#pragma unroll
                for (int q = 0; q < CT; ++q) {
                    float o[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float y = j4 == 0 ? acc[h][4 * q][i] : j4 == 1 ? acc[h][4 * q + 1][i]
                                  : j4 == 2 ? acc[h][4 * q + 2][i] : acc[h][4 * q + 3][i];
                        y *= f;
                        y += __shfl_xor(y, 4, 64);
                        o[i] = y + __shfl_xor(y, 8, 64);
                    }
                    if (j4 == 0) {
                        *reinterpret_cast<float2*>(r + 2 + 16 * q + 4 * r4) = make_float2(o[0], o[1]);
                        *reinterpret_cast<float2*>(r + 2 + 16 * q + 4 * r4 + 2) = make_float2(o[2], o[3]);
                    }
                }
            }
        };
        if (a.fuse) put(&lrec[wv][0][0], 2 + DD);
        else put(rec, 2 + D);
    });
    if (a.fuse) {
        wave_lds_order();
        if (lane < HT) {
            if (!met_lat) lrec[wv][lane][0] = -INFINITY;
            if (!met_win) reinterpret_cast<float*>(buf)[lane * (2 + D)] = -INFINITY;
        }
        finish_pair<bf16_t, D / 64>(a, HT, &lrec[0][0][0], HT * (2 + DD), 2 + DD, reinterpret_cast<const float*>(&lds[0][0]),
                                    kStage / 4, 2 + D, &qs[0][0], lane, wv);
    }
}

// Query heads of a batch, at most: pairs and heads are counted in 32 bits, and a grid
// holds 2^32 threads, 256 a pair.
constexpr long long kMaxHeads = 1 << 20;

dar_status check_decode(const dar_shape* s) {
    const dar_status st = q4_check_shape(s);
    if (st != DAR_OK) return st;
    return (long long)s->B * s->Hq > kMaxHeads ? DAR_E_UNSUPPORTED : DAR_OK;
}

bool on_matrix_cores(const dar_shape* s) {
    return s->dtype == DAR_BF16 && (s->d == 64 || s->d == 128) && (s->d_down == 16 || s->d_down == 32);
}

using Kernel = void (*)(DecodeArgs);
template <int D, int DD, int NS>
Kernel pick(bool paged) { return paged ? q4_mfma_kernel<D, DD, NS, true> : q4_mfma_kernel<D, DD, NS, false>; }
template <int D, int DD>
Kernel pick(int tile, bool paged) { return tile == 4 ? pick<D, DD, 1>(paged) : pick<D, DD, 2>(paged); }
Kernel pick(const dar_shape* s, int tile, bool paged) {
    if (s->d == 64) return s->d_down == 16 ? pick<64, 16>(tile, paged) : pick<64, 32>(tile, paged);
    return s->d_down == 16 ? pick<128, 16>(tile, paged) : pick<128, 32>(tile, paged);
}

// --- merge ---------------------------------------------------------------------
//
// The records of a query head's two regions: those of the wavefronts whose shares
// meet them (a record's reference is -inf, and its sums 0, where no window step
// began in the share). Bounded by round trips to memory and by instruction fetch,
// so records are requested U at a time with all they hold, and joined under a
// running reference. A sequence without a query position gets NaN. Measured: 6.5 us for
// 1024 heads of 12 records (B32 Hkv8 32768 tokens, wavefronts), 8 for as many of a
// ragged paged batch, 10.6 for 32 heads of 512 records (1024 threads).

// Few records a head (a batch): a wavefront a head, no barrier.
template <typename T, int R>
__global__ __launch_bounds__(256) void q4_merge_wave_kernel(DecodeArgs a, int tile, int heads) {
    __shared__ float outs[4][64 * R];
    const int lane = lane_id_x() & 63;
    const int wv = __builtin_amdgcn_readfirstlane(lane_id_x() >> 6);
    const int bh = wg_id_x() * 4 + wv;
    if (bh >= heads) return;
    const int b = bh / a.Hq, h = bh - b * a.Hq, g = h / (a.Hq / a.Hkv);
    const int d = a.d;
    T* o = (T*)a.o + (size_t)bh * d;
    const Lift<T, R> lift(a, g, lane);
    Records r;
    if (!find_records(a, tile, b, h, r)) return store_nan(o, d, lane, 64);
    Joined<R, 8> j;
    j.take_all(r, d, a.dd, 0, 1, lane);
    lift.finish(j, outs[wv], o, lane);
}

// Many records a head: a workgroup a head; its wavefronts' sums are joined through LDS.
template <typename T, int NT, int R>
__global__ __launch_bounds__(NT) void q4_merge_kernel(DecodeArgs a, int tile) {
    constexpr int NW = NT / 64;
    __shared__ float ms[NW], ls[NW], lats[NW][64 * R], wins[NW][64 * R], out[64 * R], part[NT];
    const int tid = lane_id_x(), lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int bh = wg_id_x(), b = bh / a.Hq, h = bh - b * a.Hq;
    const int g = h / (a.Hq / a.Hkv);
    const int d = a.d, dd = a.dd;
    T* o = (T*)a.o + (size_t)bh * d;
    Records r;
    if (!find_records(a, tile, b, h, r)) return store_nan(o, d, tid, NT);
    Joined<R, NT == 1024 ? 8 : 4> j;
    j.take_all(r, d, dd, wv, NW, lane);
    const float m = j.m, l = j.l;
    const float(&lat)[R] = j.lat, (&win)[R] = j.win;
    // W_up, requested ahead of the joins: thread (column col, part grp) takes latent
    // columns grp, grp + NG, ..
    constexpr int NG = NT / (64 * R), kAhead = 8;
    const int grp = tid / (64 * R), col = tid - grp * 64 * R;
    const T* wdg = (const T*)a.wd + (size_t)g * d * dd + (size_t)imin(col, d - 1) * dd;
    const T* wug = a.wu ? (const T*)a.wu + (size_t)g * dd * d + imin(col, d - 1) : nullptr;
    auto up = [&](int c) { return elem<T>::load(wug ? wug + (size_t)c * d : wdg + c); };
    float wup[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) wup[k] = grp + NG * k < dd ? up(grp + NG * k) : 0.f;
    if (lane == 0) {
        ms[wv] = m;
        ls[wv] = l;
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
        lats[wv][lane + 64 * k] = lat[k];
        wins[wv][lane + 64 * k] = win[k];
    }
    __syncthreads();
    float M = ms[0], f[NW], lsum = 0.f;
#pragma unroll
    for (int k = 1; k < NW; ++k) M = fmaxf(M, ms[k]);
#pragma unroll
    for (int k = 0; k < NW; ++k) {
        f[k] = __float_as_uint(ms[k]) == 0xff800000u ? 0.f : exp2f(ms[k] - M);
        lsum = __builtin_fmaf(f[k], ls[k], lsum);
    }
    float wsum = 0.f;
    if (tid < 64 * R) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NW; ++k) {
            s = __builtin_fmaf(f[k], lats[k][tid], s);
            wsum = __builtin_fmaf(f[k], wins[k][tid], wsum);
        }
        out[tid] = s;
    }
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (grp + NG * k < dd) s = __builtin_fmaf(out[grp + NG * k], wup[k], s);
#pragma unroll 4
    for (int c = grp + NG * kAhead; c < dd; c += NG) s = __builtin_fmaf(out[c], up(c), s);
    part[tid] = s;
    __syncthreads();
    if (tid < d) {
        s = wsum;
#pragma unroll
        for (int k = 0; k < NG; ++k) s += part[tid + 64 * R * k];
        o[tid] = elem<T>::from_f32(s / lsum);
    }
}

template <typename T, int NT>
hipError_t launch_merge(const dar_shape* s, const DecodeArgs& a, int tile, hipStream_t st) {
    auto kernel = s->d <= 64 ? q4_merge_kernel<T, NT, 1> : s->d <= 128 ? q4_merge_kernel<T, NT, 2> : q4_merge_kernel<T, NT, 4>;
    hipLaunchKernelGGL(kernel, dim3(s->B * s->Hq), dim3(NT), 0, st, a, tile);
    return hipGetLastError();
}

int tile_of(const dar_shape* s) { return on_matrix_cores(s) && s->Hq / s->Hkv > 4 ? kMaxTile : 4; }

size_t records_bytes(const dar_shape* s) {
    const int tile = tile_of(s), tiles = (s->Hq / s->Hkv + tile - 1) / tile;
    const size_t segments = (size_t)kWaves + 2 * (size_t)s->B * s->Hkv * tiles;
    return (segments * record_floats(tile, s->d) * sizeof(float) + 255) & ~(size_t)255;
}

// A window step's bytes against a block's.
int win_units_of(const dar_shape* s) {
    const int step = kStep * s->d * (s->dtype == DAR_BF16 ? 2 : 4);
    const int block = kBlock * (q4_row_bytes(s->d_down) + q4_groups(s->d_down));
    return step < block ? 1 : (step + block / 2) / block;
}

// Wavefronts that share the line: as many as the chip holds of the kernel.
int waves_of(const dar_shape* s) {
    if (!on_matrix_cores(s)) return 2 * kSimds;
    return tile_of(s) == 8 && (s->d_down == 32 || s->d == 128) ? 2 * kSimds : 3 * kSimds;
}

template <typename T>
hipError_t launch_decode_q4(const dar_shape* s, DecodeArgs a, hipStream_t st) {
    const int tile = tile_of(s);
    uint32_t waves = a.plan.waves;
    if (!a.plan.lens) {
        const uint32_t total = (uint32_t)s->B * a.plan.pairs * seq_units(a.plan.len, a.plan);
        waves = (total + share_of(total, a.plan) - 1) / share_of(total, a.plan);
    }
    // A pair of few units is a workgroup's, which finishes it: one launch, no records.
    // Up to 8 units a wavefront (8 pairs of 331 tokens: 9.3 us a call, 12.0 in two
    // launches; of 6000 tokens, 15: 14.4 and 12.2); 16 where the pairs give every
    // compute unit one (256 pairs of 4500 tokens, 12: 14.2 and 17.7; of 9000, 22: 20.4
    // and 20.1), 32 where they give it two (768 pairs of 9000 tokens: 32.6 and 39.8).
    // Paged, the lengths are not known here, and the units are a full sequence's: eight
    // sequences of some 330 tokens take 11.2 us under a table of 512 tokens and 13.9 under
    // one of 131072; 63 of some 300 and one of 8192, whose pairs' workgroups then work
    // alone, 20.3 in one launch and 21.1 shared out (d64 d_down16; d128 d_down32: 36.2 and
    // 36.6).
    const uint32_t units = seq_units(a.plan.lens ? a.plan.cap : a.plan.len, a.plan);
    const uint32_t pairs = (uint32_t)s->B * a.plan.pairs;
    a.fuse = on_matrix_cores(s) && units <= 4 * (pairs >= 512 ? 32u : pairs >= 256 ? 16u : 8u);
    if (a.fuse) waves = 4 * pairs;
    const int wgs = (int)((waves + 3) / 4);
    const Kernel kernel = on_matrix_cores(s) ? pick(s, tile, a.plan.lens != nullptr) : (Kernel)q4_vec_kernel<T>;
    hipLaunchKernelGGL(kernel, dim3(wgs), dim3(256), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.fuse) return e;
    // records a head, on average: a wavefront takes up to 24, sixteen take 128 and more
    if (waves / 24 < pairs) {
        const int heads = s->B * s->Hq;
        auto merge = s->d <= 64 ? q4_merge_wave_kernel<T, 1> : s->d <= 128 ? q4_merge_wave_kernel<T, 2> : q4_merge_wave_kernel<T, 4>;
        hipLaunchKernelGGL(merge, dim3((heads + 3) / 4), dim3(256), 0, st, a, tile, heads);
        return hipGetLastError();
    }
    return waves / 128 >= pairs ? launch_merge<T, 1024>(s, a, tile, st) : launch_merge<T, 256>(s, a, tile, st);
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
                 (float*)ws, (uint32_t*)((char*)ws + records_bytes(s)), o, rows, Plan{lens, len, rows.cap, s->w, s->B, s->Hkv * tiles, waves_of(s), win_units_of(s),
                      on_matrix_cores(s) ? 2 : 1},
                 s->Hq, s->Hkv, s->d, s->d_down, s->w, tiles, 0, 0.f};
    // (the line of a batch whose sequences are all full is numbered in 32 bits)
    if ((double)s->B * a.plan.pairs * seq_units(rows.cap, a.plan) > 2147483647.0) return DAR_E_UNSUPPORTED;
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
    if (check_decode(s) != DAR_OK || cap < 1 || cap > kQ4MaxTokens) return 0;
    return (records_bytes(s) + (1 + (size_t)s->B) * sizeof(uint32_t) + 255) & ~(size_t)255;
}

dar_status dar_attn_decode_q4(const dar_shape* s, const dar_cache_q4* c, const void* q,
                              const void* w_down, const void* w_up, void* o, void* ws,
                              size_t ws_bytes, hipStream_t stream) {
    dar_status st = check_decode(s);
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
    dar_status st = check_decode(s);
    if (st != DAR_OK) return st;
    st = q4_check_paged(s, c);
    if (st != DAR_OK) return st;
    return decode_q4(s, q4_rows(c), c->lens, 0,
                     {c->k_win, c->v_win, c->k_codes, c->v_codes, c->k_exp, c->v_exp}, q, w_down, w_up,
                     o, ws, ws_bytes, stream);
}

}  // extern "C"
