// Decode over a prefix that the sequences of a batch share (bf16, d in {64,
// 128}, d_down in {16, 32}): attention of every sequence's query heads over the
// prefix's latents, read once for all of them.
//
// With W_up absorbed, q~ = q W_up^T, the B G query heads that read a KV head are
// rows of one product S = Q~ C^T with the prefix's latents: a wavefront takes 32
// rows and walks a run of 32-token subtiles, the runs of one row tile being
// joined afterwards. Per subtile the scores are computed transposed (lane l
// owns row l % 32, tokens split between l and l ^ 32), so that the row maximum
// is a lane's own but for one exchange, and the scores' registers, the tokens
// read in a permuted order, are the operand of O^T += V^T P^T.
//
// Reading the prefix per sequence costs B times its bytes; read once, it is no
// longer memory that bounds the pass but one exponential per (row, token):
// 16 a lane and subtile, at a quarter of the vector rate.
#include "../../include/dar_serving.h"
#include "dar_common.hpp"
#include "dar_kernels.hpp"
#include "mfma_common.hpp"

namespace dar {

namespace {

constexpr int kPfxWaves = 4;
constexpr float kTau = 8.0f;  // the running reference moves when a score exceeds it by this (log2)
constexpr int kPfxMaxSplits = 64;
constexpr int kPfxMinSub = 8;  // subtiles a wavefront is given, at least

// bf16 value >= x: the fp32 pattern rounded up to 16 bits
__device__ __forceinline__ float bf16_up(float x) {
    uint32_t u = __float_as_uint(x);
    const uint32_t low = u & 0xffffu;
    u &= 0xffff0000u;
    if (low != 0) u += x > 0.f ? 0x10000u : 0u;
    return __uint_as_float(u);
}

}  // namespace

// blocks: the prefix's pages, n_prefix >> ps_shift of them. Row R = b G + j of KV
// head g is query head g G + j of sequence b; it sees prefix tokens below its own
// number of distant tokens (a sequence hardly longer than the prefix has some of
// them in its window). Record of each row and split: {m, l, acc[DD]}.
// EXACT: the absorbed query keeps 24 bits (three operands, else 16 in two) and
// row sums take p before its rounding to bf16: single weights are computed
// against them. Else the sum takes the rounded p that multiply the values.
template <int D, int DD, bool EXACT>
__global__ __launch_bounds__(64 * kPfxWaves) void prefix_attn_kernel(
    const bf16_t* __restrict__ q, const bf16_t* __restrict__ wd, const bf16_t* __restrict__ wu,
    const bf16_t* __restrict__ k_pool, const bf16_t* __restrict__ v_pool,
    const int* __restrict__ blocks, const int* __restrict__ lens, float* __restrict__ ppart, int B,
    int Hq, int Hkv, int w, int cap, int n_prefix, int ps_shift, int n_pages, int nrt, int NS,
    int sub, float qscale) {
    constexpr int KS = D / 16, DS = DD / 16, NQ = EXACT ? 3 : 2;
    constexpr int VBUF = 32 * DD;
    __shared__ __attribute__((aligned(16))) bf16_t vbuf[kPfxWaves][VBUF + 8];
    const int tid = lane_id_x(), lane = tid & 63, col = lane & 31, hg = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = wg_id_x() % Hkv, job = wg_id_x() / Hkv * kPfxWaves + wave;
    if (job >= nrt * NS) return;
    const int rt = job % nrt, sp = job / nrt;
    const int G = Hq / Hkv;
    const int t_begin = 32 * sub * sp, t_end = imin(t_begin + 32 * sub, n_prefix);
    const int R = 32 * rt + col;
    const bool rval = R < B * G;
    const int b = rval ? R / G : 0;
    const size_t bh = (size_t)b * Hq + (size_t)g * G + (rval ? R - b * G : 0);
    const int lim = rval ? imin(imax(imin(lens[b], cap) - w, 0), n_prefix) : 0;
    int lim_min = lim, lim_max = lim;
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) {
        lim_min = imin(lim_min, __shfl_xor(lim_min, off, 64));
        lim_max = imax(lim_max, __shfl_xor(lim_max, off, 64));
    }
    lim_min = __builtin_amdgcn_readfirstlane(lim_min);
    lim_max = __builtin_amdgcn_readfirstlane(lim_max);
    bf16_t* vb = vbuf[wave];
    if (lane < 4) vb[VBUF + lane] = lane == 0 ? 0x3f80 : 0;  // [1, 0, 0, 0]: the row-sum column

    const int prow = perm_row(col);
    const int ps = 1 << ps_shift;
    auto load = [&](int t0, bf16x8_t (&ak)[DS], uint4 (&vv)[DS]) {
        const int tc = imin(t0, n_prefix - 32);  // (past the run: loaded, not used)
        const int page = blocks[tc >> ps_shift];
        const bool ok = page >= 0 && page < n_pages;
        const size_t base = (((size_t)(ok ? page : 0) * Hkv + g) * ps + (tc & (ps - 1))) * DD;
#pragma unroll
        for (int k = 0; k < DS; ++k) {
            ak[k] = ok ? load_bf16x8(k_pool + base + prow * DD + 16 * k + 8 * hg) : zero_bf16x8();
            vv[k] = ok ? *reinterpret_cast<const uint4*>(v_pool + base + (lane + 64 * k) * 8)
                       : make_uint4(0, 0, 0, 0);
        }
    };
    bf16x8_t ak[2][DS];
    uint4 vv[2][DS];
    load(t_begin, ak[0], vv[0]);

    // q~^T = W_up q^T of the 32 rows, scaled, as operands of 16 or 24 bits
    bf16x8_t qa[NQ][DS];
    {
        const bf16_t* wdg = wd + (size_t)g * D * DD;
        const bf16_t* wug = wu ? wu + (size_t)g * DD * D : nullptr;
        const bf16_t* qrow = q + bh * D;
        f32x16_t qt = splat16(0.f);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            bf16x8_t a = zero_bf16x8();
            if (col < DD) {
                if (wug) {
                    a = load_bf16x8(wug + (size_t)col * D + 16 * k + 8 * hg);
                } else {
                    uint16_t t8[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) t8[j] = wdg[(size_t)(16 * k + 8 * hg + j) * DD + col];
                    a = __builtin_bit_cast(bf16x8_t, t8);
                }
            }
            qt = mfma(a, rval ? load_bf16x8(qrow + 16 * k + 8 * hg) : zero_bf16x8(), qt);
        }
#pragma unroll
        for (int k = 0; k < DS; ++k) {
            float v8[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(qt[8 * k + j]),
                                                          __float_as_uint(qt[8 * k + 4 + j]), false, false);
                v8[j] = __uint_as_float(r[0]) * qscale;
                v8[4 + j] = __uint_as_float(r[1]) * qscale;
            }
#pragma unroll
            for (int p = 0; p < NQ; ++p) {
                uint32_t h[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    h[j] = pack2(v8[2 * j], v8[2 * j + 1]);
                    v8[2 * j] -= __uint_as_float(h[j] << 16);
                    v8[2 * j + 1] -= __uint_as_float(h[j] & 0xffff0000u);
                }
                qa[p][k] = __builtin_bit_cast(bf16x8_t, make_uint4(h[0], h[1], h[2], h[3]));
            }
        }
    }

    // The reference m is a bf16 value, so that a rank-1 product subtracts it in
    // the scores' accumulators: 1 in contraction slot 0 of every token, -m there
    // of every row.
    float m = -INFINITY, thr = -INFINITY, l = 0.f;
    bf16x8_t negm = zero_bf16x8();
    const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, make_uint4(hg == 0 ? 0x3f80u : 0u, 0u, 0u, 0u));
    f32x16_t acc = splat16(0.f);
    const int quad = lane >> 4, sl = lane & 15;
    const int end = imin(t_end, lim_max);  // nothing is seen past it
    auto step = [&](int t0, const bf16x8_t (&a)[DS], const uint4 (&v)[DS]) {
#pragma unroll
        for (int k = 0; k < DS; ++k) *reinterpret_cast<uint4*>(vb + (lane + 64 * k) * 8) = v[k];
        f32x16_t x = mfma(ones, negm, splat16(0.f));
#pragma unroll
        for (int p = 0; p < NQ; ++p)
#pragma unroll
            for (int k = 0; k < DS; ++k) x = mfma(a[k], qa[p][k], x);
        if (t0 + 32 > lim_min) {
            __asm__ volatile("");  // (a branch, not 16 selects for every subtile)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (t0 + acc_row(r, hg) >= lim) x[r] = -INFINITY;
        }
        float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), x[2]), fmaxf(x[3], x[4]));
        mx = fmaxf(fmaxf(mx, x[5]), fmaxf(x[6], x[7]));
        mx = fmaxf(fmaxf(mx, x[8]), fmaxf(x[9], x[10]));
        mx = fmaxf(fmaxf(mx, x[11]), fmaxf(x[12], x[13]));
        mx = fmaxf(fmaxf(mx, x[14]), x[15]);
        mx = pair_max(mx);
        const bool need = mx > thr;
        if (__builtin_amdgcn_ballot_w64(need)) {
            __asm__ volatile("");
            const bool fresh = m == -INFINITY;
            const float mnew = need ? bf16_up(fresh ? mx : m + mx) : m;
            const float delta = need ? (fresh ? mnew : mnew - m) : 0.f;
            const float fac = need ? (fresh ? 0.f : exp2f(-delta)) : 1.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] *= fac;
            l *= fac;
            m = mnew;
            thr = m == -INFINITY ? -INFINITY : kTau;
            const uint32_t nb = m == -INFINITY ? 0u : __float_as_uint(-m) >> 16;
            negm = __builtin_bit_cast(bf16x8_t, make_uint4(hg == 0 ? nb : 0u, 0u, 0u, 0u));
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] -= delta;
        }
        f32x16_t p;
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(x[r]);
        const bf16x8_t p0 = pack8(p, 0), p1 = pack8(p, 8);
        if constexpr (EXACT) {
            float s0 = p[0], s1 = p[1];
#pragma unroll
            for (int r = 2; r < 16; r += 2) {
                s0 += p[r];
                s1 += p[r + 1];
            }
            l += s0 + s1;
        } else if constexpr (DD != 16) {
            const bf16x8_t one = __builtin_bit_cast(bf16x8_t, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
            l = dot8(p0, one, dot8(p1, one, l));
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int key = half * 16 + 8 * (quad >> 1) + (sl >> 2);
            const int c = 16 * (quad & 1) + 4 * (sl & 3);
            const bool sumcol = DD == 16 && (quad & 1);
            const bf16_t* plo = sumcol ? vb + VBUF : vb + key * DD + c;
            const bf16_t* phi = sumcol ? vb + VBUF : vb + (key + 4) * DD + c;
            const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)plo);
            const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)phi);
            const uint2 ulo = __builtin_bit_cast(uint2, lo), uhi = __builtin_bit_cast(uint2, hi);
            acc = mfma(__builtin_bit_cast(bf16x8_t, make_uint4(ulo.x, ulo.y, uhi.x, uhi.y)), half ? p1 : p0, acc);
        }
    };
    for (int t0 = t_begin; t0 < end; t0 += 64) {
        load(t0 + 32, ak[1], vv[1]);
        step(t0, ak[0], vv[0]);
        if (t0 + 32 >= end) break;
        load(t0 + 64, ak[0], vv[0]);
        step(t0 + 32, ak[1], vv[1]);
    }
    if (DD == 16 && !EXACT) l = acc[8];  // the constant column: row 16 on both halves' registers
    else l = pair_sum(l);
    if (rval) {
        float* rec = ppart + (bh * NS + sp) * (2 + DD);
        if (hg == 0) {
            rec[0] = m;
            rec[1] = l;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int c = 8 * (r >> 2) + 4 * hg + (r & 3);
            if (c < DD) rec[2 + c] = acc[r];
        }
    }
}

// Runs of the prefix that a row tile is cut into: about 16 wavefronts a compute
// unit over the whole grid, runs of at least kPfxMinSub subtiles.
static int prefix_run(int B, int Hq, int Hkv, int n_prefix) {
    const long long nsub = n_prefix / 32;
    const long long tiles = (long long)Hkv * ((B * (Hq / Hkv) + 31) / 32);
    long long ns = (256 * 16 + tiles - 1) / tiles;
    if (ns > kPfxMaxSplits) ns = kPfxMaxSplits;
    long long sub = (nsub + ns - 1) / ns;
    if (sub < kPfxMinSub) sub = kPfxMinSub;
    return (int)sub;
}

int prefix_splits(int B, int Hq, int Hkv, int n_prefix) {
    if (n_prefix <= 0) return 0;
    const int sub = prefix_run(B, Hq, Hkv, n_prefix);
    return (n_prefix / 32 + sub - 1) / sub;
}

hipError_t launch_prefix_attn(const bf16_t* q, const bf16_t* wd, const bf16_t* wu,
                              const bf16_t* k_pool, const bf16_t* v_pool, const int* blocks,
                              const PagedArgs& pg, float* ppart, int B, int Hq, int Hkv, int d, int dd,
                              int w, int n_prefix, bool exact, hipStream_t st) {
    const float qscale = 1.4426950408889634f / sqrtf((float)d);
    const int sub = prefix_run(B, Hq, Hkv, n_prefix), NS = prefix_splits(B, Hq, Hkv, n_prefix);
    const int nrt = (B * (Hq / Hkv) + 31) / 32;
    const dim3 grid(Hkv * ((nrt * NS + kPfxWaves - 1) / kPfxWaves));
#define DAR_PREFIX(D_, DD_, E_)                                                                    \
    hipLaunchKernelGGL((prefix_attn_kernel<D_, DD_, E_>), grid, dim3(64 * kPfxWaves), 0, st, q, wd, \
                       wu, k_pool, v_pool, blocks, pg.lens, ppart, B, Hq, Hkv, w, pg.maxb * pg.ps,  \
                       n_prefix, pg.ps_shift, pg.n_pages, nrt, NS, sub, qscale)
#define DAR_PREFIX_E(D_, DD_)              \
    if (exact) DAR_PREFIX(D_, DD_, true);  \
    else DAR_PREFIX(D_, DD_, false);
    if (d == 64 && dd == 16) { DAR_PREFIX_E(64, 16) }
    else if (d == 64 && dd == 32) { DAR_PREFIX_E(64, 32) }
    else if (d == 128 && dd == 16) { DAR_PREFIX_E(128, 16) }
    else { DAR_PREFIX_E(128, 32) }
#undef DAR_PREFIX_E
#undef DAR_PREFIX
    return hipGetLastError();
}

}  // namespace dar
