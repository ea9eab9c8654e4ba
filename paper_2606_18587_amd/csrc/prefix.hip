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
constexpr int kPfxPerCu = 8;  // wavefronts a compute unit: 12 fit, but more runs are more records to join
constexpr int kPfxMinSub = 8;  // subtiles a wavefront is given, at least

typedef unsigned int pu32x4 __attribute__((ext_vector_type(4)));
constexpr int kBufWord3 = 0x00020000;  // raw buffer, 32-bit data: reads past its size are zero

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
//
// 64 tokens a pass, two subtiles side by side (the products of one run under the
// exponentials of the other), the next pass in flight. Page numbers come a pass
// ahead through the scalar cache and rows through descriptors that end with
// them, so that no vector load waits for another: with a branch around the
// loads, or with page numbers kept in a vector register and fetched again now
// and then, the compiler waits for everything in flight once or twice a pass.
// The wavefronts of a workgroup take row tiles side by side over the same
// tokens, whose rows they find in the first-level cache.
template <int D, int DD, bool EXACT>
__global__ __launch_bounds__(64 * kPfxWaves, 3) void prefix_attn_kernel(
    const bf16_t* __restrict__ q, const bf16_t* __restrict__ wd, const bf16_t* __restrict__ wu,
    const bf16_t* __restrict__ k_pool, const bf16_t* __restrict__ v_pool,
    const int* __restrict__ blocks, const int* __restrict__ lens, float* __restrict__ ppart, int B,
    int Hq, int Hkv, int w, int cap, int n_prefix, int ps_shift, int n_pages, int nrt, int NS,
    int sub, float qscale) {
    constexpr int KS = D / 16, DS = DD / 16, NQ = EXACT ? 3 : 2;
    constexpr int LDW = D + 8;                     // W_up row in LDS
    constexpr int VB = 64 * DD;                    // two subtiles' values
    constexpr int WB = DD * LDW > D * DD + 16 ? DD * LDW : D * DD + 16;
    constexpr int BUF = VB > WB ? VB : WB;         // (the weights pass through it first)
    __shared__ __attribute__((aligned(16))) bf16_t vbuf[kPfxWaves][BUF + 8];
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
    const int quad = lane >> 4, sl = lane & 15;
    bf16_t* vb = vbuf[wave];

    // ---- the weights, the rows' queries and the first rows are requested at once
    constexpr int WV = DD * D / 512;
    pu32x4 wreg[WV];
    {
        const bf16_t* wsrc = wu ? wu + (size_t)g * DD * D : wd + (size_t)g * D * DD;
#pragma unroll
        for (int k = 0; k < WV; ++k) wreg[k] = *reinterpret_cast<const pu32x4*>(wsrc + (lane + 64 * k) * 8);
    }
    bf16x8_t qop[KS];
    {
        const bf16_t* qrow = q + bh * D;
#pragma unroll
        for (int k = 0; k < KS; ++k) qop[k] = load_bf16x8(qrow + 16 * k + 8 * hg);
    }
    const int n_blk = n_prefix >> ps_shift, ps = 1 << ps_shift;
    auto page_of = [&](int t0) {  // (past the prefix: some page, its rows are not read)
        return *(const __attribute__((address_space(4))) int*)(blocks + imin(t0 >> ps_shift, n_blk - 1));
    };
    int page[2] = {page_of(t_begin), page_of(t_begin + 32)};
    const int lim = rval ? imin(imax(imin(lens[b], cap) - w, 0), t_end) : 0;
    int lim_min = lim, lim_max = lim;
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) {
        lim_min = imin(lim_min, __shfl_xor(lim_min, off, 64));
        lim_max = imax(lim_max, __shfl_xor(lim_max, off, 64));
    }
    lim_min = __builtin_amdgcn_readfirstlane(lim_min);
    const int end = __builtin_amdgcn_readfirstlane(lim_max);  // nothing is seen past it

    // rows of the 32 tokens from t0 on (zeros past `end` and for no such page)
    const int koff = perm_row(col) * DD * 2 + hg * 16, voff = lane * 16;
    auto load = [&](int t0, int page, pu32x4 (&ak)[DS], pu32x4 (&vv)[DS]) {
        const bool ok = t0 < end && page >= 0 && page < n_pages;
        const size_t base = (((size_t)(ok ? page : 0) * Hkv + g) * ps + (t0 & (ps - 1))) * DD;
        const int nb = ok ? 32 * DD * 2 : 0;
        const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc((void*)(k_pool + base), (short)0, nb, kBufWord3);
        const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void*)(v_pool + base), (short)0, nb, kBufWord3);
#pragma unroll
        for (int k = 0; k < DS; ++k) {
            ak[k] = __builtin_amdgcn_raw_buffer_load_b128(rk, koff + 32 * k, 0, 0);
            vv[k] = __builtin_amdgcn_raw_buffer_load_b128(rv, voff + 1024 * k, 0, 0);
        }
    };
    pu32x4 ak[2][DS], vv[2][DS];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        load(t_begin + 32 * j, page[j], ak[j], vv[j]);
        page[j] = page_of(t_begin + 64 + 32 * j);
    }

    // ---- q~^T = W_up q^T of the 32 rows, scaled, as operands of 16 or 24 bits
#pragma unroll
    for (int k = 0; k < WV; ++k) {
        const int i = (lane + 64 * k) * 8;
        *reinterpret_cast<pu32x4*>(vb + (wu ? (i / D) * LDW + (i & (D - 1)) : i)) = wreg[k];
    }
    bf16x8_t qa[NQ][DS];
    {
        f32x16_t qt = splat16(0.f);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            // (operand rows past d_down: finite values of no use)
            bf16x8_t a;
            if (wu) {
                a = load_bf16x8(vb + (col & (DD - 1)) * LDW + 16 * k + 8 * hg);
            } else {
                const int e = 16 * k + 8 * (quad >> 1) + (sl >> 2);
                const int c = DD == 16 ? 4 * (sl & 3) : 16 * (quad & 1) + 4 * (sl & 3);
                const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(vb + e * DD + c));
                const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(vb + (e + 4) * DD + c));
                const uint2 ulo = __builtin_bit_cast(uint2, lo), uhi = __builtin_bit_cast(uint2, hi);
                a = __builtin_bit_cast(bf16x8_t, make_uint4(ulo.x, ulo.y, uhi.x, uhi.y));
            }
            qt = mfma(a, qop[k], qt);
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
    bf16_t* one = vb + BUF;  // [1, 0, 0, 0]: the row-sum column of the values' operand
    if (lane < 4) one[lane] = lane == 0 ? 0x3f80 : 0;

    // The reference m is a bf16 value, so that a rank-1 product subtracts it in
    // the scores' accumulators: 1 in contraction slot 0 of every token, -m there
    // of every row.
    float m = -INFINITY, thr = -INFINITY, l = 0.f;
    bf16x8_t negm = zero_bf16x8();
    const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, make_uint4(hg == 0 ? 0x3f80u : 0u, 0u, 0u, 0u));
    f32x16_t acc[2] = {splat16(0.f), splat16(0.f)};
    // (tokens past `end` are past every row's limit: whole passes need no tail)
    for (int t0 = t_begin; t0 < end; t0 += 64) {
        f32x16_t x[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int k = 0; k < DS; ++k) *reinterpret_cast<pu32x4*>(vb + j * 32 * DD + (lane + 64 * k) * 8) = vv[j][k];
            x[j] = mfma(ones, negm, splat16(0.f));
        }
#pragma unroll
        for (int p = 0; p < NQ; ++p)
#pragma unroll
            for (int k = 0; k < DS; ++k)
#pragma unroll
                for (int j = 0; j < 2; ++j) x[j] = mfma(__builtin_bit_cast(bf16x8_t, ak[j][k]), qa[p][k], x[j]);
        // the next pass's rows: their registers are free once the products are issued
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            load(t0 + 64 + 32 * j, page[j], ak[j], vv[j]);
            page[j] = page_of(t0 + 128 + 32 * j);
        }
        if (t0 + 64 > lim_min) {
            __asm__ volatile("");  // (a branch, not 32 selects for every pass)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (t0 + 32 * j + acc_row(r, hg) >= lim) x[j][r] = -INFINITY;
        }
        float mx[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            mx[j] = fmaxf(fmaxf(x[j][0], x[j][1]), x[j][2]);
#pragma unroll
            for (int r = 3; r < 15; r += 2) mx[j] = fmaxf(fmaxf(mx[j], x[j][r]), x[j][r + 1]);
        }
        const float top = pair_max(fmaxf(fmaxf(mx[0], x[0][15]), fmaxf(mx[1], x[1][15])));
        const bool need = top > thr;
        if (__builtin_amdgcn_ballot_w64(need)) {
            __asm__ volatile("");
            const bool fresh = m == -INFINITY;
            const float mnew = need ? bf16_up(fresh ? top : m + top) : m;
            const float delta = need ? (fresh ? mnew : mnew - m) : 0.f;
            const float fac = need ? (fresh ? 0.f : exp2f(-delta)) : 1.f;
            l *= fac;
            m = mnew;
            thr = m == -INFINITY ? -INFINITY : kTau;
            const uint32_t nb = m == -INFINITY ? 0u : __float_as_uint(-m) >> 16;
            negm = __builtin_bit_cast(bf16x8_t, make_uint4(hg == 0 ? nb : 0u, 0u, 0u, 0u));
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    acc[j][r] *= fac;
                    x[j][r] -= delta;
                }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int r = 0; r < 16; ++r) x[j][r] = __builtin_amdgcn_exp2f(x[j][r]);
            const bf16x8_t p[2] = {pack8(x[j], 0), pack8(x[j], 8)};
            if constexpr (EXACT) {
                float s0 = x[j][0], s1 = x[j][1];
#pragma unroll
                for (int r = 2; r < 16; r += 2) {
                    s0 += x[j][r];
                    s1 += x[j][r + 1];
                }
                l += s0 + s1;
            } else if constexpr (DD != 16) {
                const bf16x8_t u = __builtin_bit_cast(bf16x8_t, make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u));
                l = dot8(p[0], u, dot8(p[1], u, l));
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int key = 32 * j + half * 16 + 8 * (quad >> 1) + (sl >> 2);
                const int c = 16 * (quad & 1) + 4 * (sl & 3);
                const bool sumcol = DD == 16 && (quad & 1);
                const bf16_t* plo = sumcol ? one : vb + key * DD + c;
                const bf16_t* phi = sumcol ? one : vb + (key + 4) * DD + c;
                const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)plo);
                const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)phi);
                const uint2 ulo = __builtin_bit_cast(uint2, lo), uhi = __builtin_bit_cast(uint2, hi);
                acc[j] = mfma(__builtin_bit_cast(bf16x8_t, make_uint4(ulo.x, ulo.y, uhi.x, uhi.y)), p[half], acc[j]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[0][r] += acc[1][r];
    if (DD == 16 && !EXACT) l = acc[0][8];  // the constant column: row 16 on both halves' registers
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
            if (c < DD) rec[2 + c] = acc[0][r];
        }
    }
}

// Runs of the prefix that a row tile is cut into: as many wavefronts as the
// chip holds, runs of at least kPfxMinSub subtiles.
static int prefix_run(int B, int Hq, int Hkv, int n_prefix) {
    const long long nsub = n_prefix / 32;
    const long long tiles = (long long)Hkv * ((B * (Hq / Hkv) + 31) / 32);
    long long ns = (256 * kPfxPerCu + tiles - 1) / tiles;
    if (ns > kPfxMaxSplits) ns = kPfxMaxSplits;
    long long sub = (nsub + ns - 1) / ns;
    if (sub < kPfxMinSub) sub = kPfxMinSub;
    return (int)sub;
}

// Read by every sequence on its own, a prefix costs B times its bytes; read once,
// a launch and its records. Per sequence against once (Hkv8 d64 d_down16 G4, whole
// call): 2 x 512 tokens 16.8 and 20.0 us, 32 x 2048 (33.6 MB) 21.3 and 21.5, 64 x
// 2048 (67 MB) 28.6 and 24.4, 64 x 8192 59 and 27.
constexpr long long kPfxApartBytes = 32 << 20;
bool prefix_apart(int B, int Hkv, int dd, int n_prefix) {
    return n_prefix > 0 && 4ll * dd * n_prefix * B * Hkv > kPfxApartBytes;
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
