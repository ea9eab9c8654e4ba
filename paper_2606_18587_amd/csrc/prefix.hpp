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
// longer memory that bounds the pass but vector work per (row, token): an
// exponential at a quarter of the vector rate and about nine plain operations. Once
// is the better way where the prefix is long, and costs up to 14% where many
// sequences share a short one (Hq32 Hkv8 d64 d_down16, 64..256 own tokens, per
// sequence against once: 1 x 64 tokens 12.6 and 12.1 us, 2 x 512 15.2 and 12.1,
// 32 x 256 14.9 and 14.5, 32 x 2048 21.2 and 15.0, 64 x 8192 70.8 and 27.0; 64 x 64
// 17.8 and 19.9, 64 x 256 19.0 and 21.6; one head a group, 64 x 256 18.1 and 19.5,
// 64 x 1024 23.4 and 20.8).
//
// A part of the paged decode kernel: the workgroups of the prefix, bound by the
// vector ALU, and those of the sequences' own tokens, bound by memory, share a
// launch.
#pragma once

#include "dar_common.hpp"
#include "dar_kernels.hpp"
#include "mfma_common.hpp"

namespace dar {

constexpr int kPfxWaves = 4;
constexpr float kPfxTau = 8.0f;  // the running reference moves when a score exceeds it by this (log2)
typedef unsigned int pu32x4 __attribute__((ext_vector_type(4)));
constexpr int kPfxBufWord3 = 0x00020000;  // raw buffer, 32-bit data: reads past its size are zero

// bf16 elements of LDS that a wavefront needs: two subtiles' values, before them
// the weights (W_up's rows padded, or W_down).
template <int D, int DD>
struct PrefixLds {
    static constexpr int LDW = D + 8;
    static constexpr int WB = DD * LDW > D * DD + 16 ? DD * LDW : D * DD + 16;
    static constexpr int value = 64 * DD > WB ? 64 * DD : WB;
};

// blocks: the prefix's pages, n_prefix >> ps_shift of them. Row R = b G + j of KV
// head g is query head g G + j of sequence b; it sees prefix tokens below its own
// number of distant tokens (a sequence hardly longer than the prefix has some of
// them in its window). Record of each row and split: {m, l, acc[DD]}.
// As in the records mode of the own parts the absorbed query keeps 24 bits (three
// operands), row sums take p before its rounding to bf16, and the values meet p
// in two operands, 16 bits: single weights are computed against these sums, and
// with p rounded to 8 bits above a sum of unrounded ones the output was off by
// 2^-9 of every weight (B64 n_prefix 32768: 49 -> 56 us, error against fp64
// 0.0022 -> 0.0017).
//
// 64 tokens a pass, two subtiles side by side (the products of one run under the
// exponentials of the other), the next pass in flight. Page numbers come a pass
// ahead through the scalar cache and rows through descriptors that end with
// them, so that no vector load waits for another: with a branch around the
// loads, or with page numbers kept in a vector register and fetched again now
// and then, the compiler waits for everything in flight once or twice a pass.
// The wavefronts of a workgroup take row tiles side by side over the same
// tokens, whose rows they find in the first-level cache.
template <int D, int DD>
__device__ __forceinline__ void prefix_attn(const int wg, bf16_t* const vb, const bf16_t* __restrict__ q,
                                            const bf16_t* __restrict__ wd, const bf16_t* __restrict__ wu,
                                            const bf16_t* __restrict__ k_pool,
                                            const bf16_t* __restrict__ v_pool, const PagedArgs& pg,
                                            int Hq, int Hkv, int w, int cap, float qscale) {
    constexpr int KS = D / 16, DS = DD / 16, NQ = 3;
    constexpr int LDW = PrefixLds<D, DD>::LDW;
    const int* __restrict__ const blocks = pg.pfx_blocks;
    const int* __restrict__ const lens = pg.lens;
    const int B = pg.nseq, n_prefix = 32 * pg.pre, ps_shift = pg.ps_shift, n_pages = pg.n_pages;
    const int nrt = pg.pfx_tiles, NS = pg.pfx_splits, sub = pg.pfx_run;
    const int tid = lane_id_x(), lane = tid & 63, col = lane & 31, hg = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = wg % Hkv, job = wg / Hkv * kPfxWaves + wave;
    if (job >= nrt * NS) return;
    const int rt = job % nrt, sp = job / nrt;
    const int G = Hq / Hkv;
    const int t_begin = 32 * sub * sp, t_end = imin(t_begin + 32 * sub, n_prefix);
    const int R = 32 * rt + col;
    const bool rval = R < B * G;
    const int b = rval ? R / G : 0;
    const size_t bh = (size_t)b * Hq + (size_t)g * G + (rval ? R - b * G : 0);
    const int quad = lane >> 4, sl = lane & 15;

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

    // rows of the 32 tokens from t0 on (zeros past `end`, where the pool may hold
    // anything, and for no such page)
    const int koff = perm_row(col) * DD * 2 + hg * 16, voff = lane * 16;
    auto load = [&](int t0, int page, pu32x4 (&ak)[DS], pu32x4 (&vv)[DS]) {
        const bool ok = t0 < end && page >= 0 && page < n_pages;
        const size_t base = (((size_t)(ok ? page : 0) * Hkv + g) * ps + (t0 & (ps - 1))) * DD;
        const int nb = ok ? imin(32, end - t0) * DD * 2 : 0;
        const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc((void*)(k_pool + base), (short)0, nb, kPfxBufWord3);
        const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void*)(v_pool + base), (short)0, nb, kPfxBufWord3);
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

    // ---- q~^T = W_up q^T of the 32 rows, scaled, as operands of 24 bits
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
            const float mnew = need ? bf16_ceil(fresh ? top : m + top) : m;
            const float delta = need ? (fresh ? mnew : mnew - m) : 0.f;
            const float fac = need ? (fresh ? 0.f : exp2f(-delta)) : 1.f;
            l *= fac;
            m = mnew;
            thr = m == -INFINITY ? -INFINITY : kPfxTau;
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
            bf16x8_t p[2], rest[2];
            split8(x[j], 0, 1.f, p[0], rest[0]);
            split8(x[j], 8, 1.f, p[1], rest[1]);
            float s0 = x[j][0], s1 = x[j][1];
#pragma unroll
            for (int r = 2; r < 16; r += 2) {
                s0 += x[j][r];
                s1 += x[j][r + 1];
            }
            l += s0 + s1;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int key = 32 * j + half * 16 + 8 * (quad >> 1) + (sl >> 2);
                // (operand rows past d_down: finite values of no use)
                const int c = DD == 16 ? 4 * (sl & 3) : 16 * (quad & 1) + 4 * (sl & 3);
                const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(vb + key * DD + c));
                const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(vb + (key + 4) * DD + c));
                const uint2 ulo = __builtin_bit_cast(uint2, lo), uhi = __builtin_bit_cast(uint2, hi);
                const bf16x8_t a = __builtin_bit_cast(bf16x8_t, make_uint4(ulo.x, ulo.y, uhi.x, uhi.y));
                acc[j] = mfma(a, p[half], acc[j]);
                acc[j] = mfma(a, rest[half], acc[j]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[0][r] += acc[1][r];
    l = pair_sum(l);
    if (rval) {
        float* rec = pg.pfx_part + (bh * NS + sp) * (2 + DD);
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

}  // namespace dar
