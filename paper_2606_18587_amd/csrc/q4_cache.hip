// Writes and reads of a cache whose distant latents are held in 4 bits
// (include/dar_q4.h): appends that quantise what leaves the window, and the
// conversions from and to a cache of bf16 or fp32 latents.
//
// Each is bounded by its bytes: the arithmetic of a value is one conversion
// (v_cvt_scalef32_pk_*, two values an instruction) and its share of the group's
// maximum. The projection of an append is that of dar_cache_append, in the same
// order of sums, so that the codes are those of the latents it would store.
#include "mfma_common.hpp"
#include "q4.hpp"

#include <type_traits>

namespace dar {

namespace {

// Lane moves inside a quad.
template <int CTRL>
__device__ __forceinline__ uint32_t quad_move(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, CTRL, 0xF, 0xF, false);
}
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
// fp32 bits of the largest magnitude of a pair of bf16
__device__ __forceinline__ uint32_t amax_pair(uint32_t u) {
    return umax((u << 16) & 0x7fffffffu, u & 0x7fff0000u);
}

// ---------------------------------------------------------------------------
// pack and unpack

struct ConvArgs {
    const void* src[2];  // key and value latents / codes
    const uint8_t* src_exp[2];
    void* dst[2];
    uint8_t* dst_exp[2];
    Q4Rows from, to;
    const int* lens;   // source lengths (NULL: len)
    int* lens_to;      // where they go (NULL: nowhere)
    const int* first;  // per sequence (NULL: first0)
    int len, first0, w, Hkv, dd;
    int grid_x;        // workgroups along a head's rows
};

// Tokens [t0, D) that sequence b converts (none: D <= t0; both at least 0: a marked
// length may be any negative number, whose difference from w would leave 32 bits).
__device__ __forceinline__ void conv_range(const ConvArgs& a, int b, int& t0, int& D) {
    const int len = a.lens ? a.lens[b] : a.len;
    t0 = a.first ? imax(a.first[b], 0) : a.first0;
    D = len > a.w && len <= a.from.cap && len <= a.to.cap ? len - a.w : 0;
}

// The lengths of a paged destination: one thread of one workgroup a sequence. One past
// either side's capacity has had nothing converted, and is marked.
__device__ __forceinline__ void conv_lens(const ConvArgs& a, int b) {
    if (a.lens_to && wg_id_x() == 0 && wg_id_z() == 0 && wg_id_y() % a.Hkv == 0 && lane_id_x() == 0) {
        const int len = a.lens[b];
        a.lens_to[b] = len > a.to.cap || len > a.from.cap ? -1 - len : len;
    }
}

// One thread a group of 32 columns: any d_down, bf16 or fp32. Bounded by its loads, an
// element at a time with the lanes a group apart, each read for the maximum and again for
// its code: 16 x 32768 tokens of 8 KV heads, d_down 16 in fp32 526 us (1.15 TB/s), 48 in
// bf16 1409 (0.7).
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(ConvArgs a) {
    const int bg = wg_id_y(), b = bg / a.Hkv, g = bg - b * a.Hkv, kv = wg_id_z();
    int t0, D;
    conv_range(a, b, t0, D);
    conv_lens(a, b);
    const int ng = q4_groups(a.dd), rb = q4_row_bytes(a.dd);
    const long long total = (long long)(D - t0) * ng;
    for (long long i = (long long)wg_id_x() * 256 + lane_id_x(); i < total;
         i += (long long)a.grid_x * 256) {
        const int e = t0 + (int)(i / ng), j = (int)(i % ng);
        const long long ri = q4_row(a.from, b, g, a.Hkv, e), ro = q4_row(a.to, b, g, a.Hkv, e);
        if (ro < 0) continue;
        const int c0 = 32 * j, nc = imin(32, a.dd - c0);
        const T* x = (const T*)a.src[kv] + (ri < 0 ? 0 : ri) * a.dd + c0;
        uint32_t m = 0;
        for (int c = 0; c < nc; ++c)
            m = umax(m, ri < 0 ? 0u : __float_as_uint(elem<T>::load(x + c)) & 0x7fffffffu);
        const int E = q4_scale_byte(m);
        const float s = q4_scale(E);
        uint32_t* out = (uint32_t*)((uint8_t*)a.dst[kv] + ro * rb + 16 * j);
        for (int k = 0; k < (nc + 7) / 8; ++k) {
            uint32_t w = 0;
            if (E != 255 && ri >= 0)
                for (int p = 0; p < 4; ++p) {
                    const int c = 8 * k + 2 * p;
                    const float v0 = c < nc ? elem<T>::load(x + c) : 0.f;
                    const float v1 = c + 1 < nc ? elem<T>::load(x + c + 1) : 0.f;
                    w |= q4_pair_f32(v0, v1, s) << (8 * p);
                }
            out[k] = w;
        }
        a.dst_exp[kv][ro * ng + j] = (uint8_t)E;
    }
}

// One thread eight values: any d_down, bf16 or fp32. Bounded by its stores, an element
// at a time with the lanes eight apart: the same rows in fp32 320 us (1.9 TB/s), of 48
// bf16 columns 492 (2.1).
template <typename T>
__global__ __launch_bounds__(256) void unpack_kernel(ConvArgs a) {
    const int bg = wg_id_y(), b = bg / a.Hkv, g = bg - b * a.Hkv, kv = wg_id_z();
    int t0, D;
    conv_range(a, b, t0, D);
    conv_lens(a, b);
    const int nw = q4_row_bytes(a.dd) / 4, ng = q4_groups(a.dd);
    const long long total = (long long)(D - t0) * nw;
    for (long long i = (long long)wg_id_x() * 256 + lane_id_x(); i < total;
         i += (long long)a.grid_x * 256) {
        const int e = t0 + (int)(i / nw), k = (int)(i % nw);
        const long long ri = q4_row(a.from, b, g, a.Hkv, e), ro = q4_row(a.to, b, g, a.Hkv, e);
        if (ro < 0) continue;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (ri >= 0)
            q4_values_f32(((const uint32_t*)a.src[kv])[ri * nw + k],
                          q4_scale(a.src_exp[kv][ri * ng + (k >> 2)]), v);
        T* out = (T*)a.dst[kv] + ro * a.dd + 8 * k;
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (8 * k + c < a.dd) out[c] = elem<T>::from_f32(v[c]);
    }
}

// The hot form (bf16, d_down 16 or 32: one group a row). A lane takes eight values
// (16 bytes of latents, one word of codes), so that both sides are read and written
// in whole lines; the 2 or 4 lanes of a row join their maxima by lane moves.
// kConvRows rows' worth a thread, all requested before the first is used. Dense, 16 x
// 32768 tokens of 8 KV heads, d_down 16: packed in 60 us (5.6 TB/s), read back in 50 (6.8).
// BOTH: keys and values by one workgroup, which looks up a row's pages once (paged:
// 24 sequences of 1100 to 16000 tokens, d_down 32, read back 32 us, 26 so); dense
// caches take a workgroup each (4 x 131072 tokens, d_down 32: 111 us, together 119).
constexpr int kConvRows = 4;
typedef unsigned int conv_u32x4 __attribute__((ext_vector_type(4)));

template <int DD, bool PACK, bool BOTH, bool PAST>
__global__ __launch_bounds__(256) void conv_bf16_kernel(ConvArgs a) {
    constexpr int PR = DD / 8;  // pieces of a row
    constexpr int NK = BOTH ? 2 : 1;
    const int kv0 = BOTH ? 0 : wg_id_z();
    const int bg = wg_id_y(), b = bg / a.Hkv, g = bg - b * a.Hkv;
    int t0, D;
    conv_range(a, b, t0, D);
    conv_lens(a, b);
    const int tid = lane_id_x(), piece = tid % PR;
    constexpr int kRowsWg = 256 / PR * kConvRows;  // rows of a workgroup's turn
    for (long long e0 = t0 + (long long)wg_id_x() * kRowsWg; e0 < D; e0 += (long long)a.grid_x * kRowsWg) {
        conv_u32x4 x[kConvRows][NK];
        uint32_t c[kConvRows][NK], E[kConvRows][NK];
        long long ro[kConvRows];
        bool zero[kConvRows];
#pragma unroll
        for (int k = 0; k < kConvRows; ++k) {
            const long long want = e0 + tid / PR + 256 / PR * k;
            const int e = (int)(want < D ? want : D - 1);
            const long long ri = q4_row(a.from, b, g, a.Hkv, e);
            ro[k] = want < D ? q4_row(a.to, b, g, a.Hkv, e) : -1;
            zero[k] = ri < 0;
            const long long at = ri < 0 ? 0 : ri;
#pragma unroll
            for (int kv = 0; kv < NK; ++kv) {
                if constexpr (PACK) {
                    x[k][kv] = __builtin_nontemporal_load(
                        reinterpret_cast<const conv_u32x4*>((const bf16_t*)a.src[kv0 + kv] + at * DD + 8 * piece));
                } else {
                    c[k][kv] = *reinterpret_cast<const uint32_t*>((const uint8_t*)a.src[kv0 + kv] + at * (DD / 2) + 4 * piece);
                    E[k][kv] = a.src_exp[kv0 + kv][at];
                }
            }
        }
#pragma unroll
        for (int k = 0; k < kConvRows; ++k)
#pragma unroll
            for (int kv = 0; kv < NK; ++kv) {
                if constexpr (PACK) {
                    uint4 y = make_uint4(x[k][kv][0], x[k][kv][1], x[k][kv][2], x[k][kv][3]);
                    if (zero[k]) y = make_uint4(0, 0, 0, 0);
                    uint32_t m = umax(umax(amax_pair(y.x), amax_pair(y.y)), umax(amax_pair(y.z), amax_pair(y.w)));
                    m = umax(m, quad_move<0xB1>(m));
                    if constexpr (PR == 4) m = umax(m, quad_move<0x4E>(m));
                    const int s = q4_scale_byte(m);
                    const uint32_t w = s == 255 ? 0u : q4_word_bf16(y, q4_scale(s));
                    if (ro[k] >= 0) {
                        *reinterpret_cast<uint32_t*>((uint8_t*)a.dst[kv0 + kv] + ro[k] * (DD / 2) + 4 * piece) = w;
                        if (piece == 0) a.dst_exp[kv0 + kv][ro[k]] = (uint8_t)s;
                    }
                } else if (ro[k] >= 0) {
                    const uint4 v = zero[k] ? make_uint4(0, 0, 0, 0) : q4_values_bf16(c[k][kv], q4_scale(E[k][kv]));
                    conv_u32x4* out = reinterpret_cast<conv_u32x4*>((bf16_t*)a.dst[kv0 + kv] + ro[k] * DD + 8 * piece);
                    if constexpr (PAST) __builtin_nontemporal_store(__builtin_bit_cast(conv_u32x4, v), out);
                    else *out = __builtin_bit_cast(conv_u32x4, v);
                }
            }
    }
}

// Workgroups along a head's rows: `rows` of them each, at most 1024 (a loop takes
// the rest). Paged, what there is to convert is not known here, and rows are the
// capacity: workgroups that find nothing are not free (96 sequences that read back one
// token each, d_down 16 / 32: 8 / 10 us under tables of 2048 tokens, 103 / 186 under
// tables of 131072).
int conv_grid_x(long long cap, int rows) {
    const long long x = (cap + rows - 1) / rows;
    return (int)(x < 1 ? 1 : (x > 1024 ? 1024 : x));
}

template <typename T>
hipError_t launch_conv(ConvArgs a, bool pack, int B, long long rows, hipStream_t st) {
    if (sizeof(T) == 2 && (a.dd == 16 || a.dd == 32)) {
        a.grid_x = conv_grid_x(rows, 256 * 8 / a.dd * kConvRows);
        const bool both = a.lens != nullptr;
        // (more values than the Infinity Cache holds for whoever reads them next go past
        // it; paged, their number is not known here)
        const bool past = !both && rows * B * a.Hkv * a.dd * 4 >= 192LL << 20;
        auto pick = [&](auto dd) {
            constexpr int DD = decltype(dd)::value;
            if (pack) return both ? conv_bf16_kernel<DD, true, true, false> : conv_bf16_kernel<DD, true, false, false>;
            if (both) return conv_bf16_kernel<DD, false, true, false>;
            return past ? conv_bf16_kernel<DD, false, false, true> : conv_bf16_kernel<DD, false, false, false>;
        };
        auto kernel = a.dd == 16 ? pick(std::integral_constant<int, 16>{}) : pick(std::integral_constant<int, 32>{});
        hipLaunchKernelGGL(kernel, dim3(a.grid_x, B * a.Hkv, both ? 1 : 2), dim3(256), 0, st, a);
        return hipGetLastError();
    }
    const int per_row = pack ? q4_groups(a.dd) : q4_row_bytes(a.dd) / 4;
    a.grid_x = conv_grid_x(rows * per_row, 256);
    const dim3 grid(a.grid_x, B * a.Hkv, 2);
    if (pack)
        hipLaunchKernelGGL(pack_kernel<T>, grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL(unpack_kernel<T>, grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// append

struct AppendArgs {
    const void *k_new, *v_new, *wd;
    void *win[2];
    uint8_t *codes[2], *exps[2];
    Q4Rows rows;
    int* lens;  // paged: one token a sequence; dense: NULL
    int Hkv, d, dd, w, len, n;
    int grid_x;
};

// What new token t (at position len + t) makes leave: token e = len + t - w, from
// ring slot e % w while it is an old one (e < len), else from the new tokens. The
// same job then writes the ring slot that e had, for t < min(n, w): every slot
// that changes is read and rewritten by one job, in this order, so the whole
// append is one launch without a barrier. The slot's new owner is the last
// token at the same place of the ring.
struct ExitJob {
    int e;          // position that leaves (< 0: none yet)
    bool old;       // it is in the ring
    bool to_ring;   // the ring slot changes
    int slot, src;  // ring slot, and the new token (index) that takes it
};
__device__ __forceinline__ ExitJob exit_job(int len, int n, int w, int t) {
    ExitJob j;
    j.e = len + t - w;
    j.old = w > 0 && j.e < len && j.e >= 0;
    j.to_ring = w > 0 && t < imin(n, w);
    j.slot = 0;
    j.src = 0;
    if (j.to_ring) {
        j.slot = (len + t) % w;
        j.src = t + (n - 1 - t) / w * w;
    }
    return j;
}

// One wavefront a leaving token, a lane a column (d_down > 64: several), sums as
// project_col does them. Dense: grid (n, B * Hkv); paged (lens): a workgroup a
// sequence, its wavefronts taking the KV heads in turn, which then advances the
// length. For fp32 and sizes outside the matrix-core forms. Bounded by its loads of
// W_down, all of it for every token, a column a lane. Of a prompt dar_cache_append reads it
// once for 64 tokens, and with a pack behind it is faster for few columns: 8 x 8191
// tokens of 8 KV heads, d64, d_down 16 in fp32 1158 us here and 431 so, 48 in bf16 1065
// and 1346.
template <typename T>
__global__ __launch_bounds__(256) void append_q4_kernel(AppendArgs a) {
    const int lane = lane_id_x() & 63;
    const int wave = __builtin_amdgcn_readfirstlane(lane_id_x() >> 6);
    const bool paged = a.lens != nullptr;
    const int b = paged ? wg_id_x() : wg_id_y() / a.Hkv;
    const int len = paged ? a.lens[b] : a.len;
    const bool fits = !paged || (len >= 0 && len < a.rows.cap);
    const int rb = q4_row_bytes(a.dd), ng = q4_groups(a.dd);
    auto job = [&](int g, int t) {
        const int bg = b * a.Hkv + g;
        const ExitJob j = exit_job(len, a.n, a.w, t);
        const long long row = j.e >= 0 ? q4_row(a.rows, b, g, a.Hkv, j.e) : -1;
        const T* wdg = (const T*)a.wd + (size_t)g * a.d * a.dd;
        for (int kv = 0; kv < 2; ++kv) {
            const T* fresh = (const T*)(kv ? a.v_new : a.k_new) + (size_t)bg * a.n * a.d;
            T* ring = (T*)a.win[kv] + (size_t)bg * a.w * a.d;
            if (row >= 0) {
                const T* x = j.old ? ring + (size_t)j.slot * a.d : fresh + (size_t)(j.e - len) * a.d;
                for (int c0 = 0; c0 < a.dd; c0 += 64) {
                    const int c = c0 + lane;
                    float v = 0.f;
                    if (c < a.dd)
                        v = elem<T>::to_f32(elem<T>::from_f32(project_col<T>(x, wdg, a.d, a.dd, c)));
                    uint32_t m = __float_as_uint(v) & 0x7fffffffu;
#pragma unroll
                    for (int off = 1; off < 32; off <<= 1) m = umax(m, (uint32_t)__shfl_xor((int)m, off, 64));
                    const int E = q4_scale_byte(m);
                    const float other = __shfl_xor(v, 1, 64);
                    const uint32_t pair = E == 255 ? 0u : q4_pair_f32(v, other, q4_scale(E));
                    if (!(lane & 1) && c / 2 < rb) a.codes[kv][row * rb + c / 2] = (uint8_t)pair;
                    if (!(lane & 31) && c < a.dd) a.exps[kv][row * ng + c / 32] = (uint8_t)E;
                }
            }
            if (j.to_ring)
                for (int e = lane; e < a.d; e += 64)
                    ring[(size_t)j.slot * a.d + e] = fresh[(size_t)j.src * a.d + e];
        }
    };
    if (paged) {
        if (fits)
            for (int g = wave; g < a.Hkv; g += 4) job(g, 0);
        __syncthreads();  // every wavefront has read the length
        if (lane_id_x() == 0) {
            if (fits) a.lens[b] = len + 1;
            else if (len >= 0) a.lens[b] = -1 - len;
        }
    } else {
        for (long long t = wg_id_x() * 4 + wave; t < a.n; t += 4LL * a.grid_x)
            job(wg_id_y() - b * a.Hkv, (int)t);
    }
}

// bf16, d 64 or 128, d_down 16 or 32: the matrix-core projection of dar_cache_append
// (v_mfma_f32_32x32x16_bf16 over the same slabs in the same order: latent^T =
// W_down^T x^T, a token a column), so the same bits. Accumulator register r of lane
// l holds token l % 32, latent column 8 (r / 4) + 4 (l / 32) + r % 4.

// W_down^T as the A operand, its rows brought through LDS, which transposes them.
// (d_down = 16: the operand's other 16 rows read on, to 16 elements past the end.)
template <int D, int DD>
constexpr int kStagedWd = D * DD + (DD == 16 ? 16 : 0);
template <int D, int DD>
__device__ __forceinline__ void stage_wd(bf16_t* wsh, const bf16_t* wdg, int tid, int threads) {
    for (int i = tid * 8; i < D * DD; i += threads * 8)
        *reinterpret_cast<bf16x8_t*>(wsh + i) = load_bf16x8(wdg + i);
    if (DD == 16 && tid < 2) *reinterpret_cast<bf16x8_t*>(wsh + D * DD + 8 * tid) = zero_bf16x8();
}

// The row of a lane pair (l, l + 32) quantised: its code words (each lane has half of
// the row's words in w, `words` of them) and its scale byte.
template <int DD>
__device__ __forceinline__ int quantise_row(const f32x16_t& acc, uint32_t (&w)[DD / 16]) {
    uint32_t pk[DD / 4], m = 0;
#pragma unroll
    for (int i = 0; i < DD / 4; ++i) {
        pk[i] = pack2(acc[2 * i], acc[2 * i + 1]);
        m = umax(m, amax_pair(pk[i]));
    }
    const auto mm = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    const int E = q4_scale_byte(umax(mm[0], mm[1]));
    const float s = q4_scale(E);
    // half words: columns 8 q + 4 (l / 32) .. + 3, for q = 2 u and 2 u + 1
    uint32_t u[DD / 16];
#pragma unroll
    for (int k = 0; k < DD / 16; ++k) {
        u[k] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(q4_bf16x2, pk[4 * k]), s, 0);
        u[k] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u[k], __builtin_bit_cast(q4_bf16x2, pk[4 * k + 1]), s, 1);
        u[k] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u[k], __builtin_bit_cast(q4_bf16x2, pk[4 * k + 2]), s, 2);
        u[k] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u[k], __builtin_bit_cast(q4_bf16x2, pk[4 * k + 3]), s, 3);
        if (E == 255) u[k] = 0;
    }
    // lanes below 32 take the row's first words, the others the last
    const auto x = __builtin_amdgcn_permlane32_swap(u[0], u[DD / 16 - 1], false, false);
    const uint32_t lo = (x[0] & 0xffffu) | x[1] << 16, hi = x[0] >> 16 | (x[1] & 0xffff0000u);
    if constexpr (DD == 16) {
        w[0] = (lane_id_x() & 32) ? hi : lo;
    } else {
        w[0] = lo;
        w[1] = hi;
    }
    return E;
}

template <int DD>
__device__ __forceinline__ void store_row(uint8_t* codes, uint8_t* exps, long long row, const uint32_t (&w)[DD / 16],
                                          int E, int hg) {
    if constexpr (DD == 16) {
        *reinterpret_cast<uint32_t*>(codes + row * 8 + 4 * hg) = w[0];
    } else {
        *reinterpret_cast<uint2*>(codes + row * 16 + 8 * hg) = make_uint2(w[0], w[1]);
    }
    if (hg == 0) exps[row] = (uint8_t)E;
}

// Dense append: a wavefront 32 leaving tokens at a time, keys and values requested
// together (the first before W_down is staged; they are read once and pass by the
// caches). The lane that reads elements [16 s + 8 hg, + 8) of a ring slot is the one
// that rewrites them. Bounded by HBM, the fresh rows once and few bytes written: 8 x
// 8191 tokens of 8 KV heads, d64 d_down16, 44 us, 3.5 TB/s; keys and values in
// separate passes, more or fewer workgroups and plain loads were no faster. One token:
// 3.7 us, its round trips to memory.
template <int D, int DD>
__global__ __launch_bounds__(256) void append_q4_mfma_kernel(AppendArgs a) {
    constexpr int KS = D / 16;
    __shared__ __attribute__((aligned(16))) bf16_t wsh[kStagedWd<D, DD>];
    const int tid = lane_id_x(), lane = tid & 63, tl = lane & 31, hg = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int bg = wg_id_y(), b = bg / a.Hkv, g = bg - b * a.Hkv;
    const size_t fresh0 = (size_t)bg * a.n * D + 8 * hg, ring0 = (size_t)bg * a.w * D + 8 * hg;
    long long c0 = (long long)(wg_id_x() * 4 + wave) * 32;
    bf16x8_t x[2][KS];
    ExitJob j{};
    // (a lane past the last token takes that token's, and drops it)
    auto load = [&]() {
        j = exit_job(a.len, a.n, a.w, (int)(c0 + tl < a.n ? c0 + tl : a.n - 1));
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            const bf16_t* row = j.old ? (const bf16_t*)a.win[kv] + ring0 + (size_t)j.slot * D
                                      : (const bf16_t*)(kv ? a.v_new : a.k_new) + fresh0 + (size_t)imax(j.e - a.len, 0) * D;
#pragma unroll
            for (int s = 0; s < KS; ++s)
                x[kv][s] = __builtin_bit_cast(bf16x8_t, __builtin_nontemporal_load(reinterpret_cast<const conv_u32x4*>(row + 16 * s)));
        }
    };
    if (c0 < a.n) load();
    stage_wd<D, DD>(wsh, (const bf16_t*)a.wd + (size_t)g * D * DD, tid, 256);
    __syncthreads();
    bf16x8_t wa[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) wa[s] = lds_tr_operand(wsh, DD, 16 * s, 0, lane);
    while (c0 < a.n) {
        const bool valid = c0 + tl < a.n, project = valid && j.e >= 0, to_ring = valid && j.to_ring;
        if (__builtin_amdgcn_ballot_w64(project)) {
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                f32x16_t acc = splat16(0.f);
#pragma unroll
                for (int s = 0; s < KS; ++s) acc = mfma(wa[s], x[kv][s], acc);
                uint32_t w[DD / 16];
                const int E = quantise_row<DD>(acc, w);
                if (project) store_row<DD>(a.codes[kv], a.exps[kv], (long long)bg * a.rows.cap + j.e, w, E, hg);
            }
        }
        if (to_ring) {
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                const bf16_t* from = (const bf16_t*)(kv ? a.v_new : a.k_new) + fresh0 + (size_t)j.src * D;
                bf16_t* slot = (bf16_t*)a.win[kv] + ring0 + (size_t)j.slot * D;
#pragma unroll
                for (int s = 0; s < KS; ++s) x[kv][s] = load_bf16x8(from + 16 * s);
#pragma unroll
                for (int s = 0; s < KS; ++s) *reinterpret_cast<bf16x8_t*>(slot + 16 * s) = x[kv][s];
            }
        }
        c0 += 128LL * a.grid_x;
        if (c0 < a.n) load();
    }
}

// Paged append, a token a sequence: a workgroup a sequence, a wavefront a KV head in
// turn; column 0 is the token's key, column 1 its value. One launch: the workgroup
// that read the length advances it. Bounded by three dependent round trips (length,
// page, rows): 96 sequences of 8 KV heads, d128 d_down32, 6.9 us.
template <int D, int DD>
__global__ __launch_bounds__(512) void append_q4_paged_mfma_kernel(AppendArgs a) {
    constexpr int KS = D / 16;
    __shared__ __attribute__((aligned(16))) bf16_t wsh[8][kStagedWd<D, DD>];
    const int lane = lane_id_x() & 63, tl = lane & 31, hg = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(lane_id_x() >> 6), waves = a.grid_x;
    const int b = wg_id_x(), len = a.lens[b];
    const bool fits = len >= 0 && len < a.rows.cap;
    if (fits) {
        const ExitJob j = exit_job(len, 1, a.w, 0);
        const int kv = tl & 1;
        const bool mine = tl < 2;
        for (int g = wave; g < a.Hkv; g += waves) {
            const int bg = b * a.Hkv + g;
            const long long row = j.e >= 0 ? q4_row(a.rows, b, g, a.Hkv, j.e) : -1;
            const bf16_t* fresh = (const bf16_t*)(kv ? a.v_new : a.k_new) + (size_t)bg * D + 8 * hg;
            bf16_t* slot = (bf16_t*)a.win[kv] + ((size_t)bg * a.w + j.slot) * D + 8 * hg;
            bf16x8_t x[KS], y[KS];
            // (a ring that is not full yet: the slot is read all the same, and not used)
            const bf16_t* from = j.to_ring ? slot : fresh;
#pragma unroll
            for (int s = 0; s < KS; ++s) y[s] = load_bf16x8(fresh + 16 * s);
#pragma unroll
            for (int s = 0; s < KS; ++s) x[s] = load_bf16x8(from + 16 * s);
            if (row >= 0) {  // wave-uniform
                wave_lds_order();
                stage_wd<D, DD>(wsh[wave], (const bf16_t*)a.wd + (size_t)g * D * DD, lane, 64);
                wave_lds_order();
                f32x16_t acc = splat16(0.f);
#pragma unroll
                for (int s = 0; s < KS; ++s) acc = mfma(lds_tr_operand(wsh[wave], DD, 16 * s, 0, lane), x[s], acc);
                uint32_t w[DD / 16];
                const int E = quantise_row<DD>(acc, w);
                if (mine) store_row<DD>(a.codes[kv], a.exps[kv], row, w, E, hg);
            }
            if (mine && j.to_ring)
#pragma unroll
                for (int s = 0; s < KS; ++s) *reinterpret_cast<bf16x8_t*>(slot + 16 * s) = y[s];
        }
    }
    __syncthreads();  // every wavefront has read the length
    if (lane_id_x() == 0) {
        if (fits) a.lens[b] = len + 1;
        else if (len >= 0) a.lens[b] = -1 - len;
    }
}

template <int D, int DD>
hipError_t launch_append_mfma(AppendArgs a, int B, hipStream_t st) {
    if (a.lens) {
        a.grid_x = a.Hkv < 8 ? a.Hkv : 8;  // wavefronts of a workgroup
        hipLaunchKernelGGL((append_q4_paged_mfma_kernel<D, DD>), dim3(B), dim3(64 * a.grid_x), 0, st, a);
    } else {
        const long long want = (a.n + 127LL) / 128, most = 4096 / (B * a.Hkv) + 1;
        a.grid_x = (int)(want < most ? want : most);
        hipLaunchKernelGGL((append_q4_mfma_kernel<D, DD>), dim3(a.grid_x, B * a.Hkv), dim3(256), 0, st, a);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t launch_append_q4(AppendArgs a, int B, hipStream_t st) {
    if (sizeof(T) == 2 && (a.d == 64 || a.d == 128) && (a.dd == 16 || a.dd == 32)) {
        if (a.d == 64) return a.dd == 16 ? launch_append_mfma<64, 16>(a, B, st) : launch_append_mfma<64, 32>(a, B, st);
        return a.dd == 16 ? launch_append_mfma<128, 16>(a, B, st) : launch_append_mfma<128, 32>(a, B, st);
    }
    a.grid_x = a.n < 4 * 16384 ? (a.n + 3) / 4 : 16384;
    const dim3 grid = a.lens ? dim3(B) : dim3(a.grid_x, B * a.Hkv);
    hipLaunchKernelGGL(append_q4_kernel<T>, grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace

// ---------------------------------------------------------------------------
// checks

bool q4_dev_ok(const void* p) { return p != nullptr && ((uintptr_t)p & 15u) == 0; }

dar_status q4_check_shape(const dar_shape* s) {
    if (!s) return DAR_E_ARG;
    if (s->B < 1 || s->Hq < 1 || s->Hkv < 1 || s->d < 1 || s->d_down < 1 || s->w < 0) return DAR_E_ARG;
    if (s->Hq % s->Hkv != 0 || s->d_down > s->d) return DAR_E_ARG;
    if (s->dtype != DAR_F32 && s->dtype != DAR_BF16) return DAR_E_ARG;
    if (s->d > 256 || s->w > kQ4MaxTokens) return DAR_E_UNSUPPORTED;
    if ((long long)s->B * s->Hkv > 65535) return DAR_E_UNSUPPORTED;  // (a grid's y)
    return DAR_OK;
}

static dar_status check_arrays(const dar_shape* s, const void* k_win, const void* v_win,
                               const void* const (&lat)[4]) {
    if (s->w > 0 && (!q4_dev_ok(k_win) || !q4_dev_ok(v_win))) return DAR_E_ARG;
    for (const void* p : lat)
        if (!q4_dev_ok(p)) return DAR_E_ARG;
    return DAR_OK;
}

dar_status q4_check_cache(const dar_shape* s, const dar_cache_q4* c) {
    if (!c || c->cap < 1 || (c->cap & 63) || c->len < 0 || c->len > c->cap) return DAR_E_ARG;
    if (c->cap > kQ4MaxTokens) return DAR_E_UNSUPPORTED;
    return check_arrays(s, c->k_win, c->v_win, {c->k_codes, c->v_codes, c->k_exp, c->v_exp});
}

static dar_status check_pages(int page_size, int max_blocks, int n_pages, const int* bt, const int* lens) {
    if (page_size < 32 || (page_size & (page_size - 1)) || max_blocks < 1 || n_pages < 1) return DAR_E_ARG;
    if ((long long)page_size * max_blocks > 0x7fffffffLL) return DAR_E_ARG;
    if (!bt || !lens || ((uintptr_t)bt & 3u) || ((uintptr_t)lens & 3u)) return DAR_E_ARG;
    if ((long long)page_size * max_blocks > kQ4MaxTokens) return DAR_E_UNSUPPORTED;
    return DAR_OK;
}

dar_status q4_check_paged(const dar_shape* s, const dar_paged_cache_q4* c) {
    if (!c) return DAR_E_ARG;
    const dar_status st = check_pages(c->page_size, c->max_blocks, c->n_pages, c->block_table, c->lens);
    if (st != DAR_OK) return st;
    return check_arrays(s, c->k_win, c->v_win, {c->k_codes, c->v_codes, c->k_exp, c->v_exp});
}

Q4Rows q4_rows(const dar_cache_q4* c) { return Q4Rows{nullptr, c->cap, 0, 0, 0}; }
Q4Rows q4_rows(const dar_paged_cache_q4* c) {
    return Q4Rows{c->block_table, c->page_size * c->max_blocks, c->max_blocks,
                  __builtin_ctz((unsigned)c->page_size), c->n_pages};
}
static Q4Rows lat_rows(const dar_cache* c) { return Q4Rows{nullptr, c->cap, 0, 0, 0}; }
static Q4Rows lat_rows(const dar_paged_cache* c) {
    return Q4Rows{c->block_table, c->page_size * c->max_blocks, c->max_blocks,
                  __builtin_ctz((unsigned)c->page_size), c->n_pages};
}

// A cache of bf16 or fp32 latents on the other side of a conversion (its ring is
// not touched).
static dar_status check_latents(const dar_cache* c) {
    if (!c || c->cap < 1 || c->len < 0 || c->len > c->cap) return DAR_E_ARG;
    if (c->cap > kQ4MaxTokens) return DAR_E_UNSUPPORTED;
    if (!q4_dev_ok(c->k_lat) || !q4_dev_ok(c->v_lat) || c->k_lat == c->v_lat) return DAR_E_ARG;
    return DAR_OK;
}

static dar_status check_latents(const dar_paged_cache* c) {
    if (!c) return DAR_E_ARG;
    const dar_status st = check_pages(c->page_size, c->max_blocks, c->n_pages, c->block_table, c->lens);
    if (st != DAR_OK) return st;
    if (!q4_dev_ok(c->k_pool) || !q4_dev_ok(c->v_pool) || c->k_pool == c->v_pool) return DAR_E_ARG;
    return DAR_OK;
}

// The integers per sequence of a paged conversion: it writes `to` in the launch that
// reads the others, so an element that they shared might be met before or after.
static dar_status check_lens(const int* from, const int* to, const int* first, int B) {
    auto meet = [&](const int* p) {
        const uintptr_t a = (uintptr_t)p, b = (uintptr_t)to, n = (size_t)B * sizeof(int);
        return a < b + n && b < a + n;
    };
    if ((uintptr_t)first & 3u) return DAR_E_ARG;
    if (from == to) return DAR_OK;  // nothing is written
    return meet(from) || (first && meet(first)) ? DAR_E_ARG : DAR_OK;
}

template <typename Q>
static dar_status check_codes(const Q* c) {
    for (const void* p : {c->k_codes, c->v_codes, c->k_exp, c->v_exp})
        if (!q4_dev_ok(p)) return DAR_E_ARG;
    return DAR_OK;
}

static dar_status conv(const dar_shape* s, const ConvArgs& a, bool pack, long long rows, hipStream_t st) {
    (void)hipGetLastError();
    const hipError_t e = s->dtype == DAR_BF16 ? launch_conv<bf16_t>(a, pack, s->B, rows, st)
                                              : launch_conv<float>(a, pack, s->B, rows, st);
    return e == hipSuccess ? DAR_OK : DAR_E_HIP;
}

}  // namespace dar

using namespace dar;

extern "C" {

dar_status dar_cache_append_q4(const dar_shape* s, dar_cache_q4* c, const void* k_new,
                               const void* v_new, int n, const void* w_down, hipStream_t stream) {
    dar_status st = q4_check_shape(s);
    if (st != DAR_OK) return st;
    st = q4_check_cache(s, c);
    if (st != DAR_OK) return st;
    if (n < 1 || !q4_dev_ok(k_new) || !q4_dev_ok(v_new) || !q4_dev_ok(w_down)) return DAR_E_ARG;
    if ((long long)c->len + n > c->cap) return DAR_E_CAPACITY;
    (void)hipGetLastError();
    const AppendArgs a{k_new, v_new, w_down, {c->k_win, c->v_win},
                       {(uint8_t*)c->k_codes, (uint8_t*)c->v_codes},
                       {(uint8_t*)c->k_exp, (uint8_t*)c->v_exp},
                       q4_rows(c), nullptr, s->Hkv, s->d, s->d_down, s->w, c->len, n, 0};
    const hipError_t e = s->dtype == DAR_BF16 ? launch_append_q4<bf16_t>(a, s->B, stream)
                                              : launch_append_q4<float>(a, s->B, stream);
    if (e != hipSuccess) return DAR_E_HIP;
    c->len += n;
    return DAR_OK;
}

dar_status dar_cache_append_paged_q4(const dar_shape* s, const dar_paged_cache_q4* c,
                                     const void* k_new, const void* v_new, const void* w_down,
                                     hipStream_t stream) {
    dar_status st = q4_check_shape(s);
    if (st != DAR_OK) return st;
    st = q4_check_paged(s, c);
    if (st != DAR_OK) return st;
    if (!q4_dev_ok(k_new) || !q4_dev_ok(v_new) || !q4_dev_ok(w_down)) return DAR_E_ARG;
    (void)hipGetLastError();
    const AppendArgs a{k_new, v_new, w_down, {c->k_win, c->v_win},
                       {(uint8_t*)c->k_codes, (uint8_t*)c->v_codes},
                       {(uint8_t*)c->k_exp, (uint8_t*)c->v_exp},
                       q4_rows(c), c->lens, s->Hkv, s->d, s->d_down, s->w, 0, 1, 0};
    const hipError_t e = s->dtype == DAR_BF16 ? launch_append_q4<bf16_t>(a, s->B, stream)
                                              : launch_append_q4<float>(a, s->B, stream);
    return e == hipSuccess ? DAR_OK : DAR_E_HIP;
}

dar_status dar_cache_pack_q4(const dar_shape* s, const dar_cache* src, int first, dar_cache_q4* dst,
                             hipStream_t stream) {
    dar_status st = q4_check_shape(s);
    if (st != DAR_OK) return st;
    st = check_latents(src);
    if (st != DAR_OK) return st;
    if (first < 0 || !dst || dst->cap < 1 || (dst->cap & 63)) return DAR_E_ARG;
    if (dst->cap > kQ4MaxTokens) return DAR_E_UNSUPPORTED;
    st = check_codes(dst);
    if (st != DAR_OK) return st;
    if (src->len > dst->cap) return DAR_E_CAPACITY;
    const long long rows = (long long)src->len - s->w - first;
    if (rows > 0) {
        const ConvArgs a{{src->k_lat, src->v_lat}, {nullptr, nullptr}, {dst->k_codes, dst->v_codes},
                         {(uint8_t*)dst->k_exp, (uint8_t*)dst->v_exp}, lat_rows(src), q4_rows(dst),
                         nullptr, nullptr, nullptr, src->len, first, s->w, s->Hkv, s->d_down, 0};
        st = conv(s, a, true, rows, stream);
        if (st != DAR_OK) return st;
    }
    dst->len = src->len;
    return DAR_OK;
}

dar_status dar_cache_unpack_q4(const dar_shape* s, const dar_cache_q4* src, int first, dar_cache* dst,
                               hipStream_t stream) {
    dar_status st = q4_check_shape(s);
    if (st != DAR_OK) return st;
    if (first < 0 || !src || src->cap < 1 || (src->cap & 63) || src->len < 0 || src->len > src->cap)
        return DAR_E_ARG;
    if (src->cap > kQ4MaxTokens) return DAR_E_UNSUPPORTED;
    st = check_codes(src);
    if (st != DAR_OK) return st;
    if (!dst) return DAR_E_ARG;
    dar_cache to = *dst;
    to.len = 0;  // (whatever it held before)
    st = check_latents(&to);
    if (st != DAR_OK) return st;
    if (src->len > dst->cap) return DAR_E_CAPACITY;
    const long long rows = (long long)src->len - s->w - first;
    if (rows > 0) {
        const ConvArgs a{{src->k_codes, src->v_codes}, {(const uint8_t*)src->k_exp, (const uint8_t*)src->v_exp},
                         {dst->k_lat, dst->v_lat}, {nullptr, nullptr}, q4_rows(src), lat_rows(dst),
                         nullptr, nullptr, nullptr, src->len, first, s->w, s->Hkv, s->d_down, 0};
        st = conv(s, a, false, rows, stream);
        if (st != DAR_OK) return st;
    }
    dst->len = src->len;
    return DAR_OK;
}

dar_status dar_cache_pack_paged_q4(const dar_shape* s, const dar_paged_cache* src, const int* first,
                                   const dar_paged_cache_q4* dst, hipStream_t stream) {
    dar_status st = q4_check_shape(s);
    if (st != DAR_OK) return st;
    st = check_latents(src);
    if (st != DAR_OK) return st;
    if (!dst) return DAR_E_ARG;
    st = check_pages(dst->page_size, dst->max_blocks, dst->n_pages, dst->block_table, dst->lens);
    if (st != DAR_OK) return st;
    st = check_lens(src->lens, dst->lens, first, s->B);
    if (st != DAR_OK) return st;
    st = check_codes(dst);
    if (st != DAR_OK) return st;
    const ConvArgs a{{src->k_pool, src->v_pool}, {nullptr, nullptr}, {dst->k_codes, dst->v_codes},
                     {(uint8_t*)dst->k_exp, (uint8_t*)dst->v_exp}, lat_rows(src), q4_rows(dst),
                     src->lens, src->lens == dst->lens ? nullptr : dst->lens, first, 0, 0, s->w,
                     s->Hkv, s->d_down, 0};
    return conv(s, a, true, a.from.cap < a.to.cap ? a.from.cap : a.to.cap, stream);
}

dar_status dar_cache_unpack_paged_q4(const dar_shape* s, const dar_paged_cache_q4* src,
                                     const int* first, const dar_paged_cache* dst,
                                     hipStream_t stream) {
    dar_status st = q4_check_shape(s);
    if (st != DAR_OK) return st;
    if (!src) return DAR_E_ARG;
    st = check_pages(src->page_size, src->max_blocks, src->n_pages, src->block_table, src->lens);
    if (st != DAR_OK) return st;
    st = check_codes(src);
    if (st != DAR_OK) return st;
    st = check_latents(dst);
    if (st != DAR_OK) return st;
    st = check_lens(src->lens, dst->lens, first, s->B);
    if (st != DAR_OK) return st;
    const ConvArgs a{{src->k_codes, src->v_codes}, {(const uint8_t*)src->k_exp, (const uint8_t*)src->v_exp},
                     {dst->k_pool, dst->v_pool}, {nullptr, nullptr}, q4_rows(src), lat_rows(dst),
                     src->lens, src->lens == dst->lens ? nullptr : dst->lens, first, 0, 0, s->w,
                     s->Hkv, s->d_down, 0};
    return conv(s, a, false, a.from.cap < a.to.cap ? a.from.cap : a.to.cap, stream);
}

}  // extern "C"
