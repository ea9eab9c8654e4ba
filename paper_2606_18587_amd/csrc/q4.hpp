// Latents held in 4 bits (include/dar_q4.h): the format on the device, where a
// row of a dense or paged cache lies, and the argument checks of its entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/dar.h"
#include "../../include/dar_q4.h"
#include "dar_common.hpp"

namespace dar {

__host__ __device__ inline int q4_row_bytes(int dd) { return 4 * ((dd + 7) / 8); }
__host__ __device__ inline int q4_groups(int dd) { return (dd + 31) / 32; }

// Rows of a cache: [B * Hkv][cap] (bt NULL), or pages [n_pages][Hkv][1 << shift].
struct Q4Rows {
    const int* bt;
    int cap;  // dense: rows a head; paged: tokens a sequence may hold
    int maxb, shift, n_pages;
};

// Row number of token e (< cap) of (sequence b, KV head g), -1 in an unmapped page.
__device__ __forceinline__ long long q4_row(const Q4Rows& r, int b, int g, int Hkv, int e) {
    if (!r.bt) return ((long long)b * Hkv + g) * r.cap + e;
    const int page = r.bt[(size_t)b * r.maxb + (e >> r.shift)];
    if (page < 0 || page >= r.n_pages) return -1;
    return ((((long long)page * Hkv + g) << r.shift)) + (e & ((1 << r.shift) - 1));
}

// Scale byte of a group whose largest |c| has the fp32 bits u (no sign): E with
// 2^(E - 127) the smallest power of two s, |c| <= 7 s. 255: an infinity or a NaN.
// (Taken from the bits: NaN orders above infinity as an integer, and the build
// assumes that no float comparison meets one.)
__device__ __forceinline__ int q4_scale_byte(uint32_t u) {
    const int e = (int)(u >> 23);
    if (e == 255) return 255;
    return imin(imax(e - 2 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0), 3), 252);
}

// 2^(E - 127); infinity for E = 255, whose values v_cvt_scalef32 gives as NaN.
__device__ __forceinline__ float q4_scale(int E) { return __uint_as_float((uint32_t)E << 23); }

// Two bf16 / fp32 values as codes, in the low byte (v_cvt_scalef32_pk_fp4_*: divides
// by the power of two, rounds to nearest even, saturates).
typedef __bf16 q4_bf16x2 __attribute__((ext_vector_type(2)));
typedef float q4_f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t q4_pair_f32(float a, float b, float s) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, a, b, s, 0) & 0xffu;
}
// Eight bf16 values (packed pairs) as one word of codes.
__device__ __forceinline__ uint32_t q4_word_bf16(uint4 x, float s) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(q4_bf16x2, x.x), s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(q4_bf16x2, x.y), s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(q4_bf16x2, x.z), s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(q4_bf16x2, x.w), s, 3);
    return w;
}
// One word of codes as eight bf16 (packed pairs) / fp32 values.
__device__ __forceinline__ uint4 q4_values_bf16(uint32_t w, float s) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3)));
}
__device__ __forceinline__ void q4_values_f32(uint32_t w, float s, float (&v)[8]) {
    const q4_f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0);
    const q4_f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
    const q4_f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2);
    const q4_f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
    v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
}

// --- checks of the entry points (q4_cache.hip) ---------------------------------
constexpr int kQ4MaxTokens = 1 << 30;
bool q4_dev_ok(const void* p);  // non-NULL and 16-byte aligned
dar_status q4_check_shape(const dar_shape* s);  // (Hq: only that Hkv divides it)
dar_status q4_check_cache(const dar_shape* s, const dar_cache_q4* c);
dar_status q4_check_paged(const dar_shape* s, const dar_paged_cache_q4* c);
Q4Rows q4_rows(const dar_cache_q4* c);
Q4Rows q4_rows(const dar_paged_cache_q4* c);

}  // namespace dar
