/*
 * dar_q4.h — a split cache (dar.h) whose distant latents are held in 4 bits:
 * quantised as tokens leave the window, or packed from a cache that a prefill
 * has filled; read back; and decode steps that attend over them as they are.
 *
 * The conventions of dar.h hold (ownership, asynchrony, validation before
 * anything is enqueued, alignment of device pointers). The window stays in
 * full dimension and full precision: only the latents, which grow with the
 * context and are what a decode step reads, shrink (bf16, d_down = 16: 32 to 9
 * bytes a key or value latent; d_down = 32: 64 to 17).
 *
 * Format. A latent row (d_down columns) is cut into groups of 32 columns, the
 * last of which may be shorter. With a the largest |c| of a group:
 *   scale  the smallest power of two s with a <= 7 s, at least 2^-124 and at most
 *          2^125, held as the byte E = log2 s + 127;
 *   codes  per column a sign bit (the highest of four) and the index of the
 *          level nearest to |c| / s among 0, 1/2, 1, 3/2, 2, 3, 4, 6 (a tie goes
 *          to the even index, values past 6 to 6).
 * A group that holds an infinity or a NaN is stored as E = 255 with codes 0, and
 * all its columns read as NaN. Column c lies in byte c / 2 of its row, the even
 * column in the low four bits; a row takes 4 ceil(d_down / 8) bytes (columns past
 * d_down are 0) and ceil(d_down / 32) scale bytes.
 *   (Scales with a <= 7 s let values between 6 s and 7 s saturate. On normal
 *   latents of 16 and 32 columns the relative error is 0.110 and 0.112; scales
 *   with a <= 6 s, where nothing saturates, give 0.113 and 0.115, and a < 8 s
 *   0.118 and 0.115.)
 * What a step's output loses against a cache of 16-bit latents hangs on how much of the
 * softmax lies outside the window. Measured on normal keys, values and latents (d = 64,
 * d_down = 16, w = 512, queries of standard deviation 1, 2, 4; relative rms of the
 * output): 4096 tokens 0.066, 0.022, 0.014; 32768 tokens 0.111, 0.049, 0.022. Without a
 * window the scores' own error shows, the more the larger they are (d = 128, d_down =
 * 32, 16384 tokens): 0.12, 0.18, 0.32.
 *
 * Limits: a cache holds at most 2^30 tokens a sequence, B * Hkv is at most 65535, and in
 * a decode step B * Hq at most 2^20 (DAR_E_UNSUPPORTED).
 */
#ifndef DAR_Q4_H
#define DAR_Q4_H

#include "dar.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Split cache with 4-bit latents (device buffers owned by the caller, this
 * struct on the host).
 *   k_win, v_win      as in dar_cache
 *   k_codes, v_codes  [B][Hkv][cap][4 ceil(d_down / 8)] bytes
 *   k_exp, v_exp      [B][Hkv][cap][ceil(d_down / 32)] bytes
 *   cap               a multiple of 64        len   tokens appended so far */
typedef struct {
    void *k_win, *v_win, *k_codes, *v_codes, *k_exp, *v_exp;
    int cap;
    int len;
} dar_cache_q4;

/* Paged split cache with 4-bit latents: as dar_paged_cache, with code pages
 * [n_pages][Hkv][page_size][4 ceil(d_down / 8)] and scale pages
 * [n_pages][Hkv][page_size][ceil(d_down / 32)] in place of the latent pages. An
 * entry of block_table outside [0, n_pages) is never read or written through:
 * such tokens are not stored and read as zeros. */
typedef struct {
    void *k_win, *v_win, *k_codes, *v_codes, *k_exp, *v_exp;
    const int* block_table;
    int* lens;
    int page_size, max_blocks, n_pages;
} dar_paged_cache_q4;

/* dar_cache_append into a cache with 4-bit latents: every token that leaves the
 * window is projected with W_down to exactly the latent that dar_cache_append
 * would store (Eq. 1, fp32 accumulation, rounded to the shape's dtype), which is
 * then quantised; the newest min(n, w) tokens go to the ring. Bit-identical to
 * n single-token appends. On success c->len += n (host side, at enqueue time).
 * Fails with DAR_E_CAPACITY if len + n > cap. */
dar_status dar_cache_append_q4(const dar_shape* s, dar_cache_q4* c, const void* k_new,
                               const void* v_new, int n, const void* w_down, hipStream_t stream);

/* dar_cache_append_paged into a paged cache with 4-bit latents: one token per
 * sequence, k_new, v_new [B][Hkv][d], lens[b] += 1 on the device, in one launch.
 * Sequences at capacity are marked as dar_cache_append_paged marks them. */
dar_status dar_cache_append_paged_q4(const dar_shape* s, const dar_paged_cache_q4* c,
                                     const void* k_new, const void* v_new, const void* w_down,
                                     hipStream_t stream);

/* Quantises the latents of tokens first..D-1 of src, D = max(src->len - w, 0)
 * (every one that src holds), into the same slots of dst, and sets dst->len to
 * src->len. The window is not touched: dst either has src's ring (the same
 * pointers) or the caller copies it. A cache that one prefill after the other
 * extends (dar_attn_prefill_chunk) is kept up by calls with first = the D of the
 * call before. first >= 0 (nothing is converted where it is at or past D).
 * DAR_E_CAPACITY if src->len > dst->cap; a src with one shared latent per token
 * (v_lat == k_lat) is refused (DAR_E_ARG). */
dar_status dar_cache_pack_q4(const dar_shape* s, const dar_cache* src, int first, dar_cache_q4* dst,
                             hipStream_t stream);

/* The reverse: the values that tokens first..D-1 of src stand for, in the shape's
 * dtype (exact in both), into the same slots of dst; dst->len = src->len. */
dar_status dar_cache_unpack_q4(const dar_shape* s, const dar_cache_q4* src, int first, dar_cache* dst,
                               hipStream_t stream);

/* The same between paged caches, whose page sizes and block tables may differ.
 * first: device int [B] (each >= 0), or NULL for 0. Sequence b converts tokens
 * first[b]..D_b-1, D_b = max(src->lens[b] - w, 0). dst->lens[b] becomes
 * src->lens[b] on the device; a sequence that does not fit dst, or whose length is past
 * the capacity of src itself, converts nothing and is marked overflowed there (-1 - n);
 * one that is empty or overflowed in src converts nothing. Where both have one array of
 * lengths it is left as it is: a sequence that does not fit both converts nothing, and
 * dst is not to be read for it. Otherwise dst->lens shares no element with src->lens or
 * first (DAR_E_ARG): they are read in the launch that writes it. */
dar_status dar_cache_pack_paged_q4(const dar_shape* s, const dar_paged_cache* src, const int* first,
                                   const dar_paged_cache_q4* dst, hipStream_t stream);
dar_status dar_cache_unpack_paged_q4(const dar_shape* s, const dar_paged_cache_q4* src,
                                     const int* first, const dar_paged_cache* dst,
                                     hipStream_t stream);

/* dar_attn_decode over a cache with 4-bit latents: Eq. 3-4 with the values that
 * the codes stand for as the distant latents. q [B][Hq][d] at position c->len - 1,
 * o [B][Hq][d]; c->len >= 1. A token whose latent reads as NaN makes the outputs of
 * its KV head's queries NaN; a value in the window that is infinite makes its column
 * of those outputs infinite or NaN. Sums, softmax statistics and, outside the matrix
 * cores, all products are fp32; on the matrix cores the absorbed query and the weights of
 * the values are pairs of bf16 (off by at most 2^-16 of themselves): against fp64 an
 * output is off by its own rounding (0.0016 to 0.0017 relative rms, as with fp32
 * products), but one in 270 to 680 is rounded to the other neighbour than the exact value
 * would be (fp32 products: one in 1000 to 1600).
 *   ws: at least dar_decode_q4_workspace_bytes(s, c->cap) bytes.
 * Supported: every shape that dar_attn_decode takes, and any Hq / Hkv (bf16 with d
 * in {64, 128} and d_down in {16, 32} runs on the matrix cores). */
dar_status dar_attn_decode_q4(const dar_shape* s, const dar_cache_q4* c, const void* q,
                              const void* w_down, const void* w_up, void* o, void* ws,
                              size_t ws_bytes, hipStream_t stream);

/* The same over a paged cache, one length per sequence, every shape too: the query
 * of sequence b at position lens[b] - 1; a sequence with lens[b] < 1 gets NaN rows,
 * one beyond its capacity is read up to it. ws: at least
 * dar_decode_q4_workspace_bytes(s, max_blocks * page_size) bytes. In both forms a batch
 * that, all sequences full, holds 2^31 blocks of 128 distant tokens or their bytes' worth
 * of the window, a KV head's counted once for every eight of its query heads (four, where
 * it has no more or runs outside the matrix cores), is refused (DAR_E_UNSUPPORTED). */
dar_status dar_attn_decode_paged_q4(const dar_shape* s, const dar_paged_cache_q4* c, const void* q,
                                    const void* w_down, const void* w_up, void* o, void* ws,
                                    size_t ws_bytes, hipStream_t stream);

/* Workspace size for a cache of capacity cap (paged: max_blocks * page_size); 0 on
 * an invalid shape or capacity. */
size_t dar_decode_q4_workspace_bytes(const dar_shape* s, int cap);

#ifdef __cplusplus
}
#endif
#endif /* DAR_Q4_H */
