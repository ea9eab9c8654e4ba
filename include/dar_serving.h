/*
 * dar_serving.h — serving operators of libdar that bound and share the split
 * cache of dar.h: decode steps that score the cached tokens by the attention
 * weight they receive, eviction of the least attended distant tokens, and decode
 * steps of a batch whose sequences share a long prefix.
 *
 * The conventions of dar.h hold (ownership, asynchrony, validation before
 * anything is enqueued, alignment of device pointers). A cache holds at most
 * 2^30 tokens a sequence and B * Hkv is at most 65535 (DAR_E_UNSUPPORTED); the
 * dense decode takes fewer, the capacities that dar_attn_decode takes (at most
 * 2^26 bytes of latents a head).
 *
 * Scores. A score array is fp32 [B][Hkv][cap] (paged: cap = max_blocks *
 * page_size), one entry per token of the cache: entry e of (sequence b, KV head
 * g) belongs to token e, 0 <= e < len. The caller owns it, clears it before the
 * first token, and clears a sequence's part when the sequence is replaced.
 *   scores is read, scores_out written; they are the same array (the update is
 *   then in place) or do not overlap at all (DAR_E_ARG if they overlap in
 *   part). Only entries of tokens 0..len-1 are read or written, so an array
 *   that stays zero past the newest token needs no clearing between calls; a
 *   caller that alternates between two arrays keeps both zero there.
 *   Decode steps are what fills a score array: no prefill does. A caller that
 *   evicts right after a prompt supplies the scores of its tokens itself.
 */
#ifndef DAR_SERVING_H
#define DAR_SERVING_H

#include "dar.h"

#ifdef __cplusplus
extern "C" {
#endif

/* dar_attn_decode that also adds to every cached token's score the attention
 * weight it receives, summed over the query heads of its KV head:
 *   scores_out[b][g][e] = scores[b][g][e] + sum over query heads h of group g of
 *   exp(S_he - log sum_j exp(S_hj)), 0 <= e < len,
 * S the scaled scores of Eq. 4 (window tokens at full dimension, distant ones
 * lifted). The weights of one head add up to 1; they are computed in fp32 from
 * unrounded absorbed queries.
 *   ws: at least dar_decode_scored_workspace_bytes(s, c->cap) bytes.
 * Arguments, output and support otherwise as dar_attn_decode; a cache with one
 * shared latent per token (v_lat == k_lat) is refused (DAR_E_ARG). */
dar_status dar_attn_decode_scored(const dar_shape* s, const dar_cache* c, const void* q,
                                  const void* w_down, const void* w_up, void* o,
                                  const float* scores, float* scores_out, void* ws, size_t ws_bytes,
                                  hipStream_t stream);

/* dar_attn_decode_paged for sequences that share their first n_prefix tokens
 * (one prompt, many continuations): the latents of tokens 0..n_prefix-1 of every
 * sequence are read once for the whole batch, from the pages prefix_blocks
 * (device int [n_prefix / page_size]; an entry outside [0, n_pages) reads as
 * zeros) in place of the block table's first entries, which normally name the
 * same pages and are not read here. n_prefix: a multiple of page_size, at most
 * max_blocks * page_size; 0: no prefix (prefix_blocks may be NULL).
 *   Position and window are as ever: sequence b's query sits at lens[b] - 1,
 *   lens[b] counting the prefix, and a sequence whose window reaches into the
 *   prefix (lens[b] < n_prefix + w) sees those tokens in its ring and only the
 *   older ones in the prefix. (A prefix latent that the batch's longest sequence
 *   sees enters the others' sums with weight zero: it has to be finite.)
 *   ws: at least dar_decode_prefix_workspace_bytes(s, max_blocks * page_size,
 *   n_prefix) bytes. Otherwise, and in support, as dar_attn_decode_paged. */
dar_status dar_attn_decode_paged_prefix(const dar_shape* s, const dar_paged_cache* c, int n_prefix,
                                        const int* prefix_blocks, const void* q, const void* w_down,
                                        const void* w_up, void* o, void* ws, size_t ws_bytes,
                                        hipStream_t stream);

/* dar_attn_decode_paged_prefix (n_prefix = 0: dar_attn_decode_paged) with the
 * scores of dar_attn_decode_scored for the tokens past the prefix: entries
 * n_prefix..lens[b]-1 of sequence b. Entries of the prefix's tokens are neither
 * read nor written; a sequence with lens[b] < 1 has none. The output is that of
 * dar_attn_decode_paged_prefix to the last bit. */
dar_status dar_attn_decode_paged_scored(const dar_shape* s, const dar_paged_cache* c, int n_prefix,
                                        const int* prefix_blocks, const void* q, const void* w_down,
                                        const void* w_up, void* o, const float* scores,
                                        float* scores_out, void* ws, size_t ws_bytes,
                                        hipStream_t stream);

/* Evicts distant tokens until about n_keep are left. With D = max(len - w, 0)
 * distant tokens (the latents) and D > n_keep, E of them leave:
 *   E = floor((D - n_keep) / w) * w   (w = 0: E = D - n_keep),
 * a multiple of w, so that every window token keeps its ring slot (token p at
 * slot p % w); up to w - 1 tokens above n_keep stay. Nothing happens while
 * D < n_keep + max(w, 1).
 * For each (sequence, KV head) on its own: the first n_fixed tokens stay; of the
 * others the D - E - n_fixed with the highest scores stay (of equal scores the
 * lower slots; -0 equals 0; NaN is below every number). The kept tokens in slots
 * at or past D - E move, in order, into the slots that evicted tokens leave
 * below D - E; no other latent changes. Scores move with their tokens, the
 * window tokens' scores (entries D..len-1) move down by E, and entries
 * len-E..len-1 become zero. Then c->len -= E (host side, at enqueue time).
 *   The entry points without "rope" in their name treat the distant tokens as a
 *   set, so they read an evicted cache like any other. Those with it take a
 *   token's position from its slot, which eviction changes: an evicted cache is
 *   not for them (rotate keys and queries before the call instead).
 *   A cache with one shared latent per token (v_lat == k_lat) keeps window
 *   tokens' latents in the same array and is refused (DAR_E_ARG).
 *   ws: device workspace of at least dar_cache_evict_workspace_bytes(s, c->cap,
 *   n_keep) bytes (caller-owned, overwritten).
 * Requires 0 <= n_fixed <= n_keep. Supported: every shape and dtype (within the
 * limits above). */
dar_status dar_cache_evict(const dar_shape* s, dar_cache* c, int n_keep, int n_fixed,
                           const float* scores, float* scores_out, void* ws, size_t ws_bytes,
                           hipStream_t stream);

/* dar_cache_evict over a paged cache, each sequence with its own D and E (from
 * lens[b], on the device); lens[b] -= E_b on the device. Latents move between
 * the pages that the sequence's block table names for their slots (an entry
 * outside [0, n_pages) is never read or written through: a token moved from
 * such a block reads as zeros, one moved to it is not stored). Pages past the
 * new end are no longer read; the caller may take them back. Pages that several
 * sequences share must hold tokens below n_fixed only. A sequence with
 * lens[b] < 1 (empty or overflowed) or beyond its capacity is left alone. */
dar_status dar_cache_evict_paged(const dar_shape* s, const dar_paged_cache* c, int n_keep,
                                 int n_fixed, const float* scores, float* scores_out, void* ws,
                                 size_t ws_bytes, hipStream_t stream);

/* Workspace sizes for a cache of capacity cap (paged: max_blocks * page_size);
 * 0 on an invalid shape, capacity, n_prefix or n_keep. */
size_t dar_decode_scored_workspace_bytes(const dar_shape* s, int cap);
size_t dar_decode_prefix_workspace_bytes(const dar_shape* s, int cap, int n_prefix);
size_t dar_cache_evict_workspace_bytes(const dar_shape* s, int cap, int n_keep);

#ifdef __cplusplus
}
#endif
#endif /* DAR_SERVING_H */
