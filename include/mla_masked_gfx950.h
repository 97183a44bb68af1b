/*
 * mla_masked_gfx950.h -- C ABI of masked attention over the latent cache on AMD
 * MI355X (gfx950): the tokens of a drafted tree, a sliding window with a few first
 * rows that stay visible, and prompts under that window.  The calls beside
 * mla_decode_paged(_multi) and mla_prefill_mha of mla_gfx950.h, whose masks are the
 * causal one: same queries, caches, page tables and types, same conventions (device
 * pointers, caller-owned buffers and workspace, 16-byte aligned tensors, a
 * hipStream_t as void*, MLA_OK or a negative mla_status, arguments validated on the
 * host before anything is launched, no allocation, no state).
 *
 * For query token i of sequence b and head h, over the cached rows j that the token
 * sees:
 *
 *   s_j   = softmax_scale * ( q_abs[b,i,h,:] . c_kv[j] + q_rope[b,i,h,:] . k_rope[j] )
 *   p     = softmax_j(s)
 *   o_lat[b,i,h,:] = sum_j p_j c_kv[j]        lse[b,i,h] = log sum_j exp(s_j)
 *
 * A token that sees no row gets zeros and -inf.  A row that a token does not see has
 * no influence on it, whatever the row holds (infinities and NaN included); rows that
 * no token sees need not have a page.  A token and head whose score with a row that it
 * sees is NaN or infinite, as with every row that is not finite, gets NaN in all of o_lat
 * and for lse.  A page id outside the pool where a row would be
 * read is not an error code: the rows of that page are seen by nobody.
 */
#ifndef MLA_MASKED_GFX950_H
#define MLA_MASKED_GFX950_H

#include "mla_gfx950.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Bytes of device workspace mla_decode_paged_tree needs (partial results where a
 * sequence's rows are shared out; 0 for many sizes, at most 640 MB).  max_rows: page_size *
 * max_pages_per_seq of the call.  Enough for every type and kernel; pure host function; 0 if
 * an argument is invalid.
 */
size_t mla_decode_tree_workspace_bytes(int B, int q_len, int heads, int d_c, int max_rows);

/*
 * Attention of a drafted tree's tokens (verification in tree-structured speculative
 * decoding).  The cache of sequence b holds prefix_lens[b] committed rows and behind
 * them those of up to q_len drafted tokens, token k's at logical position
 * prefix_lens[b] + k (mla_cache_store_at writes them there; the rope part of a node of
 * depth d turns by prefix_lens[b] + d, as that of its query).  Token i sees all
 * committed rows, and drafted row k iff bit k of tree_mask[b, i] is set: for a tree the
 * node itself and its ancestors; any mask may be passed, a lower triangle gives
 * mla_decode_paged_multi's.  Bits at and past q_len are ignored.  A sequence with fewer
 * drafted tokens leaves the rest of its masks without their bits; rows without a bit
 * anywhere are never used.  A drafted row past the table's end is seen by nobody.
 *
 *   q_abs  [B, q_len, heads, d_c]    q_rope [B, q_len, heads, d_rope]   io dtype
 *   kv_cache, kv_scale, page_table   as for mla_decode_paged
 *   prefix_lens [B] int32, each in [0, max_pages_per_seq * page_size]
 *   tree_mask  [B, q_len] uint64, the rows of sequence b mask_pitch words behind those of
 *              b - 1 (0: one tree for all, [q_len])
 *   o_lat  [B, q_len, heads, d_c] io dtype, lse [B, q_len, heads] fp32 (outputs; lse may
 *          be NULL)
 *   workspace  mla_decode_tree_workspace_bytes bytes, 256-byte aligned (may be NULL where
 *              that is 0); scratch
 *   flags  MLA_FLAG_DEFAULT or MLA_FLAG_PORTABLE_KERNEL
 *
 * q_len <= 64, q_len * heads <= 8192, max_pages_per_seq * page_size <= 2^30 (else
 * MLA_ERR_UNSUPPORTED).  io / cache dtype pairs, d_c, d_rope and page_size as for
 * mla_decode_paged.  The matrix-core kernels are used for BF16 io with a BF16 or
 * FP8 cache, page_size a multiple of 16, d_rope 64 and d_c in {256, 512}; everything else
 * runs on the portable scalar-FMA kernel.  Sums, softmax statistics and the partial results
 * that are merged are fp32; on the matrix cores the weights of the value sums are rounded to
 * bf16 (the normaliser sums them before).  One call gives the same bits every time.
 */
int mla_decode_paged_tree(const void* q_abs, const void* q_rope, const void* kv_cache, const float* kv_scale,
                          const int32_t* page_table, const int32_t* prefix_lens, const uint64_t* tree_mask,
                          int64_t mask_pitch, void* o_lat, float* lse, void* workspace, size_t workspace_bytes,
                          int B, int q_len, int heads, int d_c, int d_rope, int page_size, int num_pages,
                          int max_pages_per_seq, float softmax_scale, mla_dtype io_dtype, mla_dtype cache_dtype,
                          unsigned flags, void* hip_stream);

/*
 * Bytes of device workspace mla_decode_paged_window needs; as above.
 */
size_t mla_decode_window_workspace_bytes(int B, int q_len, int heads, int d_c, int max_rows, int window, int sinks);

/*
 * Attention with a sliding window and a few first rows that stay visible ("sinks").
 * As for mla_decode_paged_multi the cache already holds the rows of the q_len newest
 * tokens, its last q_len; token i sits at position t = seq_lens[b] - q_len + i and sees
 * row j <= t iff j > t - window or j < sinks.  A token whose position would be negative
 * sees nothing.  Rows that no token sees are not read: their pages may have been given
 * back, and their entries of the table be -1.
 *
 *   window >= 1 (the token itself counted), sinks >= 0
 * Everything else as for mla_decode_paged_tree; q_len of any size with q_len * heads <=
 * 8192.
 */
int mla_decode_paged_window(const void* q_abs, const void* q_rope, const void* kv_cache, const float* kv_scale,
                            const int32_t* page_table, const int32_t* seq_lens, void* o_lat, float* lse,
                            void* workspace, size_t workspace_bytes, int B, int q_len, int heads, int d_c, int d_rope,
                            int page_size, int num_pages, int max_pages_per_seq, int window, int sinks,
                            float softmax_scale, mla_dtype io_dtype, mla_dtype cache_dtype, unsigned flags,
                            void* hip_stream);

/*
 * Bytes of device workspace mla_prefill_window needs (mla_prefill_mha's for the pages
 * that a call can reach, a table of them, and partial results where few query rows have
 * their keys cut into chunks).  Pure host function; 0 if an argument is
 * invalid.
 */
size_t mla_prefill_window_workspace_bytes(int B, int q_len, int heads, int d_c, int max_pages_per_seq, int window,
                                          int sinks);

/*
 * mla_prefill_mha under the mask of mla_decode_paged_window: prompts, or chunks of them,
 * in the MHA paradigm (keys and values materialised per head, for the rows that some token
 * of the call sees and no others).
 * A row is taken for one that is not finite if a value of its latent part is 2^100 or more
 * in magnitude; one of which the rope part only is not finite, and whose score is -inf, counts
 * for nothing.
 *   lse [B, q_len, heads] fp32 (output, may be NULL)
 *   workspace  mla_prefill_window_workspace_bytes bytes, 256-byte aligned; scratch
 * Everything else, the sizes supported included, as for mla_prefill_mha; q_len <= 2^29 and
 * max_pages_per_seq * page_size <= 2^30.
 */
int mla_prefill_window(const void* q_nope, const void* q_rope, const void* W_UK, const void* W_UV,
                       const void* kv_cache, const int32_t* page_table, const int32_t* seq_lens, void* out, float* lse,
                       void* workspace, size_t workspace_bytes, int B, int q_len, int heads, int d_head, int d_c,
                       int d_rope, int page_size, int num_pages, int max_pages_per_seq, int window, int sinks,
                       float softmax_scale, mla_dtype io_dtype, mla_dtype cache_dtype, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MLA_MASKED_GFX950_H */
