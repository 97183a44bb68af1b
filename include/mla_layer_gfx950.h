/*
 * mla_layer_gfx950.h -- C ABI of the operators around the latent attention of one
 * layer on AMD MI355X (gfx950): the norm that feeds its projections, the 8-bit
 * projections themselves, the rotation of the queries and the write side of the
 * cache for any number of new tokens.  With the calls of mla_gfx950.h between
 * them they take a layer from hidden states to hidden states:
 *
 *   h' , codes      = mla_rms_norm(h, residual)          h' = h + residual
 *   q               = mla_gemm_fp8(codes, W_Q)           [tokens, heads * (d_head + d_rope)]
 *   q_nope, q_rope  = mla_rope_queries(q, positions)
 *   rows            = mla_gemm_fp8(codes, [W_DKV; W_KR]) [tokens, d_c + d_rope]
 *   cache          <- mla_cache_store(rows, positions)
 *   out             = absorb, decode, merge (or mla_prefill_mha)
 *   h''             = mla_gemm_fp8(mla_quantize_rows(out), W_O)
 *
 * Conventions are those of mla_gfx950.h: device pointers, caller-owned buffers,
 * a hipStream_t as void*, MLA_OK or a negative mla_status, arguments validated on
 * the host before anything is launched, no allocation, no state.
 *
 * 8-bit tensors are OCP e4m3 codes with fp32 scales; a value is code * scale.
 *  - rows (activations): codes [T, D], scales [ceil(D/128), T]: one scale per token
 *    and block of 128 columns (the last block may be short), the tokens of a block
 *    beside each other, as the product reads them.  scale = max|block| / 448, at
 *    least 2^-126, and 1 for a block of zeros; a code is value / scale, a quotient in
 *    fp32, rounded to nearest even.  A block that holds an infinity or a NaN gets a scale that is
 *    one, so that whatever is computed from it is not finite either.
 *  - weights: codes [N, K] (one output per row, as a linear layer stores them),
 *    scales [ceil(N/128), ceil(K/128)], one per 128 x 128 block.  Any positive
 *    scales may be passed, those of a published checkpoint for instance.
 */
#ifndef MLA_LAYER_GFX950_H
#define MLA_LAYER_GFX950_H

#include "mla_gfx950.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Which components of a rotated part of d_rope make up pair i. */
enum {
    MLA_ROPE_INTERLEAVED = 0, /* (2i, 2i + 1): consecutive pairs, as in the paper */
    MLA_ROPE_HALF        = 1  /* (i, i + d_rope/2)                                */
};

/* Frequencies of mla_rope_frequencies. */
enum {
    MLA_ROPE_PLAIN  = 0,  /* theta_i = base^(-2i/d_rope)                          */
    MLA_ROPE_LINEAR = 1,  /* theta_i / factor                                     */
    MLA_ROPE_YARN   = 2   /* between the two by how often a pair turns within the
                             original context length                              */
};

/*
 * RMS norm of hidden states, with the residual's addition before it and codes
 * after it where asked for.  For every token t:
 *
 *   s = x[t] + residual[t]                  (s = x[t] without a residual)
 *   y = s / sqrt(mean(s^2) + eps) * weight  (weight 1 where none is given)
 *
 *   x            [T, D] io dtype, rows x_pitch elements apart (x_pitch >= D)
 *   residual     [T, D] io dtype, dense; may be NULL
 *   residual_out [T, D] io dtype (output): s; NULL iff residual is.  May be
 *                residual itself, or x where x is dense
 *   weight       [D] io dtype; may be NULL
 *   y            [T, D] io dtype (output), may be NULL; may be x where x is dense
 *   codes        [T, D], scales [ceil(D/128), T] (output): y quantised before its
 *                rounding to the io dtype; both or neither.  y or codes is wanted
 * s and y are fp32 throughout and rounded once, where they are stored.  D up to
 * 32768, T below 2^23 (a workgroup per row, threads of a grid in 32 bits).
 */
int mla_rms_norm(const void* x, const void* residual, const void* weight, void* residual_out, void* y,
                 uint8_t* codes, float* scales, int T, int D, int64_t x_pitch, float eps, mla_dtype io_dtype,
                 void* hip_stream);

/*
 * Codes and scales of a tensor as it is (the operand of a product).
 *   x      [T, D] io dtype, rows x_pitch elements apart
 *   codes  [T, D], scales [ceil(D/128), T] (output).  D up to 32768, T below 2^23
 */
int mla_quantize_rows(const void* x, uint8_t* codes, float* scales, int T, int D, int64_t x_pitch,
                      mla_dtype io_dtype, void* hip_stream);

/*
 * Codes and scales of a weight matrix, once per matrix.
 *   w      [N, K] io dtype, dense
 *   codes  [N, K], scales [ceil(N/128), ceil(K/128)] (output)
 */
int mla_quantize_weights(const void* w, uint8_t* codes, float* scales, int N, int K,
                         mla_dtype io_dtype, void* hip_stream);

/* Flags of mla_gemm_fp8. */
enum {
    MLA_GEMM_DEFAULT   = 0,
    MLA_GEMM_FAST_SUMS = 1  /* the matrix cores may add the 8-bit products as they are,
                               at up to twice the rate, for any number of tokens (up to
                               16 by up to 4096 outputs have full sums all the same).
                               Their adders drop what lies 2^-13 below the largest of
                               eight neighbouring products: at most 7 * 2^-13 of the
                               sum of the products' magnitudes, more than a bf16
                               output's rounding where a result is far below that sum
                               and magnitudes differ widely among neighbours.  Random
                               operands give results 1.5e-5 off (2-norm)           */
};

/*
 * Bytes of device workspace mla_gemm_fp8 needs for these sizes (fp32 partial
 * products where the inner dimension is shared out over workgroups; 0 for many
 * sizes).  Pure host function; 0 if an argument is invalid.
 */
size_t mla_gemm_fp8_workspace_bytes(int M, int N, int K);

/*
 * Projection on codes:
 *   out[m, n] = sum_b a_scales[b, m] w_scales[n/128, b] sum_{k in block b} a[m, k] w[n, k]
 *
 *   a    [M, K] e4m3,  a_scales [ceil(K/128), M]
 *   w    [N, K] e4m3,  w_scales [ceil(N/128), ceil(K/128)]
 *   out  [M, N] out dtype (MLA_F32 or MLA_BF16)
 *   workspace  mla_gemm_fp8_workspace_bytes(M, N, K) bytes, 16-byte aligned (may
 *              be NULL where that is 0); scratch
 * K a multiple of 16 up to 2^23, a and w on 16 bytes, M and N up to 2^30 and no
 * more tiles than a grid holds (otherwise MLA_ERR_UNSUPPORTED).  Products are
 * exact and summed in fp32 (but see MLA_GEMM_FAST_SUMS), the blocks with their
 * scales in fp32 beside them (a token's scale times a weight block's is formed
 * first, and has to be in fp32's range itself); the order of the sums depends on the sizes alone,
 * so that a call's bits do not change from run to run.
 */
int mla_gemm_fp8(const uint8_t* a, const float* a_scales, const uint8_t* w, const float* w_scales, void* out,
                 void* workspace, size_t workspace_bytes, int M, int N, int K, mla_dtype out_dtype, unsigned flags,
                 void* hip_stream);

/*
 * Frequencies of a rotation, on the host (nothing is launched): freq[i], i <
 * d_rope / 2, radians per position of pair i, to be copied to the device once; and
 * *gain, the factor on the rotated part (1 except for MLA_ROPE_YARN).
 *   kind      MLA_ROPE_PLAIN, MLA_ROPE_LINEAR, MLA_ROPE_YARN
 *   factor    >= 1: how many times longer than the original the contexts are
 *   original  context length the model was trained on (YARN)
 * YARN (Peng et al. 2023, arXiv 2309.00071): with r_i = original theta_i / 2 pi turns
 * of pair i within that length, pairs of at least beta_fast turns keep theta_i, pairs
 * of at most beta_slow get theta_i / factor, those between are blended linearly in i
 * between the places where r_i takes the two values, the former rounded down (and at
 * least 0), the latter rounded up (which may be past the last pair: that one is then
 * blended too); gain = 0.1 ln(factor) + 1.
 */
int mla_rope_frequencies(double* freq, float* gain, int d_rope, double base, int kind, double factor,
                         int original, double beta_fast, double beta_slow);

/*
 * Queries as the projection leaves them, taken apart and rotated: what
 * mla_absorb_q and mla_decode_paged (or mla_prefill_mha) take.
 *
 *   q          [T, H, d_nope + d_rope] io dtype, heads dense, tokens q_pitch
 *              elements apart (q_pitch >= H (d_nope + d_rope)): the queries may be
 *              columns of a wider projection
 *   positions  [T] int32, any values
 *   freq       [d_rope / 2] fp64 (device), radians per position
 *   gain       factor on the rotated part
 *   layout     MLA_ROPE_INTERLEAVED or MLA_ROPE_HALF
 *   q_nope     [T, H, d_nope] (output; NULL iff d_nope is 0)
 *   q_rope     [T, H, d_rope] (output)
 * Pair i of the rotated part turns by positions[t] freq[i] (formed in fp64; the
 * turn itself is fp32).  d_rope even, 2 to 256; d_nope >= 0, H (d_nope + d_rope)
 * up to 2^30, T below 2^23, and no more heads' rows than a grid holds (at least 2^24, whatever
 * their width; otherwise MLA_ERR_UNSUPPORTED).
 */
int mla_rope_queries(const void* q, const int32_t* positions, const double* freq, void* q_nope, void* q_rope,
                     int T, int H, int d_nope, int d_rope, int64_t q_pitch, float gain, int layout,
                     mla_dtype io_dtype, void* hip_stream);

/*
 * Cache rows of new tokens from their projections, any number per sequence
 * (mla_cache_append multiplies the projection itself, for one token):
 *
 *   row = [ c | turn(k) ],  c as it is, or c / sqrt(mean(c^2) + eps) * norm_weight
 *
 *   rows        [B, new_tokens, d_c + d_rope] io dtype, rows row_pitch elements
 *               apart
 *   positions   [B, new_tokens] int32: logical position of each row, which is also
 *               what its rope part turns by.  A position outside the table, or a
 *               page id outside the pool, is not an error code: that row is skipped.
 *               No two rows of a call may name the same place
 *   freq, gain, layout   as for mla_rope_queries; the queries take the same
 *   norm_weight [d_c] io dtype; NULL: no norm
 *   kv_cache, kv_scale, page_table   as for mla_cache_append: rows are rounded once
 *               to the cache dtype, FP8 rows get scale = absmax/448 (1 for zeros)
 * io dtype F32 or BF16, cache dtype F32, BF16 or FP8_E4M3.  d_rope even, 0 to 256,
 * d_c >= 1, d_c + d_rope <= 1024, B new_tokens below 2^23.
 */
int mla_cache_store(const void* rows, const int32_t* positions, const double* freq, const void* norm_weight,
                    void* kv_cache, float* kv_scale, const int32_t* page_table, int B, int new_tokens,
                    int d_c, int d_rope, int64_t row_pitch, int page_size, int num_pages, int max_pages_per_seq,
                    float gain, int layout, float eps, mla_dtype io_dtype, mla_dtype cache_dtype, void* hip_stream);

/*
 * mla_cache_store for rows whose place is not their position (a drafted tree's: node k
 * of depth d turns by prefix + d and is stored at prefix + k).
 *   slots  [B, new_tokens] int32: logical position that each row is written to, with
 *          the rules that mla_cache_store has for positions; positions, any values, are
 *          only what the rope part turns by
 */
int mla_cache_store_at(const void* rows, const int32_t* positions, const int32_t* slots, const double* freq,
                       const void* norm_weight, void* kv_cache, float* kv_scale, const int32_t* page_table, int B,
                       int new_tokens, int d_c, int d_rope, int64_t row_pitch, int page_size, int num_pages,
                       int max_pages_per_seq, float gain, int layout, float eps, mla_dtype io_dtype,
                       mla_dtype cache_dtype, void* hip_stream);

/*
 * Cache rows moved within their sequences: row dst[b, i] of sequence b becomes its row
 * src[b, i], bit for bit, with its scale; e.g. the rows of a drafted tree's accepted path
 * to the places behind the committed rows, where the next step expects them.  All rows
 * of a sequence are read before any of them is written, so that places may be read and
 * written by one call.
 *
 *   kv_cache  [num_pages, page_size, row_bytes] bytes; kv_scale [num_pages, page_size]
 *             fp32 or NULL
 *   src, dst  [B, moves] int32 logical positions, moves <= 64.  An entry of which either
 *             lies outside the table, or on a page outside the pool, is skipped (-1 where
 *             a sequence has fewer moves).  No two entries of a call may write the same
 *             place, nor one write what another sequence's read (pages that sequences share)
 * B <= 65535, row_bytes <= 4096.
 */
int mla_cache_move(void* kv_cache, float* kv_scale, const int32_t* page_table, const int32_t* src, const int32_t* dst,
                   int B, int moves, int row_bytes, int page_size, int num_pages, int max_pages_per_seq,
                   void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MLA_LAYER_GFX950_H */
