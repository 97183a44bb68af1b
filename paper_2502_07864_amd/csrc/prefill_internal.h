// The prefill's own declarations: what its kernels and the entry point share.
#pragma once
#include "mla_internal.h"

namespace mla {

// Causal attention over materialised keys and values: a (sequence, head) pair, b * heads + h, has pages of its own and q_len
// query rows.
struct PrefillParams {
    const void* q_nope;         // [B, q_len, heads, 128] bf16
    const void* q_rope;         // [B, q_len, heads, 64]
    const void* pool;           // [pairs, max_pages] pages of 64 keys and values
    const int32_t* lens;        // [pairs]
    const void* rope;           // the keys' rope parts: of row 0 of page 0, and bytes from row to row (pages of 64 rows lie one
    int rope_pitch;             // behind the other).  16-byte aligned, both
    const int32_t* page_table;  // [B, max_pages]: their pages; an id outside [0, num_pages) leaves its 64 keys out
    int num_pages, max_pages;
    int pairs, q_len, heads;
    void* out;                  // [B, q_len, heads, 128] bf16
    float* lse;                 // [B, q_len, heads], or nullptr
    float scale;
    int window = 0, sinks = 0;  // window > 0: a query at row t sees the rows from t - window + 1 on, and those below sinks
    int splits = 1;             // (window) chunks that the pages of 128 query rows are cut into; with more than one the rows go to
    float* o_part = nullptr;    // [B, q_len, heads, splits, 128] and
    float* lse_part = nullptr;  // [B, q_len, heads, splits]
};

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// The workspace.  (Sized for keys with their rope part and a page table for every pair, as callers have sized it: the keys and values
// take four fifths of the pool's room, and rope parts that have to be copied, once for all heads, and their ids what they leave.)
struct PrefillWs {
    size_t pool_off, rope_off, ids_off, lens_off, total;
};
inline PrefillWs prefill_ws(int B, int heads, int d_c, int max_pages)
{
    PrefillWs w;
    w.pool_off = align_up((size_t)heads * 256 * d_c * 2, 256);                                   // after Wcat
    w.rope_off = w.pool_off + (size_t)B * heads * max_pages * 64 * 256 * 2;
    w.ids_off = w.pool_off + align_up((size_t)B * heads * max_pages * 64 * 320 * 2, 256);
    w.lens_off = w.ids_off + align_up((size_t)B * heads * max_pages * sizeof(int32_t), 256);
    w.total = w.lens_off + align_up((size_t)B * heads * sizeof(int32_t), 256);
    return w;
}

bool       prefill_supported(int d_head, int d_c, int d_rope, int page_size, mla_dtype io, mla_dtype cache);
// materialise [W_UK c | W_UV c] per pair into pool2, and the pairs' lengths.  window: with every value finite
hipError_t launch_prefill_materialise(const void* kv, const int32_t* page_table, const int32_t* seq_lens,
                                      const void* W_UK, const void* W_UV, void* Wcat, void* pool2, int32_t* lens2,
                                      int B, int q_len, int heads, int d_c, int num_pages, int max_pages,
                                      bool window, hipStream_t s);
// the rope parts of a cache that is not on 16 bytes: copied to dst, page by page of the sequences, [B * max_pages, 64, 64], and their
// ids there, [B, max_pages] (-1: not in the cache)
hipError_t launch_prefill_rope(const void* kv, const int32_t* page_table, const int32_t* seq_lens, void* dst, int32_t* ids,
                               int B, int d_c, int num_pages, int max_pages, hipStream_t s);
// The pages that some query of a call with a window sees (the sinks', then from the first query's window on), as a page table of
// their own and the sequences' lengths without the rows left out between them
hipError_t launch_window_pages(const int32_t* page_table, const int32_t* seq_lens, int32_t* pages, int32_t* lens, int B, int q_len,
                               int max_pages, int width, int window, int sinks, hipStream_t s);
hipError_t launch_prefill_attention(const PrefillParams& p, hipStream_t s);

}  // namespace mla
