// Declarations of the masked attention's kernels and entry points: which cached rows a query token sees.
#pragma once
#include "mla_internal.h"
#include "mla_masked_gfx950.h"

namespace mla {

// The absorbed form for the query rows of q_len tokens per sequence (token-major: row = token * heads + head).
struct MaskedParams {
    const void* q_abs;          // [B, H, d_c]     io dtype
    const void* q_rope;         // [B, H, d_rope]  io dtype
    const void* kv;             // [num_pages, page_size, d_c + d_rope] cache dtype
    const float* kv_scale;      // [num_pages, page_size] (fp8 cache) or nullptr
    const int32_t* page_table;  // [B, max_pages]
    const int32_t* lens;        // [B]: committed rows (a tree), or all of them (a window)
    const uint64_t* tree;       // [B, q_len] drafted rows that a token sees; nullptr: a window
    int64_t tree_pitch;
    void* o_part;               // [B, H, S, d_c]  chunk-normalised outputs in fp32 (S = 1: the output itself, in the io dtype)
    float* lse_part;            // [B, H, S]       (S = 1: the output's, or nullptr)
    int B, H, d_c, d_rope, page_size, num_pages, max_pages, num_splits;
    int q_len, heads, window, sinks;
    float scale;
};

constexpr int MK_TILE = 32;     // cached rows of a tile

// The tiles of a sequence that some token of the call may see, numbered without the gap between the sinks and the
// window: tile v is tile v, or v + skip from `head` on, of the sequence.
struct Reach {
    int end;                    // rows of the sequence
    int base;                   // a tree: its committed rows; a window: the position of token 0 (may be negative)
    int tiles, head, skip;
    __host__ __device__ __forceinline__ int tile(int v) const { return v < head ? v : v + skip; }
};

__host__ __device__ __forceinline__ Reach reach_of(int len, int q_len, int cap, bool tree, int window, int sinks)
{
    Reach r;
    len = len < 0 ? 0 : len > cap ? cap : len;
    r.head = r.skip = 0;
    if (tree) {
        r.base = len;
        r.end = len > cap - q_len ? cap : len + q_len;
        r.tiles = (r.end + MK_TILE - 1) / MK_TILE;
        return r;
    }
    r.base = len - q_len;
    r.end = len;
    r.tiles = (len + MK_TILE - 1) / MK_TILE;
    const int first = r.base - window + 1;                    // first row of token 0's window (the entry points see to it that it fits)
    const int first_tile = first > 0 ? first / MK_TILE : 0;
    r.head = ((sinks < len ? sinks : len) + MK_TILE - 1) / MK_TILE;
    if (first_tile > r.head) r.skip = first_tile - r.head;
    r.tiles -= r.skip;
    return r;
}

// most tiles that a sequence of the call can have (cap: rows of the page table)
inline int64_t most_tiles(int q_len, int64_t cap, bool tree, int window, int sinks)
{
    const int64_t all = (cap + MK_TILE - 1) / MK_TILE;
    if (tree) return all;
    const int64_t some = ((int64_t)sinks + MK_TILE - 1) / MK_TILE + ((int64_t)window + q_len - 1 + MK_TILE - 2) / MK_TILE + 1;
    return some < all ? some : all;
}

constexpr int MK_MAX_ROWS = 1 << 30;      // of a page table: windows, sinks and their sums fit 32 bits, and
constexpr int MK_MAX_CHUNKS = 64;         // so does a tile's number times this

// chunk s of S: tiles [chunk_start(s), chunk_start(s + 1))
__host__ __device__ __forceinline__ int chunk_start(int tiles, int s, int S) { return (int)((unsigned)tiles * (unsigned)s / (unsigned)S); }

// portable scalar-FMA kernel: every type pair, width and page size of mla_decode_paged
hipError_t launch_masked_portable(const MaskedParams& p, mla_dtype io, mla_dtype cache, hipStream_t s);
constexpr int MK_PORTABLE_ROWS = 4;       // query rows of a workgroup
// matrix-core kernel
inline bool masked_tall_width(int d_c) { return d_c == 256 || d_c == 512; }
bool       masked_tall_supported(const MaskedParams& p, mla_dtype io, mla_dtype cache);
hipError_t launch_masked_tall(const MaskedParams& p, mla_dtype cache, hipStream_t s);
constexpr int MK_TALL_ROWS = 128;
// the same with 32 query rows per workgroup, whose wavefronts take the tiles in turn; of what the other one supports
hipError_t launch_masked_thin(const MaskedParams& p, mla_dtype cache, int64_t tiles, hipStream_t s);
constexpr int MK_THIN_ROWS = 32;
// the chunks' results (S > 1) merged
hipError_t launch_masked_merge(const MaskedParams& p, void* o_lat, float* lse, mla_dtype io, hipStream_t s);

}  // namespace mla
