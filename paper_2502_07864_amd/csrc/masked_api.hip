// C-ABI entry points of the masked attention: validation on the host, then launches.
#include "masked_internal.h"
#include "prefill_internal.h"

#include <algorithm>

using namespace mla;

namespace {

constexpr int MAX_QUERY_ROWS = 8192;      // of a sequence

// Kernels by the query rows that a workgroup takes, and what a call with one of them takes in us, near enough to choose by: a round of
// workgroups (one per CU; a chunk's groups of rows run on one XCD of 32, so it is the fullest that counts) its tiles and a start and end; the
// merge, if there are chunks, its launch and what the partial rows take to be written and read.  Measured at d_c = 512; a tile and a
// partial row grow with the row.  The sequences are taken to be as long as the table allows.
struct Kernel {
    int rows;
    double tile, start;
};
constexpr Kernel PORTABLE = {MK_PORTABLE_ROWS, 2.1, 11.0}, THIN = {MK_THIN_ROWS, 0.7, 7.0}, TALL = {MK_TALL_ROWS, 2.1, 11.0};

struct Plan {
    int S;                      // chunks that a sequence's tiles are cut into: those that end first
    double cost;
    size_t lse_off, total;      // of the workspace (S > 1)
    bool thin;
};

// Most bytes of partial results.  Where the query rows nearly fill the chip by themselves chunks only even out the last round of workgroups, and would take
// gigabytes: on 131136 rows 17 sequences of 63 x 32 query rows 9.3 ms with 938 MB, 9.5 with 603; 33 of 64 x 64 34 ms with 1851 MB, 37 with 529, 41 without chunks.
constexpr size_t MAX_PARTIALS = (size_t)640 << 20;

Plan plan_of(int B, int64_t H, int d_c, int64_t tiles, const Kernel& k)
{
    const int64_t Z = (H + k.rows - 1) / k.rows;
    const double wide = (d_c + 64) / 576.0;
    auto cost = [&](int s) {
        const double rounds = (double)((((int64_t)B * s + 7) / 8 * Z + 31) / 32);
        return rounds * ((double)((tiles + s - 1) / s) * k.tile * wide + k.start) + (s > 1 ? 6.0 + 6e-4 * wide * (double)(B * H) * s : 0.0);
    };
    Plan p = {1, cost(1), 0, 0, false};
    // (in floating point: sizes may be asked for that no call has)
    const int most = (int)std::min({(double)MK_MAX_CHUNKS, (double)tiles, (double)MAX_PARTIALS / ((double)B * (double)H * ((double)d_c + 1.0) * sizeof(float))});
    for (int s = 2; s <= most && B * Z < 4096; ++s)          // (4096: rounds enough; and what is left fits the merge's grid)
        if (const double c = cost(s); c < p.cost * 0.999) {
            p.S = s;
            p.cost = c;
        }
    p.lse_off = align_up((size_t)B * H * p.S * d_c * sizeof(float), 256);
    p.total = p.S > 1 ? p.lse_off + align_up((size_t)B * H * p.S * sizeof(float), 256) : 0;
    return p;
}

// What a call takes, on the matrix cores or not.  Groups of 32 rows read the tiles again for each (from L2), 128 rows wait longer for theirs: few rows or short
// chunks of them are better off as groups of 32 (256 rows on 1000 / 16000 / 64000 rows: 24.7, 42, 86 us by 128, 21.9, 34, 66 by 32), many are not
// (16 x 560 rows on 4000: 116, 192; 2 x 256 on 64000: 101, 112).
Plan choose(int B, int64_t H, int d_c, int64_t tiles, bool matrix)
{
    if (!matrix) return plan_of(B, H, d_c, tiles, PORTABLE);
    const Plan many = plan_of(B, H, d_c, tiles, TALL);
    Plan few = plan_of(B, H, d_c, tiles, THIN);
    few.thin = few.cost < many.cost;
    return few.thin ? few : many;
}

size_t workspace_bytes_for(int B, int q_len, int heads, int d_c, int64_t tiles)
{
    // (whether a call runs on the matrix cores hangs on its types, which are not asked for here)
    const int64_t H = (int64_t)q_len * heads;
    return std::max(choose(B, H, d_c, tiles, false).total, masked_tall_width(d_c) ? choose(B, H, d_c, tiles, true).total : 0);
}

bool sizes_ok(int B, int q_len, int heads, int d_c, int max_rows)
{
    return B > 0 && q_len > 0 && heads > 0 && d_c > 0 && max_rows > 0 && (int64_t)q_len * heads <= MAX_QUERY_ROWS;
}

int masked_call(MaskedParams p, void* o_lat, float* lse, void* workspace, size_t workspace_bytes, mla_dtype io, mla_dtype cache,
                unsigned flags, void* hip_stream)
{
    const bool tree = p.tree != nullptr;
    if (!p.q_abs || !p.kv || !p.page_table || !p.lens || !o_lat || (p.d_rope > 0 && !p.q_rope)) return MLA_ERR_NULL;
    if (p.B <= 0 || p.q_len <= 0 || p.heads <= 0 || p.d_c <= 0 || p.d_rope < 0 || p.page_size <= 0 || p.num_pages <= 0 ||
        p.max_pages <= 0 || !(p.scale == p.scale) || (!tree && (p.window < 1 || p.sinks < 0)) || p.tree_pitch < 0)
        return MLA_ERR_SHAPE;
    if ((int64_t)p.max_pages * p.page_size > 0x7FFFFFFF) return MLA_ERR_SHAPE;
    if ((int64_t)p.max_pages * p.page_size > MK_MAX_ROWS) return MLA_ERR_UNSUPPORTED;
    // (a window or sinks past the table's end are all that there is)
    p.window = std::min(p.window, p.max_pages * p.page_size);
    p.sinks = std::min(p.sinks, p.max_pages * p.page_size);
    if (tree && p.tree_pitch > 0 && p.tree_pitch < p.q_len) return MLA_ERR_SHAPE;
    if (io != MLA_F32 && io != MLA_BF16) return MLA_ERR_UNSUPPORTED;
    if (cache != MLA_F32 && cache != MLA_BF16 && cache != MLA_FP8_E4M3) return MLA_ERR_UNSUPPORTED;
    if (cache == MLA_F32 && io != MLA_F32) return MLA_ERR_UNSUPPORTED;
    if (cache == MLA_FP8_E4M3 && !p.kv_scale) return MLA_ERR_NULL;
    if (cache != MLA_FP8_E4M3 && p.kv_scale) return MLA_ERR_SHAPE;
    if (p.d_c > 512 || p.d_c % 8 || p.d_rope > 64 || p.d_rope % 8 || p.B > 65535 || (flags & ~(unsigned)MLA_FLAG_PORTABLE_KERNEL))
        return MLA_ERR_UNSUPPORTED;
    const int64_t H = (int64_t)p.q_len * p.heads;
    if (H > MAX_QUERY_ROWS || (tree && p.q_len > 64)) return MLA_ERR_UNSUPPORTED;
    p.H = (int)H;
    const int64_t tiles = most_tiles(p.q_len, (int64_t)p.max_pages * p.page_size, tree, p.window, p.sinks);
    const bool matrix = !(flags & MLA_FLAG_PORTABLE_KERNEL) && masked_tall_supported(p, io, cache);
    const Plan plan = choose(p.B, H, p.d_c, tiles, matrix);
    if (plan.total && (!workspace || workspace_bytes < plan.total || (reinterpret_cast<uintptr_t>(workspace) & 255u))) return MLA_ERR_WORKSPACE;
    p.num_splits = plan.S;
    if (plan.S == 1) {
        p.o_part = o_lat;
        p.lse_part = lse;
    } else {
        p.o_part = workspace;
        p.lse_part = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.lse_off);
    }
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipError_t e = plan.thin ? launch_masked_thin(p, cache, tiles, stream) : matrix ? launch_masked_tall(p, cache, stream) : launch_masked_portable(p, io, cache, stream);
    if (e == hipSuccess && plan.S > 1) e = launch_masked_merge(p, o_lat, lse, io, stream);
    return e == hipSuccess ? MLA_OK : MLA_ERR_HIP;
}

}  // namespace

extern "C" {

size_t mla_decode_tree_workspace_bytes(int B, int q_len, int heads, int d_c, int max_rows)
{
    if (!sizes_ok(B, q_len, heads, d_c, max_rows) || q_len > 64) return 0;
    return workspace_bytes_for(B, q_len, heads, d_c, most_tiles(q_len, max_rows, true, 1, 0));
}

size_t mla_decode_window_workspace_bytes(int B, int q_len, int heads, int d_c, int max_rows, int window, int sinks)
{
    if (!sizes_ok(B, q_len, heads, d_c, max_rows) || window < 1 || sinks < 0) return 0;
    return workspace_bytes_for(B, q_len, heads, d_c, most_tiles(q_len, max_rows, false, window, sinks));
}

int mla_decode_paged_tree(const void* q_abs, const void* q_rope, const void* kv_cache, const float* kv_scale,
                          const int32_t* page_table, const int32_t* prefix_lens, const uint64_t* tree_mask, int64_t mask_pitch,
                          void* o_lat, float* lse, void* workspace, size_t workspace_bytes, int B, int q_len, int heads, int d_c,
                          int d_rope, int page_size, int num_pages, int max_pages_per_seq, float softmax_scale, mla_dtype io_dtype,
                          mla_dtype cache_dtype, unsigned flags, void* hip_stream)
{
    if (!tree_mask) return MLA_ERR_NULL;
    MaskedParams p = {};
    p.q_abs = q_abs; p.q_rope = q_rope; p.kv = kv_cache; p.kv_scale = kv_scale; p.page_table = page_table; p.lens = prefix_lens;
    p.tree = tree_mask; p.tree_pitch = mask_pitch;
    p.B = B; p.d_c = d_c; p.d_rope = d_rope; p.page_size = page_size; p.num_pages = num_pages; p.max_pages = max_pages_per_seq;
    p.q_len = q_len; p.heads = heads; p.window = 1; p.sinks = 0; p.scale = softmax_scale;
    return masked_call(p, o_lat, lse, workspace, workspace_bytes, io_dtype, cache_dtype, flags, hip_stream);
}

int mla_decode_paged_window(const void* q_abs, const void* q_rope, const void* kv_cache, const float* kv_scale,
                            const int32_t* page_table, const int32_t* seq_lens, void* o_lat, float* lse, void* workspace,
                            size_t workspace_bytes, int B, int q_len, int heads, int d_c, int d_rope, int page_size, int num_pages,
                            int max_pages_per_seq, int window, int sinks, float softmax_scale, mla_dtype io_dtype,
                            mla_dtype cache_dtype, unsigned flags, void* hip_stream)
{
    MaskedParams p = {};
    p.q_abs = q_abs; p.q_rope = q_rope; p.kv = kv_cache; p.kv_scale = kv_scale; p.page_table = page_table; p.lens = seq_lens;
    p.B = B; p.d_c = d_c; p.d_rope = d_rope; p.page_size = page_size; p.num_pages = num_pages; p.max_pages = max_pages_per_seq;
    p.q_len = q_len; p.heads = heads; p.window = window; p.sinks = sinks; p.scale = softmax_scale;
    return masked_call(p, o_lat, lse, workspace, workspace_bytes, io_dtype, cache_dtype, flags, hip_stream);
}

// pages of a sequence that a call with a window can reach
static int reachable_pages(int q_len, int max_pages, int window, int sinks)
{
    const int64_t n = ((int64_t)sinks + 63) / 64 + ((int64_t)window + q_len - 1 + 62) / 64 + 1;
    return (int)std::min<int64_t>(n, max_pages);
}

// How many chunks the pages that 128 query rows of a prompt see are cut into: the S that ends first if a round of workgroups (two per CU)
// takes as long as its pages and four more for start and end, and the merge another four.  Not split / split like this (whole call, us; 28 heads,
// d_c = 256): 2 x 136 tokens on 10539 under 4096 169 / 124 (S = 4; 2 chunks 126, 8 chunks 132), 64 tokens of one prompt 129 / 51 (S = 13),
// 500 of one at d_c = 512 165 / 119, 2 x 136 under 1024 60 / 52.  8 x 500 under 1024 has 896 groups and stays as it is: 190, in two chunks 251.
static int prefill_chunks(int64_t pairs, int q_len, int width, int window, int sinks)
{
    const int64_t groups = pairs * (((int64_t)q_len + 127) / 128);
    const int64_t pages = std::min<int64_t>(width, ((int64_t)sinks + 63) / 64 + ((int64_t)window + 127 + 62) / 64 + 1);
    int best = 1;
    double least = 1e300;
    for (int s = 1; s <= 16 && s <= pages && groups * s <= 1024; ++s) {
        const double cost = (double)((groups * s + 511) / 512) * ((double)((pages + s - 1) / s) + 4.0) + (s > 1 ? 4.0 : 0.0);
        if (cost < least * 0.999) { least = cost; best = s; }
    }
    return best;
}

size_t mla_prefill_window_workspace_bytes(int B, int q_len, int heads, int d_c, int max_pages_per_seq, int window, int sinks)
{
    if (B <= 0 || q_len <= 0 || heads <= 0 || d_c <= 0 || max_pages_per_seq <= 0 || window < 1 || sinks < 0) return 0;
    const int width = reachable_pages(q_len, max_pages_per_seq, window, sinks);
    const int S = prefill_chunks((int64_t)B * heads, q_len, width, window, sinks);
    const size_t rows = (size_t)B * q_len * heads;
    return prefill_ws(B, heads, d_c, width).total + align_up((size_t)B * (width + 1) * sizeof(int32_t), 256) +
           (S > 1 ? align_up(rows * S * 128 * sizeof(float), 256) + align_up(rows * S * sizeof(float), 256) : 0);
}

int mla_prefill_window(const void* q_nope, const void* q_rope, const void* W_UK, const void* W_UV, const void* kv_cache,
                       const int32_t* page_table, const int32_t* seq_lens, void* out, float* lse, void* workspace,
                       size_t workspace_bytes, int B, int q_len, int heads, int d_head, int d_c, int d_rope, int page_size,
                       int num_pages, int max_pages_per_seq, int window, int sinks, float softmax_scale, mla_dtype io_dtype,
                       mla_dtype cache_dtype, void* hip_stream)
{
    if (!q_nope || !q_rope || !W_UK || !W_UV || !kv_cache || !page_table || !seq_lens || !out) return MLA_ERR_NULL;
    if (B <= 0 || q_len <= 0 || heads <= 0 || d_head <= 0 || d_c <= 0 || d_rope < 0 || page_size <= 0 || num_pages <= 0 ||
        max_pages_per_seq <= 0 || window < 1 || sinks < 0 || !(softmax_scale == softmax_scale))
        return MLA_ERR_SHAPE;
    if ((int64_t)max_pages_per_seq * page_size > 0x7FFFFFFF) return MLA_ERR_SHAPE;
    if (!prefill_supported(d_head, d_c, d_rope, page_size, io_dtype, cache_dtype)) return MLA_ERR_UNSUPPORTED;
    if ((int64_t)max_pages_per_seq * page_size > MK_MAX_ROWS || q_len > MK_MAX_ROWS / 2) return MLA_ERR_UNSUPPORTED;
    const int width = reachable_pages(q_len, max_pages_per_seq, window, sinks);
    const int64_t pairs = (int64_t)B * heads;
    if (pairs > 65535 || width > 65535 * 16 || pairs * width > 0x7FFFFFFF || (pairs + 7) / 8 * 8 * (((int64_t)q_len + 63) / 64) > 0x7FFFFFFF)
        return MLA_ERR_UNSUPPORTED;
    const PrefillWs wl = prefill_ws(B, heads, d_c, width);
    if (!workspace || workspace_bytes < mla_prefill_window_workspace_bytes(B, q_len, heads, d_c, max_pages_per_seq, window, sinks) ||
        (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return MLA_ERR_WORKSPACE;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    char* ws = static_cast<char*>(workspace);
    int32_t* pages = reinterpret_cast<int32_t*>(ws + wl.total);
    int32_t* lens = pages + (size_t)B * width;
    int32_t* lens2 = reinterpret_cast<int32_t*>(ws + wl.lens_off);
    hipError_t e = launch_window_pages(page_table, seq_lens, pages, lens, B, q_len, max_pages_per_seq, width, window, sinks, stream);
    if (e != hipSuccess) return MLA_ERR_HIP;
    e = launch_prefill_materialise(kv_cache, pages, lens, W_UK, W_UV, ws, ws + wl.pool_off, lens2, B, q_len, heads, d_c, num_pages, width, true, stream);
    if (e != hipSuccess) return MLA_ERR_HIP;
    PrefillParams p;
    p.q_nope = q_nope; p.q_rope = q_rope; p.pool = ws + wl.pool_off; p.lens = lens2;
    p.rope = static_cast<const uint16_t*>(kv_cache) + d_c; p.rope_pitch = (d_c + d_rope) * 2;
    p.page_table = pages; p.num_pages = num_pages; p.max_pages = width;
    if (reinterpret_cast<uintptr_t>(kv_cache) & 15u) {       // direct-to-LDS loads are not documented to take it
        int32_t* ids = reinterpret_cast<int32_t*>(ws + wl.ids_off);
        e = launch_prefill_rope(kv_cache, pages, lens, ws + wl.rope_off, ids, B, d_c, num_pages, width, stream);
        if (e != hipSuccess) return MLA_ERR_HIP;
        p.rope = ws + wl.rope_off; p.rope_pitch = d_rope * 2;
        p.page_table = ids; p.num_pages = B * width;
    }
    p.pairs = (int)pairs; p.q_len = q_len; p.heads = heads; p.out = out; p.lse = lse;
    p.scale = softmax_scale;
    // (a window or sinks past the table's end are all that there is)
    const int rows = max_pages_per_seq * page_size;
    p.window = std::min(window, rows); p.sinks = std::min(sinks, rows);
    p.splits = prefill_chunks(pairs, q_len, width, window, sinks);
    if (p.splits > 1) {
        const size_t rows = (size_t)pairs * q_len;
        p.o_part = reinterpret_cast<float*>(ws + wl.total + align_up((size_t)B * (width + 1) * sizeof(int32_t), 256));
        p.lse_part = reinterpret_cast<float*>(reinterpret_cast<char*>(p.o_part) + align_up(rows * p.splits * 128 * sizeof(float), 256));
    }
    e = launch_prefill_attention(p, stream);
    if (e == hipSuccess && p.splits > 1) {
        MaskedParams m = {};
        m.B = B; m.H = q_len * heads; m.d_c = d_head; m.num_splits = p.splits; m.o_part = p.o_part; m.lse_part = p.lse_part;
        e = launch_masked_merge(m, out, lse, io_dtype, stream);
    }
    return e == hipSuccess ? MLA_OK : MLA_ERR_HIP;
}

}  // extern "C"
