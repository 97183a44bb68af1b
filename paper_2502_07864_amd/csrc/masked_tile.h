// What the matrix-core kernels of the masked attention share.
#pragma once
#include "masked_internal.h"
#include <type_traits>
#include "mfma_tile.h"

namespace mla {

// the lane, worked out where it is needed instead of kept (in front of a loop whose registers are all taken)
__device__ __forceinline__ int lane_again()
{
    uint32_t all = ~0u;
    asm volatile("" : "+s"(all));
    return (int)__builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0u));
}

// Swizzle of piece 64 k + lane of an even number of rows of PPR pieces each, as bits of an address: (row & 6) << 4.  A comparison or two
// per piece instead of a register kept (or, as there are none left, spilled) for each.
template <int PPR> __device__ __forceinline__ uint32_t piece_key(int k, int lane)
{
    const int first = k * 64 / PPR / 2;              // half the row of lane 0
    uint32_t half = (uint32_t)first;
#pragma unroll
    for (int i = 1; i <= 2; ++i) {
        const int from = 2 * (first + i) * PPR - 64 * k;
        if (from < 64) half += lane >= from;
    }
    return (half & 3u) << 5;
}

// The chunk that XCD x takes as its `row`th: in turn from left to right and from right to left, so that where chunks come by falling length no
// XCD has the longer one every time (63 tokens x 28 heads on 64 sequences of 512 .. 4096 rows: 363 us all from left to right, 351)
__device__ __forceinline__ int chunk_at(int row, int x) { return row * 8 + (row & 1 ? 7 - x : x); }

// the sequence that workgroups of place i take: the longest first (up to 64 sequences: every workgroup ranks the lengths by itself; a long
// one started last would run on alone)
__device__ __forceinline__ int sequence_at(const MaskedParams& p, int i, int lane)
{
    if (p.B <= 1 || p.B > 64) return i;
    const int mine = lane < p.B ? p.lens[lane] : -1;
    int rank = 0;
    for (int j = 0; j < p.B; ++j) {
        const int other = __builtin_amdgcn_readlane(mine, j);
        rank += other > mine || (other == mine && j < lane);
    }
    return __builtin_amdgcn_readfirstlane(__builtin_ffsll((long long)__ballot(lane < p.B && rank == i)) - 1);
}

// Where the two halves of a tile, 16 rows each, lie in the pool, as numbers of 16 rows (page sizes are multiples of 16); -1: not there
struct Place {
    int lo, hi;
    __device__ __forceinline__ bool whole() const { return lo >= 0 && hi >= 0; }
    __device__ __forceinline__ uint32_t rows() const { return (lo >= 0 ? 0xFFFFu : 0u) | (hi >= 0 ? 0xFFFF0000u : 0u); }
};
// rows 16 k .. 16 k + 15 of the sequence, in two parts: the page's id, and what follows from it
__device__ __forceinline__ int half_page(const MaskedParams& p, const int32_t* table, int per_page, int k) { return table[min(k / per_page, p.max_pages - 1)]; }
__device__ __forceinline__ int half_at(const MaskedParams& p, int page, int per_page, int k)
{
    const int q = k / per_page;
    return q < p.max_pages && page >= 0 && page < p.num_pages ? page * per_page + (k - q * per_page) : -1;
}
template <typename Table>
__device__ __forceinline__ Place tile_place(const MaskedParams& p, Table table, int per_page, int tile)
{
    const int q = 2 * tile / per_page, r = 2 * tile - q * per_page;
    const bool on = r + 1 < per_page;                   // the second half lies on the same page
    const int q2 = on ? q : q + 1, first = table[q], second = table[min(q2, p.max_pages - 1)];
    auto at = [&](int page, int r) { return page >= 0 && page < p.num_pages ? page * per_page + r : -1; };
    return Place{at(first, r), q2 < p.max_pages ? at(second, on ? r + 1 : 0) : -1};
}

// Tiles that all of the tokens [first, last] see whole, where their pages are there: [0, whole) and [from, to)
struct WholeTiles {
    int whole, from, to;
    __device__ __forceinline__ bool holds(int v) const { return v < whole || (v >= from && v < to); }
};
__device__ __forceinline__ WholeTiles whole_tiles(const MaskedParams& p, const Reach& r, int first, int last)
{
    if (p.tree) return WholeTiles{r.base / MK_TILE, 0, 0};
    const int outside = r.base + last - p.window;       // last row that the last token does not see for its age
    const int end = max(0, r.base + first + 1);
    return WholeTiles{min(p.sinks, end) / MK_TILE, (outside < 0 ? 0 : outside / MK_TILE + 1) - r.skip, end / MK_TILE - r.skip};
}

__device__ __forceinline__ uint32_t low_bits(int k) { return k <= 0 ? 0u : k >= 32 ? ~0u : (1u << k) - 1u; }

// rows (bit: row) of the tile of rows [row, row + 32) that a token sees; mask: its word of the tree
__device__ __forceinline__ uint32_t visible_rows(const MaskedParams& p, const Reach& r, int row, int token, uint64_t mask)
{
    uint32_t sees;
    if (p.tree) {
        const int d = r.base - row;                     // committed rows of the tile
        sees = d >= 32 ? ~0u : d > 0 ? (uint32_t)(mask << d) | low_bits(d) : d > -64 ? (uint32_t)(mask >> -d) : 0u;
    } else {
        const int t = r.base + token;
        sees = low_bits(t + 1 - row) & (~low_bits(t - p.window + 1 - row) | low_bits(p.sinks - row));
    }
    return sees & low_bits(r.end - row);
}
__device__ __forceinline__ uint64_t tree_word(const MaskedParams& p, int b, int token)
{
    return p.tree[b * p.tree_pitch + token] & (p.q_len < 64 ? (1ull << p.q_len) - 1 : ~0ull);
}

// the two bf16 values of a word, zero where they are not finite
__device__ __forceinline__ uint32_t finite_halves(uint32_t w)
{
    if ((w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
    if ((w & 0x7F800000u) == 0x7F800000u) w &= 0xFFFFu;
    return w;
}

// the four e4m3 codes of a word, zero where they are NaN
__device__ __forceinline__ uint32_t finite_codes(uint32_t w)
{
#pragma unroll
    for (int s = 0; s < 32; s += 8)
        if ((w >> s & 0x7Fu) == 0x7Fu) w &= ~(0xFFu << s);
    return w;
}

// eight e4m3 codes in bf16, which holds them exactly
__device__ __forceinline__ bf16x8 widened(uint32_t lo, uint32_t up)
{
    auto two = [](uint32_t v, auto high) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 1.f, decltype(high)::value)); };
    return __builtin_bit_cast(bf16x8, (u32x4){two(lo, std::false_type{}), two(lo, std::true_type{}), two(up, std::false_type{}), two(up, std::true_type{})});
}

// maximum of three (a NaN loses, as in fmaxf; written out: fmaxf would quieten every operand first)
__device__ __forceinline__ float max_of(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// minimum of three (likewise)
__device__ __forceinline__ float min_of(float a, float b, float c)
{
    float r;
    asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// A score of a row that a query row sees which is not finite makes a NaN of the query row's sum, and of its result with it.  NaN and +inf do that by themselves; -inf, whose
// weight is zero, does it here: the sum plus zero times the least of a tile's scores.
__device__ __forceinline__ float with_least(float sum, f32x4 a, f32x4 b)
{
    const float least = min_of(min_of(min_of(a[0], a[1], a[2]), a[3], b[0]), min_of(b[1], b[2], b[3]), b[3]);
    return fmaf(least, 0.f, sum);
}
constexpr uint32_t QUIET_NAN = 0x7FC00000u;

// maximum over the four lane groups, on every lane
__device__ __forceinline__ float over_groups(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

}  // namespace mla
