// Masked attention over the latent cache on scalar FMAs: every type pair, width and page size that mla_decode_paged takes, the
// only path for fp32, for pages that are no multiple of 16 rows and for tensors off 16 bytes.
//
//   s_j = scale (q_abs . c_j + q_rope . k_j),  p = softmax over the rows j that the token sees,  o = sum_j p_j c_j
//
// A workgroup takes a chunk of a sequence's tiles for four query rows; its four wavefronts take the chunk's rows four at a time,
// in turn.  A row lies in the registers of one wavefront, lane l holding the latent values 4 l .. 4 l + 3, the four from 256
// further on and (the first lanes) four of the rope part: the same registers serve score and sum.  A running softmax per wavefront,
// joined over the four at the end.  What a row that a token does not see holds is never multiplied, not even by zero.
//
// Bound by vector instructions and, with two wavefronts per SIMD, by the waits for rows between them: 57 for a row and a query row, of which 20 are products (the sum over the wavefront
// takes seven, exponentials and masks most of the rest).  8 tokens x 32 heads on 4 x 4096 rows in fp32: 561 us, 16 TFLOP/s, vector pipes busy 72 % of the time, wavefronts waiting for data
// 37 % of theirs; the same in bf16 and pages of 8 rows 684, 50 % and 59 % (the matrix cores' kernels in pages of 16: 34).
#include "masked_internal.h"
#include <type_traits>

namespace mla {
namespace {

constexpr int PM_HG = MK_PORTABLE_ROWS, PM_ROWS = 4, PM_WAVES = 4;
constexpr int PM_MAX_DC = 512;

struct bf16_tag {};
struct fp8_tag {};

template <typename T> __device__ __forceinline__ float4 load4(const void* base, size_t elem)
{
    if constexpr (std::is_same_v<T, float>) {
        return *reinterpret_cast<const float4*>(static_cast<const float*>(base) + elem);
    } else if constexpr (std::is_same_v<T, bf16_tag>) {
        return load_part4<true>(base, elem);
    } else {
        const uint32_t v = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(base) + elem);
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(v, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(v, true);
        return make_float4(lo[0], lo[1], hi[0], hi[1]);
    }
}

__device__ __forceinline__ float dot4(float4 a, float4 b, float s) { return fmaf(a.w, b.w, fmaf(a.z, b.z, fmaf(a.y, b.y, fmaf(a.x, b.x, s)))); }
__device__ __forceinline__ void add4(float4& a, float w, float4 v)
{
    a.x = fmaf(w, v.x, a.x); a.y = fmaf(w, v.y, a.y); a.z = fmaf(w, v.z, a.z); a.w = fmaf(w, v.w, a.w);
}

template <typename QT, typename CT>
__global__ __launch_bounds__(64 * PM_WAVES) void masked_portable_kernel(MaskedParams p)
{
    __shared__ __attribute__((aligned(16))) float o_s[PM_WAVES][PM_HG][PM_MAX_DC];
    __shared__ float m_s[PM_WAVES][PM_HG], l_s[PM_WAVES][PM_HG];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the groups of query rows of one chunk get linear ids 8 apart: same XCD, so all but the first find the rows in its L2
    const int Z = (p.H + PM_HG - 1) / PM_HG;
    const long id = (long)blockIdx.y * gridDim.x + blockIdx.x, rr = id >> 3;
    const long wg = (rr / Z) * 8 + (id & 7);
    if (wg >= (long)p.B * p.num_splits) return;
    const int h0 = (int)(rr % Z) * PM_HG, split = (int)(wg % p.num_splits), b = (int)(wg / p.num_splits);
    const int nh = min(PM_HG, p.H - h0), row = p.d_c + p.d_rope;
    const Reach reach = reach_of(p.lens[b], p.q_len, p.max_pages * p.page_size, p.tree != nullptr, p.window, p.sinks);
    const int v0 = chunk_start(reach.tiles, split, p.num_splits) * MK_TILE, v1 = chunk_start(reach.tiles, split + 1, p.num_splits) * MK_TILE;

    const bool has[3] = {4 * lane < p.d_c, 256 + 4 * lane < p.d_c, 4 * lane < p.d_rope};
    float4 q[PM_HG][3], acc[PM_HG][2];
    uint64_t sees[PM_HG];          // a tree: the token's mask
    int at[PM_HG];                 // a window: the token's position
    float m[PM_HG], l[PM_HG];
#pragma unroll
    for (int h = 0; h < PM_HG; ++h) {
        const int hq = h0 + min(h, nh - 1), token = hq / p.heads;
        const size_t bh = (size_t)b * p.H + hq;
        sees[h] = p.tree ? p.tree[b * p.tree_pitch + token] : 0;
        at[h] = reach.base + token;
#pragma unroll
        for (int c = 0; c < 3; ++c)
            q[h][c] = !has[c] ? make_float4(0.f, 0.f, 0.f, 0.f) : c < 2 ? load4<QT>(p.q_abs, bh * p.d_c + c * 256 + 4 * lane)
                                                                       : load4<QT>(p.q_rope, bh * p.d_rope + 4 * lane);
        acc[h][0] = acc[h][1] = make_float4(0.f, 0.f, 0.f, 0.f);
        m[h] = -INFINITY;
        l[h] = 0.f;
    }
    auto visible = [&](int h, int j) {
        if (p.tree) return j < reach.base || (j - reach.base < p.q_len && ((sees[h] >> (j - reach.base)) & 1u));
        return j <= at[h] && (j > (int64_t)at[h] - p.window || j < p.sinks);
    };

    for (int vb = v0 + wave * PM_ROWS; vb < v1; vb += PM_WAVES * PM_ROWS) {
        const int jb = vb < reach.head * MK_TILE ? vb : vb + reach.skip * MK_TILE;      // (a batch lies in one tile)
        // lane r < 4 looks up row r (-1: past the sequence, or on a page outside the pool)
        long where = -1;
        float scale = 1.f;
        if (lane < PM_ROWS && jb + lane < reach.end) {
            const int page = p.page_table[(size_t)b * p.max_pages + (jb + lane) / p.page_size];
            if (page >= 0 && page < p.num_pages) {
                where = (long)page * p.page_size + (jb + lane) % p.page_size;
                if constexpr (std::is_same_v<CT, fp8_tag>) scale = p.kv_scale[where];
            }
        }
        const unsigned there = (unsigned)__ballot(where >= 0);
        if (!there) continue;
        float4 x[PM_ROWS][3];
#pragma unroll
        for (int r = 0; r < PM_ROWS; ++r) {
            const long a = max(0L, (long)(((unsigned long)(unsigned)__builtin_amdgcn_readlane((int)(where >> 32), r) << 32) |
                                          (unsigned)__builtin_amdgcn_readlane((int)where, r)));
            const size_t base = (size_t)a * row + 4 * lane;
#pragma unroll
            for (int c = 0; c < 3; ++c)
                x[r][c] = has[c] ? load4<CT>(p.kv, base + (c == 0 ? 0 : c == 1 ? 256 : p.d_c)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int h = 0; h < PM_HG; ++h) {
            // scores of the four rows, on every lane
            float s[PM_ROWS], tm = -INFINITY;
            bool seen[PM_ROWS];
#pragma unroll
            for (int r = 0; r < PM_ROWS; ++r) {
                const float d = wave_sum(dot4(q[h][2], x[r][2], dot4(q[h][1], x[r][1], dot4(q[h][0], x[r][0], 0.f))));
                seen[r] = ((there >> r) & 1u) && visible(h, jb + r);
                s[r] = seen[r] ? d * lane_value(scale, r) * p.scale : -INFINITY;
                tm = fmaxf(tm, s[r]);
            }
            const float top = fmaxf(m[h], tm);
            const float ref = top == -INFINITY ? 0.f : top;    // (scores of -inf have no weight, a NaN stays one)
            if (top != m[h]) {
                const float f = expf(m[h] - top);              // (0 on the first rows)
                l[h] *= f;
                acc[h][0] = make_float4(acc[h][0].x * f, acc[h][0].y * f, acc[h][0].z * f, acc[h][0].w * f);
                acc[h][1] = make_float4(acc[h][1].x * f, acc[h][1].y * f, acc[h][1].z * f, acc[h][1].w * f);
                m[h] = top;
            }
#pragma unroll
            for (int r = 0; r < PM_ROWS; ++r) {
                if (!seen[r]) continue;                        // (uniform)
                const float e = expf(s[r] - ref), w = e * lane_value(scale, r);
                l[h] = fmaf(s[r], 0.f, l[h] + e);              // (a NaN for good where the score is infinite: -inf alone would have the weight zero)
                add4(acc[h][0], w, x[r][0]);
                add4(acc[h][1], w, x[r][1]);
            }
        }
    }

    // ---- the wavefronts' states joined
#pragma unroll
    for (int h = 0; h < PM_HG; ++h) {
        if (lane == 0) { m_s[wave][h] = m[h]; l_s[wave][h] = l[h]; }
        if (has[0]) *reinterpret_cast<float4*>(&o_s[wave][h][4 * lane]) = acc[h][0];
        if (has[1]) *reinterpret_cast<float4*>(&o_s[wave][h][256 + 4 * lane]) = acc[h][1];
    }
    __syncthreads();
    for (int h = wave; h < nh; h += PM_WAVES) {
        float mt = -INFINITY;
#pragma unroll
        for (int w = 0; w < PM_WAVES; ++w) mt = fmaxf(mt, m_s[w][h]);
        float f[PM_WAVES], lt = 0.f;
#pragma unroll
        for (int w = 0; w < PM_WAVES; ++w) {
            f[w] = l_s[w][h] == 0.f ? 0.f : m_s[w][h] == -INFINITY ? 1.f : expf(m_s[w][h] - mt);     // (-inf with a sum: a NaN)
            lt = fmaf(l_s[w][h], f[w], lt);
        }
        const bool nothing = lt == 0.f;                        // (a NaN is something)
        const size_t pi = part_index(b, h0 + h, split, p.H, p.num_splits);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            if (!has[c]) continue;
            const int col = c * 256 + 4 * lane;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < PM_WAVES; ++w)
                if (l_s[w][h] != 0.f) add4(o, f[w], *reinterpret_cast<const float4*>(&o_s[w][h][col]));
            const float inv = nothing ? 0.f : 1.f / lt;
            o = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
            if (std::is_same_v<QT, bf16_tag> && p.num_splits == 1)
                *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.o_part) + pi * p.d_c + col) =
                    make_uint2(f32_to_bf16_bits(o.x) | (f32_to_bf16_bits(o.y) << 16), f32_to_bf16_bits(o.z) | (f32_to_bf16_bits(o.w) << 16));
            else
                *reinterpret_cast<float4*>(static_cast<float*>(p.o_part) + pi * p.d_c + col) = o;
        }
        if (lane == 0 && p.lse_part) p.lse_part[pi] = nothing ? -INFINITY : mt + logf(lt);
    }
}

template <typename QT, typename CT> hipError_t launch(const MaskedParams& p, hipStream_t s)
{
    const long long n = ((long long)p.B * p.num_splits + 7) / 8 * 8, wgs = n * ((p.H + PM_HG - 1) / PM_HG);
    const long long gx = wgs < (1 << 20) ? wgs : 1 << 20, gy = (wgs + gx - 1) / gx;   // a grid dimension holds 2^32 threads
    if (gy > 65535) return hipErrorInvalidValue;
    masked_portable_kernel<QT, CT><<<dim3((unsigned)gx, (unsigned)gy), dim3(64 * PM_WAVES), 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_masked_portable(const MaskedParams& p, mla_dtype io, mla_dtype cache, hipStream_t s)
{
    if (io == MLA_F32 && cache == MLA_F32) return launch<float, float>(p, s);
    if (io == MLA_F32 && cache == MLA_BF16) return launch<float, bf16_tag>(p, s);
    if (io == MLA_F32 && cache == MLA_FP8_E4M3) return launch<float, fp8_tag>(p, s);
    if (io == MLA_BF16 && cache == MLA_BF16) return launch<bf16_tag, bf16_tag>(p, s);
    if (io == MLA_BF16 && cache == MLA_FP8_E4M3) return launch<bf16_tag, fp8_tag>(p, s);
    return hipErrorInvalidValue;
}

}  // namespace mla
