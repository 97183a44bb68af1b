// Rotation of queries and cache rows.
//     queries: [nope | rope] rows of every head -> q_nope, q_rope, the rope part turned by position * freq
//     rows:    [c | k] -> c (normed where asked for), k turned, rounded to the cache's type, through the page table
// Both move every value once; the angles are worked out once per token, not per head.
#include "layer_internal.h"

namespace mla {
namespace {

constexpr int MAX_PAIRS = 128;

// One workgroup per token and group of heads: the token's turns go to LDS, then its values stream past.
template <bool F32, bool HALF>
__global__ __launch_bounds__(256) void rope_queries_kernel(RopeParams p)
{
    __shared__ float cs[MAX_PAIRS], sn[MAX_PAIRS];
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, pairs = p.d_rope / 2, width = p.d_nope + p.d_rope;
    if (tid < pairs) turn_of(p.positions[t], p.freq[tid], p.gain, cs[tid], sn[tid]);
    __syncthreads();
    auto get = [&](int64_t i) { return F32 ? static_cast<const float*>(p.q)[i] : bf16_bits_to_f32(static_cast<const uint16_t*>(p.q)[i]); };
    auto put = [&](void* base, int64_t i, float v) {
        if (F32) static_cast<float*>(base)[i] = v;
        else     static_cast<uint16_t*>(base)[i] = (uint16_t)f32_to_bf16_bits(v);
    };
    const int64_t src = t * p.pitch;
    for (int j = tid; j < p.H * p.d_nope; j += 256) {
        const int h = j / p.d_nope, c = j - h * p.d_nope;
        if (F32) static_cast<float*>(p.q_nope)[t * p.H * p.d_nope + j] = static_cast<const float*>(p.q)[src + (int64_t)h * width + c];
        else     static_cast<uint16_t*>(p.q_nope)[t * p.H * p.d_nope + j] = static_cast<const uint16_t*>(p.q)[src + (int64_t)h * width + c];
    }
    for (int j = tid; j < p.H * pairs; j += 256) {
        const int h = j / pairs, i = j - h * pairs;
        const int re = HALF ? i : 2 * i, im = HALF ? i + pairs : 2 * i + 1;
        const int64_t from = src + (int64_t)h * width + p.d_nope, to = (t * p.H + h) * (int64_t)p.d_rope;
        const float a = get(from + re), b = get(from + im);
        put(p.q_rope, to + re, a * cs[i] - b * sn[i]);
        put(p.q_rope, to + im, a * sn[i] + b * cs[i]);
    }
}

// One workgroup per row: the row in LDS as fp32, its rope part turned there, then rounded and stored.
constexpr int MAX_ROW = 1024;
template <bool F32, bool HALF, int CACHE>
__global__ __launch_bounds__(256) void cache_store_kernel(StoreParams p)
{
    __shared__ float row[MAX_ROW];
    __shared__ float part[4];
    __shared__ uint32_t tops[4];
    const int r = blockIdx.x, b = r / p.new_tokens, tid = threadIdx.x;
    const int n = p.d_c + p.d_rope, pairs = p.d_rope / 2;
    const int pos = p.positions[r];
    if (pos < 0 || pos >= p.max_pages * p.page_size) return;                       // outside the table
    const int page = p.page_table[(int64_t)b * p.max_pages + pos / p.page_size];
    if (page < 0 || page >= p.num_pages) return;                                   // outside the pool
    const int64_t at = (int64_t)page * p.page_size + pos % p.page_size;
    auto load = [&](const void* base, int64_t i) {
        return F32 ? static_cast<const float*>(base)[i] : bf16_bits_to_f32(static_cast<const uint16_t*>(base)[i]);
    };
    float sum = 0.f;
    for (int j = tid; j < n; j += 256) {
        const float v = load(p.rows, (int64_t)r * p.pitch + j);
        row[j] = v;
        if (j < p.d_c) sum += v * v;
    }
    float cs = 0.f, sn = 0.f;
    if (tid < pairs) turn_of(pos, p.freq[tid], p.gain, cs, sn);
    sum = wave_sum(sum);
    if (tid % 64 == 0) part[tid / 64] = sum;
    __syncthreads();
    if (p.norm_weight) {
        const float inv = 1.f / sqrtf((part[0] + part[1] + part[2] + part[3]) / (float)p.d_c + p.eps);
        for (int j = tid; j < p.d_c; j += 256) row[j] = row[j] * inv * load(p.norm_weight, j);
    }
    if (tid < pairs) {
        const int re = p.d_c + (HALF ? tid : 2 * tid), im = p.d_c + (HALF ? tid + pairs : 2 * tid + 1);
        const float x = row[re], y = row[im];
        row[re] = x * cs - y * sn;
        row[im] = x * sn + y * cs;
    }
    __syncthreads();
    if (CACHE == MLA_F32) {
        for (int j = tid; j < n; j += 256) static_cast<float*>(p.kv)[at * n + j] = row[j];
    } else if (CACHE == MLA_BF16) {
        for (int j = tid; j < n; j += 256) static_cast<uint16_t*>(p.kv)[at * n + j] = (uint16_t)f32_to_bf16_bits(row[j]);
    } else {
        uint32_t top = 0;
        for (int j = tid; j < n; j += 256) top = max(top, magnitude(row[j]));
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        if (tid % 64 == 0) tops[tid / 64] = top;
        __syncthreads();
        const float scale = block_scale(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
        for (int j = tid; j < n; j += 256) static_cast<uint8_t*>(p.kv)[at * n + j] = (uint8_t)e4m3_quad(row[j] / scale, 0.f, 0.f, 0.f);
        if (tid == 0) p.kv_scale[at] = scale;
    }
}

}  // namespace

hipError_t launch_rope_queries(const RopeParams& p, int layout, mla_dtype io, hipStream_t s)
{
    const dim3 grid((unsigned)p.T), block(256);
    if (io == MLA_F32) {
        if (layout == MLA_ROPE_HALF) rope_queries_kernel<true, true><<<grid, block, 0, s>>>(p);
        else                         rope_queries_kernel<true, false><<<grid, block, 0, s>>>(p);
    } else {
        if (layout == MLA_ROPE_HALF) rope_queries_kernel<false, true><<<grid, block, 0, s>>>(p);
        else                         rope_queries_kernel<false, false><<<grid, block, 0, s>>>(p);
    }
    return hipGetLastError();
}

namespace {
template <bool F32, bool HALF> void store_rows(const StoreParams& p, mla_dtype cache, hipStream_t s)
{
    const dim3 grid((unsigned)p.rows_total), block(256);
    if (cache == MLA_F32)       cache_store_kernel<F32, HALF, MLA_F32><<<grid, block, 0, s>>>(p);
    else if (cache == MLA_BF16) cache_store_kernel<F32, HALF, MLA_BF16><<<grid, block, 0, s>>>(p);
    else                        cache_store_kernel<F32, HALF, MLA_FP8_E4M3><<<grid, block, 0, s>>>(p);
}
}  // namespace

hipError_t launch_cache_store(const StoreParams& p, int layout, mla_dtype io, mla_dtype cache, hipStream_t s)
{
    if (io == MLA_F32) layout == MLA_ROPE_HALF ? store_rows<true, true>(p, cache, s) : store_rows<true, false>(p, cache, s);
    else               layout == MLA_ROPE_HALF ? store_rows<false, true>(p, cache, s) : store_rows<false, false>(p, cache, s);
    return hipGetLastError();
}

}  // namespace mla
