// Rotation of queries and cache rows.
//     queries: [nope | rope] rows of every head -> q_nope, q_rope, the rope part turned by position * freq
//     rows:    [c | k] -> c (normed where asked for), k turned, rounded to the cache's type, through the page table
// Both move every value once; the angles are worked out once per token, not per head.
#include "layer_internal.h"

#include <algorithm>
#include <type_traits>

namespace mla {
namespace {

constexpr int MAX_PAIRS = 128;

// (re + i im) (cs + i sn); which product is rounded first is fixed, so that every kernel gives the same bits
__device__ __forceinline__ float2 rotate(float re, float im, float cs, float sn)
{
    return make_float2(__builtin_fmaf(re, cs, -(im * sn)), __builtin_fmaf(re, sn, im * cs));
}

// ---------------------------------------------------------------- queries

// V values at a time.  A workgroup takes `tokens` tokens of `heads` heads: every thread asks for its values first, the
// turns of the tokens are worked out while they travel and go to LDS, the nope values leave as they came.  HALF: a thread
// holds the vector of real parts and that of imaginary parts; otherwise V / 2 whole pairs.
// Memory bound: 32768 tokens x 32 heads x (128 + 64) bf16, 805 MB moved in 128 - 131 us (6.2 TB/s); 16 tokens: 2.3 us from a
// graph, the launch and a round trip.
constexpr int ROPE_TOKENS = 16, ROPE_UNITS = 4;

// j / d for j < 2^21: the quotient's error, j / d 2^-22, stays below the half of 1 / d that separates it from the next whole number
__device__ __forceinline__ int divide(int j, float inv_d) { return (int)(((float)j + 0.5f) * inv_d); }

template <bool F32, bool HALF, int V, bool STREAM>
__global__ __launch_bounds__(256) void rope_queries_kernel(RopeParams p, int tokens, int heads, int groups)
{
    __shared__ float2 turns[ROPE_TOKENS * MAX_PAIRS];
    const int tid = threadIdx.x, pairs = p.d_rope / 2, width = p.d_nope + p.d_rope;
    const int t0 = (int)(blockIdx.x / groups) * tokens, h0 = (int)(blockIdx.x % groups) * heads;
    const int nt = min(tokens, p.T - t0), nh = min(heads, p.H - h0), rows = nt * nh;
    const int nv = p.d_nope / V, rv = (HALF ? pairs : p.d_rope) / V;       // vectors of a head's row
    const int n_nope = rows * nv, n_rope = rows * rv;
    const float inv_nv = 1.f / (float)max(nv, 1), inv_rv = 1.f / (float)rv, inv_nh = 1.f / (float)nh;
    using vec = std::conditional_t<V == 8 || F32, words4, words2>;
    constexpr int PARTS = F32 && V == 8 ? 2 : 1;                           // 16-byte accesses of a vector

    auto row_of = [&](int r, int& t, int& h) { t = divide(r, inv_nh); h = h0 + r - t * nh; t += t0; };
    // nope: copied as it lies, ROPE_UNITS vectors of a thread on their way at once
    auto nope = [&](int j0, auto store) {
        vec buf[ROPE_UNITS][PARTS];
        const int size = F32 ? 4 : 2;
#pragma unroll
        for (int i = 0; i < ROPE_UNITS; ++i) {
            const int j = j0 + i * 256 + tid;
            if (j >= n_nope) continue;
            const int r = divide(j, inv_nv);
            int t, h;
            row_of(r, t, h);
            const char* src = static_cast<const char*>(p.q) + ((int64_t)t * p.pitch + (int64_t)h * width + (j - r * nv) * V) * size;
#pragma unroll
            for (int k = 0; k < PARTS; ++k) buf[i][k] = reinterpret_cast<const vec*>(src)[k];
        }
        store();
#pragma unroll
        for (int i = 0; i < ROPE_UNITS; ++i) {
            const int j = j0 + i * 256 + tid;
            if (j >= n_nope) continue;
            const int r = divide(j, inv_nv);
            int t, h;
            row_of(r, t, h);
            char* dst = static_cast<char*>(p.q_nope) + (((int64_t)t * p.H + h) * p.d_nope + (j - r * nv) * V) * size;
#pragma unroll
            for (int k = 0; k < PARTS; ++k) put_words<STREAM>(reinterpret_cast<vec*>(dst) + k, buf[i][k]);
        }
    };
    using Raw = RawVec<F32, V>;
    auto load = [&](int j, Raw& a, Raw& b, int64_t& to, int& at) {
        const int r = divide(j, inv_rv), c = (j - r * rv) * V;
        int t, h;
        row_of(r, t, h);
        const int64_t from = (int64_t)t * p.pitch + (int64_t)h * width + p.d_nope + c;
        a = raw_vec<F32, V>(p.q, from);
        if (HALF) b = raw_vec<F32, V>(p.q, from + pairs);
        to = ((int64_t)t * p.H + h) * p.d_rope + c;
        at = (t - t0) * pairs + (HALF ? c : c / 2);
    };
    auto turn = [&](const Raw& ra, const Raw& rb, int64_t to, int at) {
        float a[V], b[V];
        values_of<F32, V>(ra, a);
        if constexpr (HALF) {
            values_of<F32, V>(rb, b);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float2 w = turns[at + k], z = rotate(a[k], b[k], w.x, w.y);
                a[k] = z.x;
                b[k] = z.y;
            }
            store_vec<F32, V, STREAM>(p.q_rope, to, a);
            store_vec<F32, V, STREAM>(p.q_rope, to + pairs, b);
        } else {
#pragma unroll
            for (int k = 0; k < V; k += 2) {
                const float2 w = turns[at + k / 2], z = rotate(a[k], a[k + 1], w.x, w.y);
                a[k] = z.x;
                a[k + 1] = z.y;
            }
            store_vec<F32, V, STREAM>(p.q_rope, to, a);
        }
    };

    Raw a[2], b[2];
    int64_t to[2];
    int at[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (i * 256 + tid < n_rope) load(i * 256 + tid, a[i], b[i], to[i], at[i]);
    nope(0, [&] {
        for (int i = tid; i < nt * pairs; i += 256) {
            const int t = i / pairs;
            float cs, sn;
            turn_of(p.positions[t0 + t], p.freq[i - t * pairs], p.gain, cs, sn);
            turns[i] = make_float2(cs, sn);
        }
    });
    for (int j0 = ROPE_UNITS * 256; j0 < n_nope; j0 += ROPE_UNITS * 256) nope(j0, [] {});
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (i * 256 + tid < n_rope) turn(a[i], b[i], to[i], at[i]);
    for (int j = 512 + tid; j < n_rope; j += 256) {
        load(j, a[0], b[0], to[0], at[0]);
        turn(a[0], b[0], to[0], at[0]);
    }
}

// any widths and addresses, value by value; one workgroup per token (32 heads of 128 + 64 in bf16 on an odd address: 4096 tokens
// 27 us, in vectors 15.5, 32768 tokens 280 and 128, 16 tokens 6.0 and 3.7)
template <bool F32, bool HALF>
__global__ __launch_bounds__(256) void rope_queries_any_kernel(RopeParams p)
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
        const float2 z = rotate(get(from + re), get(from + im), cs[i], sn[i]);
        put(p.q_rope, to + re, z.x);
        put(p.q_rope, to + im, z.y);
    }
}

// ---------------------------------------------------------------- cache rows

constexpr int MAX_ROW = 1024;

// where row r, of logical position pos, goes: its row of the pool, or -1 where it has no place
__device__ __forceinline__ int64_t place_of(const StoreParams& p, int r, int pos)
{
    if (pos < 0 || pos >= p.max_pages * p.page_size) return -1;                    // outside the table
    const int page = p.page_table[(int64_t)(r / p.new_tokens) * p.max_pages + pos / p.page_size];
    if (page < 0 || page >= p.num_pages) return -1;                                // outside the pool
    return (int64_t)page * p.page_size + pos % p.page_size;
}

// A wavefront per row, four rows per workgroup, so that a workgroup needs no barrier and its rows no order.  A lane holds eight
// values of c and a pair of k, whose turn it works out itself, NV times (512 NV >= d_c, 128 NV >= d_rope > 0).
// 32768 rows of 576 in bf16, the latents normed, are 75 MB in 15.5 us (4.9 TB/s; the launch, a round trip for position and
// page, and the stores count at this size), from fp32 to fp8 94 MB in 16.2 (5.8); one row each of 64 sequences 2.8 us.
template <bool F32, bool HALF, int CACHE, int NV>
__global__ __launch_bounds__(256) void cache_store_kernel(StoreParams p)
{
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = blockIdx.x * 4 + wave;
    if (r >= p.rows_total) return;
    const int n = p.d_c + p.d_rope, pairs = p.d_rope / 2, cv = p.d_c / 8;
    // Every load that depends on no other goes out before the first wait: lanes past the end repeat the last vector or pair
    // (with branches around the loads, and a wait in each, 18.1 us).
    const int64_t row = (int64_t)r * p.pitch;
    const uint16_t* halves = static_cast<const uint16_t*>(p.rows) + row;
    const float* words = static_cast<const float*>(p.rows) + row;
    const int pos = p.positions[r], slot = p.slots[r];
    RawVec<F32, 8> v_raw[NV], w_raw[NV];
    float re[NV], im[NV];
    uint32_t k_raw[NV];
    double freq[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) v_raw[i] = raw_vec<F32, 8>(p.rows, row + min(lane + i * 64, cv - 1) * 8);
    // columns of k that make up pair i
    auto re_at = [&](int i) { return p.d_c + (HALF ? i : 2 * i); };
    auto im_at = [&](int i) { return p.d_c + (HALF ? i + pairs : 2 * i + 1); };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = min(lane + i * 64, pairs - 1);
        if (F32) {
            re[i] = words[re_at(c)];
            im[i] = words[im_at(c)];
        } else {
            k_raw[i] = HALF ? halves[re_at(c)] | (uint32_t)halves[im_at(c)] << 16 : *reinterpret_cast<const uint32_t*>(halves + re_at(c));
        }
        freq[i] = p.freq[c];
    }
    if (p.norm_weight) {
#pragma unroll
        for (int i = 0; i < NV; ++i) w_raw[i] = raw_vec<F32, 8>(p.norm_weight, min(lane + i * 64, cv - 1) * 8);
    }
    __builtin_amdgcn_sched_barrier(0);
    const int64_t at = place_of(p, r, slot);
    if (at < 0) return;
    float v[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) values_of<F32, 8>(v_raw[i], v[i]);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (!F32) {
            re[i] = __uint_as_float(k_raw[i] << 16);
            im[i] = __uint_as_float(k_raw[i] & 0xFFFF0000u);
        }
        float cs, sn;
        turn_of(pos, freq[i], p.gain, cs, sn);
        const float2 z = rotate(re[i], im[i], cs, sn);
        re[i] = z.x;
        im[i] = z.y;
    }
    if (p.norm_weight) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (lane + i * 64 < cv) {
#pragma unroll
                for (int k = 0; k < 8; ++k) sum += v[i][k] * v[i][k];
            }
        const float inv = 1.f / sqrtf(wave_sum(sum) / (float)p.d_c + p.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float w[8];
            values_of<F32, 8>(w_raw[i], w);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[i][k] = v[i][k] * inv * w[k];
        }
    }
    Divisor by = {1.f, 1.f};
    if (CACHE == MLA_FP8_E4M3) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (lane + i * 64 < cv) {
#pragma unroll
                for (int k = 0; k < 8; ++k) top = max(top, magnitude(v[i][k]));
            }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (lane + i * 64 < pairs) top = max(top, max(magnitude(re[i]), magnitude(im[i])));
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        const float scale = block_scale(top);
        by = divisor(scale);
        if (lane == 0) p.kv_scale[at] = scale;
    }
    auto q = [&](float x) { return quotient(x, by); };
    const int64_t o = at * n;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = lane + i * 64;
        if (c >= cv) continue;
        if constexpr (CACHE == MLA_FP8_E4M3)
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.kv) + o + c * 8) =
                make_uint2(e4m3_quad(q(v[i][0]), q(v[i][1]), q(v[i][2]), q(v[i][3])), e4m3_quad(q(v[i][4]), q(v[i][5]), q(v[i][6]), q(v[i][7])));
        else
            store_vec<CACHE == MLA_F32, 8>(p.kv, o + c * 8, v[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = lane + i * 64;
        if (c >= pairs) continue;
        if constexpr (CACHE == MLA_F32) {
            float* dst = static_cast<float*>(p.kv) + o;
            dst[re_at(c)] = re[i];
            dst[im_at(c)] = im[i];
        } else if constexpr (CACHE == MLA_BF16) {
            const uint32_t two = bf16_pair(re[i], im[i]);
            uint16_t* dst = static_cast<uint16_t*>(p.kv) + o;
            if (HALF) {
                dst[re_at(c)] = (uint16_t)two;
                dst[im_at(c)] = (uint16_t)(two >> 16);
            } else {
                *reinterpret_cast<uint32_t*>(dst + re_at(c)) = two;
            }
        } else {
            const uint32_t two = e4m3_quad(q(re[i]), q(im[i]), 0.f, 0.f);
            uint8_t* dst = static_cast<uint8_t*>(p.kv) + o;
            if (HALF) {
                dst[re_at(c)] = (uint8_t)two;
                dst[im_at(c)] = (uint8_t)(two >> 8);
            } else {
                *reinterpret_cast<uint16_t*>(dst + re_at(c)) = (uint16_t)two;
            }
        }
    }
}

// any widths and addresses, and rows without a rotated part; one workgroup per row, the row in LDS as fp32 (32768 rows of 512 + 64
// from bf16 on an odd address: to bf16 44 us, in vectors 14, to fp8 53 and 15; of 512 + 0: 35 and 44; 64 rows 3.7 either way)
template <bool F32, bool HALF, int CACHE>
__global__ __launch_bounds__(256) void cache_store_any_kernel(StoreParams p)
{
    __shared__ float row[MAX_ROW];
    __shared__ float part[4];
    __shared__ uint32_t tops[4];
    const int r = blockIdx.x, tid = threadIdx.x;
    const int n = p.d_c + p.d_rope, pairs = p.d_rope / 2;
    const int pos = p.positions[r], slot = p.slots[r];
    const int64_t at = place_of(p, r, slot);
    if (at < 0) return;
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
        const float2 z = rotate(row[re], row[im], cs, sn);
        row[re] = z.x;
        row[im] = z.y;
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

bool on(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// How the queries are shared out: v values per access (0: any width and address, a workgroup per token), heads and tokens of a
// workgroup
struct RopePlan {
    int v, heads, tokens;
    int64_t grid(const RopeParams& p) const { return v ? (int64_t)((p.T + tokens - 1) / tokens) * ((p.H + heads - 1) / heads) : p.T; }
};

RopePlan rope_plan(const RopeParams& p, bool f32, bool half)
{
    // vectors of 8 or 4 values: they have to fit the parts of a head's row, and every row to lie on their bytes
    const int unit = half ? p.d_rope / 2 : p.d_rope;
    auto fits = [&](int v) {
        const int bytes = f32 ? 16 : 2 * v, per = bytes / (f32 ? 4 : 2);
        return p.d_nope % v == 0 && unit % v == 0 && p.pitch % per == 0 && on(p.q, bytes) && on(p.q_nope, bytes) && on(p.q_rope, bytes) &&
               p.d_nope <= 4096;
    };
    RopePlan plan = {fits(8) ? 8 : fits(4) ? 4 : 0, 1, 1};
    if (!plan.v) return plan;
    // As many heads' rows per workgroup as have 128 vectors to turn (32768 tokens x 32 heads, 8 / 16 / 32 rows: pairs 160 / 128 /
    // 141 us; 16 / 32 / 64: halves 131 / 142 / 148), fewer while that leaves CUs without one
    const int rows = std::max(1, 128 / (p.d_rope / plan.v));
    plan.heads = std::min(p.H, rows);
    plan.tokens = std::max(1, std::min(rows / plan.heads, ROPE_TOKENS));
    while (plan.grid(p) < 512 && plan.tokens > 1) plan.tokens = (plan.tokens + 1) / 2;
    while (plan.grid(p) < 512 && plan.heads > 4) plan.heads = (plan.heads + 1) / 2;
    return plan;
}

template <bool F32, bool HALF> void rope(const RopeParams& p, hipStream_t s)
{
    const RopePlan plan = rope_plan(p, F32, HALF);
    const dim3 grid((unsigned)plan.grid(p)), block(256);
    if (!plan.v) {
        rope_queries_any_kernel<F32, HALF><<<grid, block, 0, s>>>(p);
        return;
    }
    const int groups = (p.H + plan.heads - 1) / plan.heads;
    const bool stream = (int64_t)p.T * p.H * (p.d_nope + p.d_rope) * (F32 ? 4 : 2) > STREAM_BYTES;
    auto run = [&](auto vec) {
        constexpr int V = decltype(vec)::value;
        if (stream) rope_queries_kernel<F32, HALF, V, true><<<grid, block, 0, s>>>(p, plan.tokens, plan.heads, groups);
        else        rope_queries_kernel<F32, HALF, V, false><<<grid, block, 0, s>>>(p, plan.tokens, plan.heads, groups);
    };
    if (plan.v == 8) run(std::integral_constant<int, 8>{});
    else             run(std::integral_constant<int, 4>{});
}

template <bool F32, bool HALF, int CACHE> void store_rows(const StoreParams& p, hipStream_t s)
{
    const int n = p.d_c + p.d_rope;
    const bool vec = p.d_c % 8 == 0 && p.d_rope % 8 == 0 && p.d_rope > 0 && p.pitch % (F32 ? 4 : 8) == 0 && on(p.rows, 16) && on(p.norm_weight, 16) &&
                     on(p.kv, 16) && n <= MAX_ROW;
    const dim3 grid((unsigned)((p.rows_total + 3) / 4)), block(256);
    if (vec && p.d_c <= 512 && p.d_rope <= 128) cache_store_kernel<F32, HALF, CACHE, 1><<<grid, block, 0, s>>>(p);
    else if (vec) cache_store_kernel<F32, HALF, CACHE, 2><<<grid, block, 0, s>>>(p);
    else          cache_store_any_kernel<F32, HALF, CACHE><<<dim3((unsigned)p.rows_total), dim3(256), 0, s>>>(p);
}

template <bool F32, bool HALF> void store(const StoreParams& p, mla_dtype cache, hipStream_t s)
{
    if (cache == MLA_F32)       store_rows<F32, HALF, MLA_F32>(p, s);
    else if (cache == MLA_BF16) store_rows<F32, HALF, MLA_BF16>(p, s);
    else                        store_rows<F32, HALF, MLA_FP8_E4M3>(p, s);
}

}  // namespace

bool rope_queries_supported(const RopeParams& p, int layout, mla_dtype io)
{
    return rope_plan(p, io == MLA_F32, layout == MLA_ROPE_HALF).grid(p) < 1l << 24;              // (256 threads each)
}

hipError_t launch_rope_queries(const RopeParams& p, int layout, mla_dtype io, hipStream_t s)
{
    if (io == MLA_F32) layout == MLA_ROPE_HALF ? rope<true, true>(p, s) : rope<true, false>(p, s);
    else               layout == MLA_ROPE_HALF ? rope<false, true>(p, s) : rope<false, false>(p, s);
    return hipGetLastError();
}

hipError_t launch_cache_store(const StoreParams& p, int layout, mla_dtype io, mla_dtype cache, hipStream_t s)
{
    if (io == MLA_F32) layout == MLA_ROPE_HALF ? store<true, true>(p, cache, s) : store<true, false>(p, cache, s);
    else               layout == MLA_ROPE_HALF ? store<false, true>(p, cache, s) : store<false, false>(p, cache, s);
    return hipGetLastError();
}

}  // namespace mla
