// Parameters and launchers of the operators around the attention (mla_layer_gfx950.h).
#pragma once
#include "mla_internal.h"
#include "mla_layer_gfx950.h"

#include <type_traits>

namespace mla {

constexpr int QBLOCK = 128;        // columns (and weight rows) per scale
constexpr float E4M3_MAX = 448.f;
// Outputs of a call beyond this many bytes together go past the caches (us of the call, kept / streamed: queries of 32768 tokens x 32
// heads 167 / 131, norm of 32768 x 4096 165 / 159, product of 32768 x 6144 697 / 659, each pair on one card; at 8192 tokens and
// below no difference).  What it costs the call that reads them next has not been measured: of the norm's outputs the codes, a third of
// the bytes, are read at once, by two products.
constexpr int64_t STREAM_BYTES = (int64_t)64 << 20;

struct NormParams {
    const void* x;
    const void* residual;      // or nullptr
    const void* weight;        // or nullptr
    void* residual_out;
    void* y;                   // or nullptr
    uint8_t* codes;            // or nullptr
    float* scales;
    int T, D;
    int64_t x_pitch;
    float eps;
};

struct GemmFp8Params {
    const uint8_t* a;          // [M, K]
    const float* a_scales;     // [ceil(K/128), M]
    const uint8_t* w;          // [N, K]
    const float* w_scales;     // [ceil(N/128), ceil(K/128)]
    void* out;                 // [M, N]
    float* part;               // workspace
    int M, N, K;
    int scale_pitch;           // tokens per row of a_scales
};

struct RopeParams {
    const void* q;
    const int32_t* positions;
    const double* freq;
    void* q_nope;
    void* q_rope;
    int T, H, d_nope, d_rope;
    int64_t pitch;
    float gain;
};

struct StoreParams {
    const void* rows;
    const int32_t* positions;
    const double* freq;
    const void* norm_weight;   // or nullptr
    void* kv;
    float* kv_scale;
    const int32_t* page_table;
    int rows_total, new_tokens, d_c, d_rope, page_size, num_pages, max_pages;
    int64_t pitch;
    float gain, eps;
};

// the norm (norm = true) or the codes of x as it is
hipError_t launch_rms_norm(const NormParams& p, bool norm, mla_dtype io, hipStream_t s);
hipError_t launch_quantize_weights(const void* w, uint8_t* codes, float* scales, int N, int K, mla_dtype io, hipStream_t s);
size_t     gemm_fp8_workspace(int M, int N, int K);
bool       gemm_fp8_supported(int M, int N, int K);      // (the grid's threads are counted in 32 bits)
hipError_t launch_gemm_fp8(const GemmFp8Params& p, mla_dtype out, bool fast_sums, hipStream_t s);
bool       rope_queries_supported(const RopeParams& p, int layout, mla_dtype io);      // (the same)
hipError_t launch_rope_queries(const RopeParams& p, int layout, mla_dtype io, hipStream_t s);
hipError_t launch_cache_store(const StoreParams& p, int layout, mla_dtype io, mla_dtype cache, hipStream_t s);

// ---- device helpers

typedef __attribute__((ext_vector_type(4))) uint32_t words4;
typedef __attribute__((ext_vector_type(2))) uint32_t words2;

// V (8 or 4) consecutive values in accesses of up to 16 bytes, which the address has to allow.  As they come (raw_vec) and as
// floats (values_of): kernels ask for all they can before they unpack any, or the compiler waits for each in turn.
template <bool F32, int V> struct RawVec {
    static constexpr int N = F32 && V == 8 ? 2 : 1;
    std::conditional_t<F32 || V == 8, words4, words2> w[N];
};
template <bool F32, int V> __device__ __forceinline__ RawVec<F32, V> raw_vec(const void* base, int64_t at)
{
    RawVec<F32, V> r;
    const auto* src = reinterpret_cast<const std::remove_reference_t<decltype(r.w[0])>*>(static_cast<const char*>(base) + at * (F32 ? 4 : 2));
#pragma unroll
    for (int i = 0; i < r.N; ++i) r.w[i] = src[i];
    return r;
}
template <bool F32, int V> __device__ __forceinline__ void values_of(const RawVec<F32, V>& r, float (&v)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t word = F32 ? r.w[i / 4 % r.N][i % 4] : r.w[0][i / 2];
        v[i] = __uint_as_float(F32 ? word : i % 2 ? word & 0xFFFF0000u : word << 16);
    }
}
template <bool F32, int V> __device__ __forceinline__ void load_vec(const void* base, int64_t at, float (&v)[V])
{
    values_of<F32, V>(raw_vec<F32, V>(base, at), v);
}

// two values as bf16, each rounded to nearest even (v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    typedef __attribute__((ext_vector_type(2))) float f2;
    typedef __attribute__((ext_vector_type(2))) __bf16 b2;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){lo, hi}, b2));
}

// STREAM: past the caches
template <bool STREAM, typename W> __device__ __forceinline__ void put_words(void* dst, W w)
{
    if constexpr (STREAM) __builtin_nontemporal_store(w, static_cast<W*>(dst));
    else                  *static_cast<W*>(dst) = w;
}

// accesses at any address of a value (the hardware takes them apart where they cross a line)
typedef words4 __attribute__((aligned(2))) words4_any;
typedef words2 __attribute__((aligned(1))) words2_any;
typedef uint32_t __attribute__((aligned(1))) word_any;
typedef uint16_t __attribute__((aligned(1))) half_any;
template <bool STREAM> __device__ __forceinline__ void put_words_any(void* dst, words4 w)
{
    if constexpr (STREAM) __builtin_nontemporal_store(w, static_cast<words4_any*>(dst));
    else                  *static_cast<words4_any*>(dst) = w;
}

template <bool F32, int V, bool STREAM = false> __device__ __forceinline__ void store_vec(void* base, int64_t at, const float (&v)[V])
{
    if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < V; i += 4)
            put_words<STREAM>(static_cast<float*>(base) + at + i,
                              (words4){__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])});
    } else if constexpr (V == 8) {
        put_words<STREAM>(static_cast<uint16_t*>(base) + at, (words4){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])});
    } else {
        put_words<STREAM>(static_cast<uint16_t*>(base) + at, (words2){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])});
    }
}

// Eight consecutive values at any address of the type.  Fewer than eight, `left`: four, two and one of them, as its bits say.
template <bool F32> __device__ __forceinline__ RawVec<F32, 8> raw8_any(const void* base, int64_t at)
{
    RawVec<F32, 8> r;
    const words4_any* src = reinterpret_cast<const words4_any*>(static_cast<const char*>(base) + at * (F32 ? 4 : 2));
#pragma unroll
    for (int i = 0; i < r.N; ++i) r.w[i] = src[i];
    return r;
}
template <bool F32> __device__ __forceinline__ void load_few(const void* base, int64_t at, int left, float (&v)[8])
{
    const bool four = left & 4, two = left & 2, one = left & 1;
    const char* src = static_cast<const char*>(base) + at * (F32 ? 4 : 2);
    words4 q = {};                     // four | two | one, as they come
    words2 h = {};
    uint32_t s = 0;
    constexpr int B = F32 ? 4 : 2;
    if (four) { if (F32) q = *reinterpret_cast<const words4_any*>(src); else { const words2 t = *reinterpret_cast<const words2_any*>(src); q[0] = t[0]; q[1] = t[1]; } }
    if (two)  { if (F32) h = *reinterpret_cast<const words2_any*>(src + (left & 4) * B); else h[0] = *reinterpret_cast<const word_any*>(src + (left & 4) * B); }
    if (one)  { if (F32) s = *reinterpret_cast<const word_any*>(src + (left & 6) * B); else s = *reinterpret_cast<const half_any*>(src + (left & 6) * B); }
    auto low = [](uint32_t w) { return __uint_as_float(F32 ? w : w << 16); };
    auto high = [](uint32_t w, uint32_t next) { return __uint_as_float(F32 ? next : w & 0xFFFF0000u); };
    const float p0 = low(h[0]), p1 = high(h[0], h[1]), s0 = low(s);
    const float t0 = two ? p0 : s0, t1 = p1, t2 = two ? s0 : 0.f;        // what follows the four
    v[0] = four ? low(q[0]) : t0;
    v[1] = four ? high(q[0], q[1]) : t1;
    v[2] = four ? low(F32 ? q[2] : q[1]) : t2;
    v[3] = four ? high(q[1], q[3]) : 0.f;
    v[4] = four ? t0 : 0.f;
    v[5] = four ? t1 : 0.f;
    v[6] = four ? t2 : 0.f;
    v[7] = 0.f;
}

// (VEC: whole vectors on their bytes)
template <bool F32, bool VEC, bool STREAM = false> __device__ __forceinline__ void store8(void* base, int64_t at, int left, const float (&v)[8])
{
    if constexpr (VEC) {
        store_vec<F32, 8, STREAM>(base, at, v);
        return;
    }
    char* dst = static_cast<char*>(base) + at * (F32 ? 4 : 2);
    constexpr int B = F32 ? 4 : 2;
    auto quad = [](char* to, float a, float b, float c, float d) {
        if constexpr (F32) *reinterpret_cast<words4_any*>(to) = (words4){__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d)};
        else               *reinterpret_cast<words2_any*>(to) = (words2){bf16_pair(a, b), bf16_pair(c, d)};
    };
    if (left >= 8) {
        if constexpr (F32) {
            quad(dst, v[0], v[1], v[2], v[3]);
            quad(dst + 16, v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<words4_any*>(dst) = (words4){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
        }
        return;
    }
    const bool four = left & 4, two = left & 2;
    // (a choice between values; between elements it would be one of addresses, and the array would go to memory)
    const float v0 = v[0], v1 = v[1], v2 = v[2], v4 = v[4], v5 = v[5], v6 = v[6];
    const float p0 = four ? v4 : v0, p1 = four ? v5 : v1, last = four ? (two ? v6 : v4) : (two ? v2 : v0);
    if (four) quad(dst, v[0], v[1], v[2], v[3]);
    if (two) {
        if constexpr (F32) *reinterpret_cast<words2_any*>(dst + (left & 4) * B) = (words2){__float_as_uint(p0), __float_as_uint(p1)};
        else               *reinterpret_cast<word_any*>(dst + (left & 4) * B) = bf16_pair(p0, p1);
    }
    if (left & 1) {
        if constexpr (F32) *reinterpret_cast<word_any*>(dst + (left & 6) * B) = __float_as_uint(last);
        else               *reinterpret_cast<half_any*>(dst + (left & 6) * B) = (uint16_t)f32_to_bf16_bits(last);
    }
}

// four values as e4m3 codes, rounded to nearest even; magnitudes up to 464 (exclusive) give at most 448
__device__ __forceinline__ uint32_t e4m3_quad(float a, float b, float c, float d)
{
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// bits of |v|: as integers they order as the magnitudes do, with NaN above infinity, so that a maximum keeps a NaN
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// maximum over the 16 lanes of a row, on every lane of it
__device__ __forceinline__ uint32_t row_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false));   // row_ror:8, 4, 2, 1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, false));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, false));
}

// value / scale with the rounding of a division where nothing underflows: one step from the product with the rounded
// reciprocal, which alone is another number in a quarter of the cases and moves a value near the middle between two codes to
// the wrong one.  (Divisions, ten instructions each, took as long as the memory in cache_store.)  The signs of zeros stay.  By an
// infinite scale, that of a block that holds an infinity, finite values give zeros and the infinity NaN: its d is 0 here,
// because infinity times a quotient of zero is not a number.
struct Divisor { float d, reciprocal; };
__device__ __forceinline__ Divisor divisor(float scale) { return {scale == __builtin_inff() ? 0.f : scale, 1.f / scale}; }
__device__ __forceinline__ float quotient(float v, Divisor by)
{
    const float q = v * by.reciprocal;
    return __builtin_fmaf(-__builtin_fmaf(q, by.d, -v), by.reciprocal, q);
}

// Scale of a block whose largest magnitude has these bits.  At least 2^-126, so that the scale and its reciprocal are
// normal numbers.  (The quotient by 448 is the division's for every magnitude of which it is kept: all 2^31 were compared.)
__device__ __forceinline__ float block_scale(uint32_t top)
{
    if (top == 0) return 1.f;
    if (top >= 0x7F800000u) return __uint_as_float(top);       // infinity, NaN
    return fmaxf(quotient(__uint_as_float(top), {E4M3_MAX, 1.f / E4M3_MAX}), 1.17549435e-38f);
}

// Cosine and sine of position * freq, times gain.  The number of turns is formed and reduced in fp64 (positions reach
// 10^5 radians, where fp32 has no digits left); what is left, in [-1/2, 1/2], loses 2^-25 of a turn as fp32.
__device__ __forceinline__ void turn_of(int position, double freq, float gain, float& cs, float& sn)
{
    const double turns = (double)position * (freq * 0.15915494309189533577);
    const float r = (float)(turns - rint(turns));
    sincospif(2.f * r, &sn, &cs);
    cs *= gain;
    sn *= gain;
}

}  // namespace mla
