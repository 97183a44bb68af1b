// Projection on e4m3 codes with a scale per token and 128 input columns, and per 128 x 128 block of the weights:
//     out[m, n] = sum_b sa[b, m] sw[n / 128, b] sum_{k in b} a[m, k] w[n, k]
// The inner sum runs on the matrix cores, starts from zero and is added to the running sum with the two scales.  The
// weights are the instruction's row operand, so that a lane's outputs belong to one token and take one scale.
//
// Which instruction: v_mfma_f32_16x16x128_f8f6f4 takes the codes as they are, but its adders align the products of eight
// neighbouring k to the largest of them and keep 13 bits below it (measured: 2^16 + 2^2 in one group gives 2^16; across
// groups, and to the accumulator, nothing is lost).  A result of 128 random products is 1.4e-5 off.  Every e4m3
// value is an f16 value, and v_mfma_f32_16x16x32_f16 adds such products without loss, at half the rate.
#include "layer_internal.h"
#include "mfma_tile.h"

namespace mla {
namespace {

typedef __attribute__((ext_vector_type(8))) int i32x8;

typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

// eight codes as f16 (exact)
__device__ __forceinline__ f16x8 widen8(int lo, int hi)
{
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    return (f16x8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// rows of 128 codes -> 16 x 16 sums: lane (g, n) supplies the same 32 columns of row n of either operand, in the same
// order (which 32 does not matter), and holds results (row 4 g + i of w, row n of a)
__device__ __forceinline__ f32x4 block_products(const i32x8& w, const i32x8& a)
{
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8(w[2 * i], w[2 * i + 1]), widen8(a[2 * i], a[2 * i + 1]), s, 0, 0, 0);
    return s;
}

// 32 codes of a row; columns at and past K (a multiple of 16) are zeros
__device__ __forceinline__ i32x8 codes32(const uint8_t* row, int k, int K)
{
    u32x4 lo = {0u, 0u, 0u, 0u}, hi = lo;
    if (k < K) lo = *reinterpret_cast<const u32x4*>(row + k);
    if (k + 16 < K) hi = *reinterpret_cast<const u32x4*>(row + k + 16);
    return __builtin_bit_cast(i32x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// 64 tokens x 64 outputs per workgroup, 16 outputs per wavefront, operands straight from memory.
template <bool F32>
__global__ __launch_bounds__(256) void gemm_fp8_kernel(GemmFp8Params p)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
    const int m0 = blockIdx.x * 64, n0 = blockIdx.y * 64 + wave * 16;
    if (n0 >= p.N) return;
    const int blocks = (p.K + QBLOCK - 1) / QBLOCK;
    const uint8_t* w = p.w + (int64_t)min(n0 + n, p.N - 1) * p.K;
    const float* ws = p.w_scales + (int64_t)(n0 / QBLOCK) * blocks;
    f32x4 acc[4] = {};
    for (int b = 0; b < blocks; ++b) {
        const int k = b * QBLOCK + g * 32;
        const i32x8 wv = codes32(w, k, p.K);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = min(m0 + i * 16 + n, p.M - 1);
            const f32x4 s = block_products(wv, codes32(p.a + (int64_t)m * p.K, k, p.K));
            const float scale = p.a_scales[(int64_t)b * p.M + m] * ws[b];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] += s[j] * scale;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + i * 16 + n;
        if (m >= p.M) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = n0 + 4 * g + j;
            if (c >= p.N) continue;
            if (F32) static_cast<float*>(p.out)[(int64_t)m * p.N + c] = acc[i][j];
            else     static_cast<uint16_t*>(p.out)[(int64_t)m * p.N + c] = (uint16_t)f32_to_bf16_bits(acc[i][j]);
        }
    }
}

}  // namespace

size_t gemm_fp8_workspace(int, int, int) { return 0; }

hipError_t launch_gemm_fp8(const GemmFp8Params& p, mla_dtype out, bool, hipStream_t s)
{
    const dim3 grid((unsigned)((p.M + 63) / 64), (unsigned)((p.N + 63) / 64)), block(256);
    if (out == MLA_F32) gemm_fp8_kernel<true><<<grid, block, 0, s>>>(p);
    else                gemm_fp8_kernel<false><<<grid, block, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace mla
