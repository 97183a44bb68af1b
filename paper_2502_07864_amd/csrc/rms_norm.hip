// RMS norm with the residual's addition before it and e4m3 codes after it; codes of rows and of weights.
//     s = x (+ residual),  y = s / sqrt(mean(s^2) + eps) * weight,  per 128 columns: scale = max|y| / 448, code = e4m3(y / scale)
// One pass over memory: a row stays in registers between the sum of its squares and its output.  A thread holds whole
// vectors of eight columns, so that a block of 128 columns is one row of 16 lanes and its maximum takes four
// row rotations.
#include "layer_internal.h"

namespace mla {
namespace {

// TPR threads per row, NV vectors of eight columns per thread (8 TPR NV >= D).
template <bool F32, int TPR, int NV, bool VEC, bool NORM>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_norm_kernel(NormParams p)
{
    constexpr int THREADS = TPR < 256 ? 256 : TPR;
    const int tid = threadIdx.x, t = tid % TPR;
    const int row = blockIdx.x * (THREADS / TPR) + tid / TPR;
    if (TPR <= 64 && row >= p.T) return;                 // (wider rows are a workgroup each: the grid is T)

    float v[NV][8];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) v[i][k] = 0.f;
        if (c < p.D) {
            load8<F32, VEC>(p.x, (int64_t)row * p.x_pitch + c, p.D - c, v[i]);
            if (NORM && p.residual) {
                float r[8];
                load8<F32, VEC>(p.residual, (int64_t)row * p.D + c, p.D - c, r);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[i][k] += r[k];
                store8<F32, VEC>(p.residual_out, (int64_t)row * p.D + c, p.D - c, v[i]);
            }
        }
        if (NORM) {
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += v[i][k] * v[i][k];
        }
    }
    if (NORM) {
        sum = wave_sum(sum);
        if constexpr (TPR > 64) {
            __shared__ float part[TPR / 64];
            if (t % 64 == 0) part[t / 64] = sum;
            __syncthreads();
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < TPR / 64; ++i) sum += part[i];
        }
        const float inv = 1.f / sqrtf(sum / (float)p.D + p.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * 8;
            float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
            if (p.weight && c < p.D) load8<F32, VEC>(p.weight, c, p.D - c, w);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[i][k] = v[i][k] * inv * w[k];
            if (p.y && c < p.D) store8<F32, VEC>(p.y, (int64_t)row * p.D + c, p.D - c, v[i]);
        }
    }
    if (!p.codes) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * 8;
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = max(top, magnitude(v[i][k]));
        const float scale = block_scale(row_max(top)), inv = 1.f / scale;      // (columns past D are zeros)
        if (c >= p.D) continue;
        if (c % QBLOCK == 0) p.scales[(int64_t)(c / QBLOCK) * p.T + row] = scale;
        const uint32_t lo = e4m3_quad(v[i][0] * inv, v[i][1] * inv, v[i][2] * inv, v[i][3] * inv);
        const uint32_t hi = e4m3_quad(v[i][4] * inv, v[i][5] * inv, v[i][6] * inv, v[i][7] * inv);
        uint8_t* dst = p.codes + (int64_t)row * p.D + c;
        if constexpr (VEC) {
            *reinterpret_cast<words2*>(dst) = (words2){lo, hi};
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < p.D) dst[k] = (uint8_t)((k < 4 ? lo : hi) >> (8 * (k & 3)));
        }
    }
}

// One workgroup per 128 x 128 block of a weight matrix (once per matrix: nothing here is hurried).
template <bool F32>
__global__ __launch_bounds__(256) void quantize_weights_kernel(const void* w, uint8_t* codes, float* scales, int N, int K)
{
    __shared__ uint32_t part[4];
    const int k0 = blockIdx.x * QBLOCK, n0 = blockIdx.y * QBLOCK, tid = threadIdx.x;
    const int rows = min(QBLOCK, N - n0), cols = min(QBLOCK, K - k0);
    auto at = [&](int r, int c) {
        const int64_t i = (int64_t)(n0 + r) * K + k0 + c;
        return F32 ? static_cast<const float*>(w)[i] : bf16_bits_to_f32(static_cast<const uint16_t*>(w)[i]);
    };
    const int c = tid % QBLOCK;
    uint32_t top = 0;
    if (c < cols)
        for (int r = tid / QBLOCK; r < rows; r += 256 / QBLOCK) top = max(top, magnitude(at(r, c)));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if (tid % 64 == 0) part[tid / 64] = top;
    __syncthreads();
    const float scale = block_scale(max(max(part[0], part[1]), max(part[2], part[3]))), inv = 1.f / scale;
    if (tid == 0) scales[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = scale;
    if (c < cols)
        for (int r = tid / QBLOCK; r < rows; r += 256 / QBLOCK)
            codes[(int64_t)(n0 + r) * K + k0 + c] = (uint8_t)e4m3_quad(at(r, c) * inv, 0.f, 0.f, 0.f);
}

template <bool F32, int TPR, int NV, bool NORM> void launch_rows(const NormParams& p, bool vec, hipStream_t s)
{
    constexpr int THREADS = TPR < 256 ? 256 : TPR, ROWS = THREADS / TPR;
    const dim3 grid((unsigned)((p.T + ROWS - 1) / ROWS)), block(THREADS);
    if (vec) rms_norm_kernel<F32, TPR, NV, true, NORM><<<grid, block, 0, s>>>(p);
    else     rms_norm_kernel<F32, TPR, NV, false, NORM><<<grid, block, 0, s>>>(p);
}

template <bool F32, bool NORM> void launch_dim(const NormParams& p, bool vec, hipStream_t s)
{
    if      (p.D <= 2048)  launch_rows<F32, 256, 1, NORM>(p, vec, s);
    else if (p.D <= 4096)  launch_rows<F32, 256, 2, NORM>(p, vec, s);
    else if (p.D <= 8192)  launch_rows<F32, 256, 4, NORM>(p, vec, s);
    else if (p.D <= 16384) launch_rows<F32, 256, 8, NORM>(p, vec, s);
    else                   launch_rows<F32, 256, 16, NORM>(p, vec, s);
}

bool on(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

}  // namespace

hipError_t launch_rms_norm(const NormParams& p, bool norm, mla_dtype io, hipStream_t s)
{
    // 16-byte accesses: whole vectors, and every row of every tensor on 16 bytes (codes on 8)
    const int per16 = io == MLA_F32 ? 4 : 8;
    const bool vec = p.D % 8 == 0 && p.x_pitch % per16 == 0 && on(p.x, 16) && on(p.residual, 16) && on(p.residual_out, 16) &&
                     on(p.weight, 16) && on(p.y, 16) && on(p.codes, 8);
    if (io == MLA_F32) norm ? launch_dim<true, true>(p, vec, s) : launch_dim<true, false>(p, vec, s);
    else               norm ? launch_dim<false, true>(p, vec, s) : launch_dim<false, false>(p, vec, s);
    return hipGetLastError();
}

hipError_t launch_quantize_weights(const void* w, uint8_t* codes, float* scales, int N, int K, mla_dtype io, hipStream_t s)
{
    const dim3 grid((unsigned)((K + QBLOCK - 1) / QBLOCK), (unsigned)((N + QBLOCK - 1) / QBLOCK)), block(256);
    if (io == MLA_F32) quantize_weights_kernel<true><<<grid, block, 0, s>>>(w, codes, scales, N, K);
    else               quantize_weights_kernel<false><<<grid, block, 0, s>>>(w, codes, scales, N, K);
    return hipGetLastError();
}

}  // namespace mla
