// RMS norm with the residual's addition before it and e4m3 codes after it; codes of rows and of weights.
//     s = x (+ residual),  y = s / sqrt(mean(s^2) + eps) * weight,  per 128 columns: scale = max|y| / 448, code = e4m3(y / scale)
// One pass over memory: a row stays in registers between the sum of its squares and its output.  A thread holds whole
// vectors of eight columns, so that a block of 128 columns is one row of 16 lanes and its maximum takes four
// row rotations.
#include "layer_internal.h"

namespace mla {
namespace {

// TPR threads per row, NV vectors of eight columns per thread (8 TPR NV >= D).
// Memory bound: 32768 x 4096 bf16 with residual and codes moves 940 MB in 160 us (5.9 TB/s).  Wide rows take 512 threads
// with one vector each: with 256, 128, 64 threads and 2, 4, 8 vectors it was 4, 9, 25 % slower, and 3.6, 5.4, 8.5 us
// against 3.1 for 64 tokens, whose time is the launch and two dependent steps (load, sum).
// Rows on no 16 bytes, or of a width that is no multiple of 8 (VEC = false): 32768 x 4095 in 232 us, 6517 x 3443 in 38 (with one
// value per access 574 and 94).
template <bool F32, int TPR, int NV, bool VEC, bool NORM, bool STREAM>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_norm_kernel(NormParams p)
{
    constexpr int THREADS = TPR < 256 ? 256 : TPR, WAVES = TPR / 64;       // wavefronts per row
    __shared__ float part[THREADS / 64];
    const int tid = threadIdx.x, t = tid % TPR;
    const int64_t mine = (int64_t)blockIdx.x * (THREADS / TPR) + tid / TPR;
    const bool live = mine < p.T;                                          // (the others repeat the last row and store nothing)
    const int64_t row = live ? mine : p.T - 1;

    float v[NV][8], w[NV][8];
    float sum = 0.f;
    // Everything is asked for before the first wait; threads past the end, and the one whose vector is cut short, take the
    // row's last eight values (the latter gets its own below).
    RawVec<F32, 8> x_raw[NV], r_raw[NV], w_raw[NV];
    if (VEC || p.D >= 8) {
        auto ask = [&](const void* base, int64_t at, auto& raw) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t from = at + min((i * TPR + t) * 8, p.D - 8);
                if constexpr (VEC) raw[i] = raw_vec<F32, 8>(base, from);
                else               raw[i] = raw8_any<F32>(base, from);
            }
        };
        ask(p.x, row * p.x_pitch, x_raw);
        if (NORM && p.residual) ask(p.residual, row * p.D, r_raw);
        if (NORM && p.weight) ask(p.weight, 0, w_raw);
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) { v[i][k] = 0.f; w[i][k] = 1.f; }
        const bool whole = VEC ? c < p.D : c + 8 <= p.D;
        float r[8];
        if (whole) {
            values_of<F32, 8>(x_raw[i], v[i]);
            if (NORM && p.residual) values_of<F32, 8>(r_raw[i], r);
            if (NORM && p.weight) values_of<F32, 8>(w_raw[i], w[i]);
        } else if (!VEC && c < p.D) {
            load_few<F32>(p.x, row * p.x_pitch + c, p.D - c, v[i]);
            if (NORM && p.residual) load_few<F32>(p.residual, row * p.D + c, p.D - c, r);
            if (NORM && p.weight) load_few<F32>(p.weight, c, p.D - c, w[i]);
        }
        if (NORM && p.residual && c < p.D) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[i][k] += r[k];
        }
        if (NORM) {
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += v[i][k] * v[i][k];
        }
    }
    if (NORM) {
        if (p.residual_out && live) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * TPR + t) * 8;
                if (c < p.D) store8<F32, VEC, STREAM>(p.residual_out, row * p.D + c, p.D - c, v[i]);
            }
        }
        sum = wave_sum(sum);
        if constexpr (WAVES > 1) {
            if (tid % 64 == 0) part[tid / 64] = sum;
            __syncthreads();
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) sum += part[tid / TPR * WAVES + i];
        }
        const float inv = 1.f / sqrtf(sum / (float)p.D + p.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * 8;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[i][k] = v[i][k] * inv * w[i][k];
            if (p.y && c < p.D && live) store8<F32, VEC, STREAM>(p.y, row * p.D + c, p.D - c, v[i]);
        }
    }
    if (!p.codes) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * 8;
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = max(top, c + k < p.D ? magnitude(v[i][k]) : 0u);
        const float scale = block_scale(row_max(top));
        const Divisor by = divisor(scale);
        auto q = [&](int k) { return quotient(v[i][k], by); };
        if (c >= p.D || !live) continue;
        if (c % QBLOCK == 0) p.scales[(int64_t)(c / QBLOCK) * p.T + row] = scale;
        const uint32_t lo = e4m3_quad(q(0), q(1), q(2), q(3));
        const uint32_t hi = e4m3_quad(q(4), q(5), q(6), q(7));
        uint8_t* dst = p.codes + row * p.D + c;
        if constexpr (VEC) {
            put_words<STREAM>(dst, (words2){lo, hi});
        } else {
            const int left = p.D - c;
            const uint64_t all = (uint64_t)hi << 32 | lo;
            if (left >= 8) {
                *reinterpret_cast<words2_any*>(dst) = (words2){lo, hi};
            } else {
                if (left & 4) *reinterpret_cast<word_any*>(dst) = lo;
                if (left & 2) *reinterpret_cast<half_any*>(dst + (left & 4)) = (uint16_t)(all >> 8 * (left & 4));
                if (left & 1) dst[left & 6] = (uint8_t)(all >> 8 * (left & 6));
            }
        }
    }
}

// One workgroup per 128 x 128 block of a weight matrix, a value per access and every value read twice (once per matrix: nothing here
// is hurried; 6144 x 4096 from bf16 45 us, 1.7 TB/s, from fp32 48 us; 576 x 4096 18 us).
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
    const float scale = block_scale(max(max(part[0], part[1]), max(part[2], part[3])));
    const Divisor by = divisor(scale);
    if (tid == 0) scales[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = scale;
    if (c < cols)
        for (int r = tid / QBLOCK; r < rows; r += 256 / QBLOCK)
            codes[(int64_t)(n0 + r) * K + k0 + c] = (uint8_t)e4m3_quad(quotient(at(r, c), by), 0.f, 0.f, 0.f);
}

template <bool F32, int TPR, int NV, bool NORM> void launch_rows(const NormParams& p, bool vec, bool stream, hipStream_t s)
{
    constexpr int THREADS = TPR < 256 ? 256 : TPR, ROWS = THREADS / TPR;
    const dim3 grid((unsigned)((p.T + ROWS - 1) / ROWS)), block(THREADS);
    if (!vec)        rms_norm_kernel<F32, TPR, NV, false, NORM, false><<<grid, block, 0, s>>>(p);
    else if (stream) rms_norm_kernel<F32, TPR, NV, true, NORM, true><<<grid, block, 0, s>>>(p);
    else             rms_norm_kernel<F32, TPR, NV, true, NORM, false><<<grid, block, 0, s>>>(p);
}

template <bool F32, bool NORM> void launch_dim(const NormParams& p, bool vec, bool stream, hipStream_t s)
{
    if      (p.D <= 512)   launch_rows<F32, 64, 1, NORM>(p, vec, stream, s);
    else if (p.D <= 1024)  launch_rows<F32, 128, 1, NORM>(p, vec, stream, s);
    else if (p.D <= 2048)  launch_rows<F32, 256, 1, NORM>(p, vec, stream, s);
    else if (p.D <= 4096)  launch_rows<F32, 512, 1, NORM>(p, vec, stream, s);
    else if (p.D <= 8192)  launch_rows<F32, 512, 2, NORM>(p, vec, stream, s);
    else if (p.D <= 16384) launch_rows<F32, 512, 4, NORM>(p, vec, stream, s);
    else                   launch_rows<F32, 512, 8, NORM>(p, vec, stream, s);
}

bool on(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

}  // namespace

hipError_t launch_rms_norm(const NormParams& p, bool norm, mla_dtype io, hipStream_t s)
{
    // 16-byte accesses: whole vectors, and every row of every tensor on 16 bytes (codes on 8)
    const int per16 = io == MLA_F32 ? 4 : 8;
    const bool vec = p.D % 8 == 0 && p.x_pitch % per16 == 0 && on(p.x, 16) && on(p.residual, 16) && on(p.residual_out, 16) &&
                     on(p.weight, 16) && on(p.y, 16) && on(p.codes, 8);
    const int wide = (p.residual_out ? 1 : 0) + (p.y ? 1 : 0);
    const bool stream = (int64_t)p.T * p.D * (wide * (io == MLA_F32 ? 4 : 2) + (p.codes ? 1 : 0)) > STREAM_BYTES;
    if (io == MLA_F32) norm ? launch_dim<true, true>(p, vec, stream, s) : launch_dim<true, false>(p, vec, stream, s);
    else               norm ? launch_dim<false, true>(p, vec, stream, s) : launch_dim<false, false>(p, vec, stream, s);
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
