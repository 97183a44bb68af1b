// C-ABI entry points of the operators around the attention: validation on the host, then launches.
#include "layer_internal.h"

#include <cmath>

using namespace mla;

namespace {

bool io_ok(mla_dtype t) { return t == MLA_F32 || t == MLA_BF16; }
int status_of(hipError_t e) { return e == hipSuccess ? MLA_OK : MLA_ERR_HIP; }
bool layout_ok(int l) { return l == MLA_ROPE_INTERLEAVED || l == MLA_ROPE_HALF; }

// A workgroup of up to 512 threads per row: the grid's threads are counted in 32 bits
constexpr int MAX_ROWS = (1 << 23) - 1;

int rows_call(const NormParams& p, bool norm, mla_dtype io, void* stream)
{
    if (p.T <= 0 || p.D <= 0 || p.x_pitch < p.D || !(p.eps >= 0.f)) return MLA_ERR_SHAPE;
    if (!io_ok(io) || p.D > 32768 || p.T > MAX_ROWS) return MLA_ERR_UNSUPPORTED;
    return status_of(launch_rms_norm(p, norm, io, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" int mla_rms_norm(const void* x, const void* residual, const void* weight, void* residual_out, void* y,
                            uint8_t* codes, float* scales, int T, int D, int64_t x_pitch, float eps, mla_dtype io_dtype,
                            void* hip_stream)
{
    if (!x || (!y && !codes) || !codes != !scales || !residual != !residual_out) return MLA_ERR_NULL;
    return rows_call(NormParams{x, residual, weight, residual_out, y, codes, scales, T, D, x_pitch, eps}, true, io_dtype, hip_stream);
}

extern "C" int mla_quantize_rows(const void* x, uint8_t* codes, float* scales, int T, int D, int64_t x_pitch,
                                 mla_dtype io_dtype, void* hip_stream)
{
    if (!x || !codes || !scales) return MLA_ERR_NULL;
    return rows_call(NormParams{x, nullptr, nullptr, nullptr, nullptr, codes, scales, T, D, x_pitch, 0.f}, false, io_dtype, hip_stream);
}

extern "C" int mla_quantize_weights(const void* w, uint8_t* codes, float* scales, int N, int K, mla_dtype io_dtype, void* hip_stream)
{
    if (!w || !codes || !scales) return MLA_ERR_NULL;
    if (N <= 0 || K <= 0) return MLA_ERR_SHAPE;
    if (!io_ok(io_dtype) || N > 65535 * QBLOCK) return MLA_ERR_UNSUPPORTED;
    return status_of(launch_quantize_weights(w, codes, scales, N, K, io_dtype, static_cast<hipStream_t>(hip_stream)));
}

extern "C" size_t mla_gemm_fp8_workspace_bytes(int M, int N, int K)
{
    return M > 0 && N > 0 && K > 0 ? gemm_fp8_workspace(M, N, K) : 0;
}

extern "C" int mla_gemm_fp8(const uint8_t* a, const float* a_scales, const uint8_t* w, const float* w_scales, void* out,
                            void* workspace, size_t workspace_bytes, int M, int N, int K, mla_dtype out_dtype, unsigned flags,
                            void* hip_stream)
{
    if (!a || !a_scales || !w || !w_scales || !out) return MLA_ERR_NULL;
    if (M <= 0 || N <= 0 || K <= 0) return MLA_ERR_SHAPE;
    if (!io_ok(out_dtype) || K % 16 || reinterpret_cast<uintptr_t>(a) % 16 || reinterpret_cast<uintptr_t>(w) % 16 ||
        K > 1 << 23 || (flags & ~(unsigned)MLA_GEMM_FAST_SUMS) || !gemm_fp8_supported(M, N, K))
        return MLA_ERR_UNSUPPORTED;
    const size_t need = gemm_fp8_workspace(M, N, K);
    if (need && (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 16)) return MLA_ERR_WORKSPACE;
    const GemmFp8Params p{a, a_scales, w, w_scales, out, static_cast<float*>(workspace), M, N, K, M};
    return status_of(launch_gemm_fp8(p, out_dtype, (flags & MLA_GEMM_FAST_SUMS) != 0, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int mla_rope_frequencies(double* freq, float* gain, int d_rope, double base, int kind, double factor, int original,
                                    double beta_fast, double beta_slow)
{
    if (!freq || !gain) return MLA_ERR_NULL;
    if (d_rope < 2 || d_rope % 2 || !(base > 1.0) || !std::isfinite(base)) return MLA_ERR_SHAPE;
    if (kind != MLA_ROPE_PLAIN && kind != MLA_ROPE_LINEAR && kind != MLA_ROPE_YARN) return MLA_ERR_UNSUPPORTED;
    if (kind != MLA_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return MLA_ERR_SHAPE;
    const int pairs = d_rope / 2;
    *gain = 1.f;
    double low = 0.0, high = 0.0;
    if (kind == MLA_ROPE_YARN) {
        if (original < 1 || !(beta_slow > 0.0) || !(beta_fast >= beta_slow) || !std::isfinite(beta_fast)) return MLA_ERR_SHAPE;
        // pair (a real number) that turns `turns` times within the original length
        auto pair_at = [&](double turns) { return d_rope * std::log(original / (turns * 2.0 * M_PI)) / (2.0 * std::log(base)); };
        low = std::fmax(std::floor(pair_at(beta_fast)), 0.0);
        high = std::ceil(pair_at(beta_slow));      // (beyond the last pair where even that turns more often than beta_slow)
        *gain = (float)(0.1 * std::log(factor) + 1.0);
    }
    for (int i = 0; i < pairs; ++i) {
        const double theta = std::pow(base, -2.0 * i / d_rope);
        if (kind == MLA_ROPE_PLAIN) {
            freq[i] = theta;
        } else if (kind == MLA_ROPE_LINEAR) {
            freq[i] = theta / factor;
        } else {
            const double r = i >= high ? 1.0 : std::fmax((i - low) / (high - low), 0.0);
            freq[i] = theta * (1.0 - r) + theta / factor * r;
        }
    }
    return MLA_OK;
}

extern "C" int mla_rope_queries(const void* q, const int32_t* positions, const double* freq, void* q_nope, void* q_rope,
                                int T, int H, int d_nope, int d_rope, int64_t q_pitch, float gain, int layout, mla_dtype io_dtype,
                                void* hip_stream)
{
    if (!q || !positions || !freq || !q_rope || (d_nope > 0 && !q_nope)) return MLA_ERR_NULL;
    if (T <= 0 || H <= 0 || d_nope < 0 || d_rope <= 0 || d_rope % 2) return MLA_ERR_SHAPE;
    const int64_t width = (int64_t)H * ((int64_t)d_nope + d_rope);
    if (q_pitch < width || !(gain == gain)) return MLA_ERR_SHAPE;
    if (!io_ok(io_dtype) || !layout_ok(layout) || d_rope > 256 || width > 1 << 30 || T > MAX_ROWS) return MLA_ERR_UNSUPPORTED;
    const RopeParams p{q, positions, freq, q_nope, q_rope, T, H, d_nope, d_rope, q_pitch, gain};
    if (!rope_queries_supported(p, layout, io_dtype)) return MLA_ERR_UNSUPPORTED;
    return status_of(launch_rope_queries(p, layout, io_dtype, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int mla_cache_store_at(const void* rows, const int32_t* positions, const int32_t* slots, const double* freq, const void* norm_weight,
                                  void* kv_cache, float* kv_scale, const int32_t* page_table, int B, int new_tokens, int d_c,
                                  int d_rope, int64_t row_pitch, int page_size, int num_pages, int max_pages_per_seq, float gain,
                                  int layout, float eps, mla_dtype io_dtype, mla_dtype cache_dtype, void* hip_stream)
{
    if (!rows || !positions || !slots || !kv_cache || !page_table || (d_rope > 0 && !freq)) return MLA_ERR_NULL;
    if (B <= 0 || new_tokens <= 0 || d_c <= 0 || d_rope < 0 || d_rope % 2 || page_size <= 0 || num_pages <= 0 ||
        max_pages_per_seq <= 0 || row_pitch < (int64_t)d_c + d_rope || !(gain == gain) || !(eps >= 0.f))
        return MLA_ERR_SHAPE;
    if ((int64_t)max_pages_per_seq * page_size > 0x7FFFFFFF ) return MLA_ERR_SHAPE;
    if (!io_ok(io_dtype) || !layout_ok(layout) || d_rope > 256 || d_c > 1024 || d_c + d_rope > 1024 || (int64_t)B * new_tokens > MAX_ROWS) return MLA_ERR_UNSUPPORTED;
    if (cache_dtype != MLA_F32 && cache_dtype != MLA_BF16 && cache_dtype != MLA_FP8_E4M3) return MLA_ERR_UNSUPPORTED;
    if (cache_dtype == MLA_FP8_E4M3 && !kv_scale) return MLA_ERR_NULL;
    if (cache_dtype != MLA_FP8_E4M3 && kv_scale) return MLA_ERR_SHAPE;
    const StoreParams p{rows, positions, slots, freq, norm_weight, kv_cache, kv_scale, page_table, B * new_tokens, new_tokens, d_c, d_rope,
                        page_size, num_pages, max_pages_per_seq, row_pitch, gain, eps};
    return status_of(launch_cache_store(p, layout, io_dtype, cache_dtype, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int mla_cache_store(const void* rows, const int32_t* positions, const double* freq, const void* norm_weight,
                               void* kv_cache, float* kv_scale, const int32_t* page_table, int B, int new_tokens, int d_c,
                               int d_rope, int64_t row_pitch, int page_size, int num_pages, int max_pages_per_seq, float gain,
                               int layout, float eps, mla_dtype io_dtype, mla_dtype cache_dtype, void* hip_stream)
{
    return mla_cache_store_at(rows, positions, positions, freq, norm_weight, kv_cache, kv_scale, page_table, B, new_tokens, d_c, d_rope,
                              row_pitch, page_size, num_pages, max_pages_per_seq, gain, layout, eps, io_dtype, cache_dtype, hip_stream);
}

extern "C" int mla_cache_move(void* kv_cache, float* kv_scale, const int32_t* page_table, const int32_t* src, const int32_t* dst, int B,
                              int moves, int row_bytes, int page_size, int num_pages, int max_pages_per_seq, void* hip_stream)
{
    if (!kv_cache || !page_table || !src || !dst) return MLA_ERR_NULL;
    if (B <= 0 || moves <= 0 || row_bytes <= 0 || page_size <= 0 || num_pages <= 0 || max_pages_per_seq <= 0) return MLA_ERR_SHAPE;
    if ((int64_t)max_pages_per_seq * page_size > 0x7FFFFFFF) return MLA_ERR_SHAPE;
    if (moves > MAX_MOVES || B > 65535 || row_bytes > 4096) return MLA_ERR_UNSUPPORTED;
    const MoveParams p{kv_cache, kv_scale, page_table, src, dst, B, moves, row_bytes, page_size, num_pages, max_pages_per_seq};
    return status_of(launch_cache_move(p, static_cast<hipStream_t>(hip_stream)));
}
