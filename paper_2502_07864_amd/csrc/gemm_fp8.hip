// Projection on e4m3 codes with a scale per token and 128 input columns, and per 128 x 128 block of the weights:
//     out[m, n] = sum_b sa[b, m] sw[n / 128, b] sum_{k in b} a[m, k] w[n, k]
// The inner sum runs on the matrix cores, starts from zero and is added to the running sum with the two scales.  The
// weights are the instruction's row operand, so that a lane's outputs belong to one token and take one scale.
//
// Which instruction: the f8f6f4 ones take the codes as they are, but their adders align the products of eight
// neighbouring k to the largest of them and keep 13 bits below it (measured: 2^16 + 2^2 in one group gives 2^16; across
// groups, and to the accumulator, nothing is lost).  A result of 128 random products is 1.4e-5 off.  Every e4m3
// value is an f16 value, and the f16 instructions add such products without loss, at half the rate.  So: f16,
// unless the caller allows the other (MLA_GEMM_FAST_SUMS), and f16 all the same where 16 tokens and fewer wait for memory anyway
// (the first kernel).
//
// The columns of a block may go into the operands in any order that is the same for both: a lane takes 16-byte pieces
// that suit the loads.
#include "layer_internal.h"
#include "mfma_tile.h"

#include <algorithm>
#include <type_traits>

namespace mla {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;

// eight codes as f16 (exact)
__device__ __forceinline__ f16x8 widen8(int lo, int hi)
{
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
    const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    return (f16x8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// c + 32 x 32 sums over 64 columns: lane (h, n) supplies 32 columns of row n of either operand and holds results (row
// 8 r + 4 h + i of w, row n of a); on the codes (FAST) or on their f16 values
template <bool FAST> __device__ __forceinline__ f32x16 products(const i32x8& w, const i32x8& a, const f32x16& c)
{
    if constexpr (FAST) {
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, a, c, 0, 0, 0, 0, 0, 0);
    } else {
        f32x16 s = c;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(widen8(w[2 * i], w[2 * i + 1]), widen8(a[2 * i], a[2 * i + 1]), s, 0, 0, 0);
        return s;
    }
}

// the same with the f16 values at hand (32 columns a lane)
struct Wide { f16x8 h[4]; };
__device__ __forceinline__ Wide widen32(const i32x8& a)
{
    return Wide{{widen8(a[0], a[1]), widen8(a[2], a[3]), widen8(a[4], a[5]), widen8(a[6], a[7])}};
}
__device__ __forceinline__ f32x16 products(const Wide& w, const Wide& a, const f32x16& c)
{
    f32x16 s = c;
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(w.h[i], a.h[i], s, 0, 0, 0);
    return s;
}

// Which tile a workgroup takes.  Workgroups whose ids are equal mod 8 run on one XCD, whose L2 its tiles' operands pass
// through: the XCDs share out the tiles as `across` x 8 / `across` rectangles of rows x columns tiles, as square as they go.
// (Tiles in a row instead, all tokens of some outputs on an XCD: 2000 x 320 x 7168 in tiles of 64 x 32 28.7 us, so 20.0, in
// tiles of 64 x 64 16.7 and 14.3; no difference where the tiles are few.)  Where rectangles would take one more round of an
// XCD's 32 CUs, the tiles are in a row all the same: `columns` an XCD (log_across < 0), rows = the tiles down the tokens.
struct Layout {
    int log_across, rows, columns;
    float inv_rows;
    // false, or m and n past the tiles: nothing to do
    __device__ __forceinline__ bool at(int id, int& m, int& n) const
    {
        const int x = id & 7, s = id >> 3;
        if (log_across < 0) {
            const int lin = x * columns + s;
            n = lin / rows;
            m = lin - n * rows;
            return s < columns;
        }
        const int column = __builtin_amdgcn_readfirstlane((int)(((float)s + 0.5f) * inv_rows));      // s / rows (s < 2^21)
        m = (x & ((1 << log_across) - 1)) * rows + s - column * rows;
        n = (x >> log_across) * columns + column;
        return column < columns;
    }
    int workgroups() const { return 8 * columns * (log_across < 0 ? 1 : rows); }
};

// workgroup barrier over which the compiler moves no access to memory (waits are placed by hand)
__device__ __forceinline__ void barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <bool F32> __device__ __forceinline__ void put(void* out, int64_t at, float v)
{
    if (F32) static_cast<float*>(out)[at] = v;
    else     static_cast<uint16_t*>(out)[at] = (uint16_t)f32_to_bf16_bits(v);
}

// ---------------------------------------------------------------- few tokens

// A workgroup takes 16 outputs of up to 16 tokens over the whole depth, its wavefronts share out the blocks: what
// bounds it is reading the weights once, and with every block of a wavefront on its way at once that is one round trip.
// The partial sums meet in LDS and are added in the wavefronts' order.  One token by 3584 x 3584: 4.5 us, 2.9 TB/s (13 MB; a
// launch of nothing takes 1.6); 16 tokens by 576 x 4096: 5.6.
template <int WAVES, int U, bool F32>
__global__ __launch_bounds__(WAVES * 64) void gemm_rows_kernel(GemmFp8Params p)
{
    __shared__ __attribute__((aligned(16))) float red[WAVES][256];
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = blockIdx.x * 16;
    const int blocks = (p.K + QBLOCK - 1) / QBLOCK;
    const uint8_t* w = p.w + (int64_t)min(n0 + n, p.N - 1) * p.K + 16 * g;
    const float* ws = p.w_scales + (int64_t)(n0 / QBLOCK) * blocks;
    const uint8_t* a = p.a + (int64_t)min(n, p.M - 1) * p.K + 16 * g;
    const float* as = p.a_scales + min(n, p.M - 1);
    f32x4 acc = {};
    const u32x4 zero = {0u, 0u, 0u, 0u};
    for (int b0 = wave; b0 < blocks; b0 += WAVES * U) {
        u32x4 wv[U][2], av[U][2];
        float f[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = b0 + u * WAVES, k = b * QBLOCK;
#pragma unroll
            for (int i = 0; i < 2; ++i) {              // the pieces at columns 16 g and 64 + 16 g
                const bool in = k + 64 * i + 16 * g < p.K;
                wv[u][i] = zero;
                if (in) wv[u][i] = *reinterpret_cast<const u32x4*>(w + k + 64 * i);
                av[u][i] = zero;
                if (in) av[u][i] = *reinterpret_cast<const u32x4*>(a + k + 64 * i);
            }
            // (a block past the end is zeros, but its scale need not be finite)
            f[u] = b < blocks ? ws[b] * as[(int64_t)b * p.scale_pitch] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            f16x8 ah[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) ah[q] = widen8((int)av[u][q >> 1][2 * (q & 1)], (int)av[u][q >> 1][2 * (q & 1) + 1]);
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < 4; ++q)
                s = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8((int)wv[u][q >> 1][2 * (q & 1)], (int)wv[u][q >> 1][2 * (q & 1) + 1]), ah[q], s, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] += s[j] * f[u];
        }
    }
    *reinterpret_cast<f32x4*>(&red[wave][n * 16 + 4 * g]) = acc;
    __syncthreads();
    if (tid < 256) {
        const int m = tid >> 4, c = n0 + (tid & 15);
        float v = 0.f;
#pragma unroll
        for (int q = 0; q < WAVES; ++q) v += red[q][tid];
        if (m < p.M && c < p.N) put<F32>(p.out, (int64_t)m * p.N + c, v);
    }
}

// ---------------------------------------------------------------- many tokens

__device__ __attribute__((aligned(16))) const uint32_t zeros16[4] = {0u, 0u, 0u, 0u};

// A workgroup of eight wavefronts, WN of them abreast, computes 32 NI WN outputs of 32 MT (8 / WN) tokens, a wavefront 32 NI
// outputs of 32 MT tokens: 256 tokens by 256 outputs, 64 x 128 a wavefront, 256 by 128 (64 x 64) or 128 by 128 (32 x 64).
// 128 tokens by 256 outputs take as long as 256 by 128 at 6144 outputs, and at few 5 - 40 % longer: 25000 x 576 x 4096 80 us,
// these 61.  128 by 128 fill the CUs sooner: 512 x 6144 x 4096 22.7 us with 256 x 128, 18.0 with these; 1024 x 3584 x 3584 21.0
// and 17.5.  The codes of a block travel by direct-to-LDS loads, `STAGES` blocks deep; 16-byte piece c of a row lies at position
// c ^ (row >> 1 & 7) of its 128 bytes, so that the operand reads (32 rows, one piece each half) are free of bank conflicts.
//
// A step is one block: NI MT units of 32 outputs x 32 tokens, each one chain of instructions whose result is scaled and
// added while the next chain runs (32 x 32 x 64 and not 16 x 16 x 128 instructions: beside the latter vector
// instructions hardly issue, 33.5 against 45 cycles per 16 x 16 x 128 with its four additions).  Operands are
// read a unit ahead.  One barrier per step, before its last outputs: by then everybody has read the block, and the next
// one has arrived; the loads of the block after take its place and are spread over the units, because a wavefront stands
// still while a load is accepted.
//
// What bounds it: power.  At 32768 x 6144 x 4096 on codes (680 - 720 us from card to card, 2290 - 2430 Tflop/s) the matrix cores are busy 70 % of the
// cycles at 1.51 GHz of the card's 2.4.  On f16, whose instructions do half the work a cycle, 1340 - 1390 us.
template <int NI, int MT, int WN, int STAGES, bool FAST, bool F32, bool SPLIT, bool STREAM>
__global__ __launch_bounds__(512, 2) void gemm_tile_kernel(GemmFp8Params p, int tiles_m, int tiles_n, int splits)
{
    constexpr int TOKENS = 32 * MT * (8 / WN), SWAVES = TOKENS / 64;                       // (a wavefront brings 64 scales)
    constexpr int OUTPUTS = 32 * NI * WN, W_B = OUTPUTS * QBLOCK, A_B = TOKENS * QBLOCK, STAGE = W_B + A_B + 2048;     // weights | tokens | scales
    constexpr int WLOADS = OUTPUTS / 64, ALOADS = TOKENS / 64, LOADS = WLOADS + ALOADS + 1;                // per wavefront and block
    constexpr int UNITS = NI * MT;
    constexpr int PITCH = 272;                                                             // epilogue: a token's 256 bytes and 16 more
    static_assert(OUTPUTS % QBLOCK == 0 && UNITS % 2 == 0 && NI % 2 == 0 && LOADS <= 2 * UNITS + 1 && SWAVES < 8);
    static_assert(8 * 32 * PITCH <= STAGES * STAGE && STAGES * STAGE <= 160 * 1024);
    __shared__ __attribute__((aligned(1024))) unsigned char smem[STAGES * STAGE];
    LDS_AS unsigned char* lds = (LDS_AS unsigned char*)smem;
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // Workgroup -> tile: consecutive tiles on one XCD (ids equal mod 8), in bands of four tiles of tokens, so that what
    // an XCD runs at once shares its operands in its L2
    const int total = tiles_m * tiles_n * splits, per = (total + 7) / 8;
    int lin = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if (lin >= total) return;
    const int split = lin % splits;
    lin /= splits;
    constexpr int BAND = 4;
    const int band = lin / (BAND * tiles_n), rows_in = min(BAND, tiles_m - band * BAND), in = lin - band * BAND * tiles_n;
    const int m0 = (band * BAND + in % rows_in) * TOKENS, n0 = in / rows_in * OUTPUTS;
    const int blocks = (p.K + QBLOCK - 1) / QBLOCK, whole = p.K / QBLOCK;
    const int first = (int)((int64_t)whole * split / splits), last = (int)((int64_t)whole * (split + 1) / splits);

    // Loads: load i of a wavefront brings rows 8 (8 i + wave) .. + 7; rows past the end repeat the last (their outputs
    // are not stored)
    const int piece = (lane & 7) ^ ((lane >> 4) | ((wave & 1) << 2));
    uint32_t off_w[WLOADS], off_a[ALOADS];
#pragma unroll
    for (int i = 0; i < WLOADS; ++i) off_w[i] = (uint32_t)min((i * 8 + wave) * 8 + (lane >> 3), p.N - 1 - n0) * (uint32_t)p.K + piece * 16;
#pragma unroll
    for (int i = 0; i < ALOADS; ++i) off_a[i] = (uint32_t)min((i * 8 + wave) * 8 + (lane >> 3), p.M - 1 - m0) * (uint32_t)p.K + piece * 16;
    const uint8_t* a0 = p.a + (int64_t)m0 * p.K;
    const uint8_t* w0 = p.w + (int64_t)n0 * p.K;
    // scales: the first SWAVES wavefronts bring the tokens', the others the weights' (only those of the next are read)
    const bool tokens = wave < SWAVES;
    const float* scale0 = tokens ? p.a_scales + m0 : p.w_scales + (int64_t)(n0 / QBLOCK) * blocks;
    const int64_t scale_step = tokens ? p.scale_pitch : 1;
    const uint32_t off_s = 4u * (tokens ? (uint32_t)min(wave * 64 + lane, p.M - 1 - m0) : (uint32_t)min(lane % (OUTPUTS / QBLOCK), (p.N - 1 - n0) / QBLOCK) * (uint32_t)blocks);
    auto load = [&](int kb, uint32_t stage, int k) {
        if (k < WLOADS + ALOADS) {
            const bool W = k < WLOADS;
            const int i = W ? k : k - WLOADS;
            const uint8_t* src = (W ? w0 : a0) + (int64_t)kb * QBLOCK;
            const uint32_t dst = lds0 + stage + (W ? 0 : W_B) + i * 8192 + wave * 1024;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(dst), "v"(W ? off_w[i] : off_a[i]), "s"(src) : "memory");
        } else {
            const float* src = scale0 + kb * scale_step;
            const uint32_t dst = lds0 + stage + W_B + A_B + wave * 256;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" :: "s"(dst), "v"(off_s), "s"(src) : "memory");
        }
    };

    // Operands: lane (h, n) takes pieces h, 2 + h, 4 + h, 6 + h of row n
    const int wn = wave % WN, wm = wave / WN, key = (n >> 1) & 7;
    const uint32_t w_row = (wn * 32 * NI + n) * QBLOCK, a_row = W_B + (wm * 32 * MT + n) * QBLOCK;
    uint32_t at[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) at[r] = ((2 * r + h) ^ key) * 16;
    auto half = [&](uint32_t stage, uint32_t row, int q) -> i32x8 {
        LDS_AS unsigned char* st = lds + stage + row;
        const i32x4 lo = *(LDS_AS i32x4*)(st + at[2 * q]), hi = *(LDS_AS i32x4*)(st + at[2 * q + 1]);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    struct Raw { float a[MT], w; } raw;
    auto scales = [&](uint32_t stage) {
        LDS_AS unsigned char* st = lds + stage + W_B + A_B;
#pragma unroll
        for (int j = 0; j < MT; ++j) raw.a[j] = *(LDS_AS float*)(st + (wm * 32 * MT + j * 32 + n) * 4);
        raw.w = *(LDS_AS float*)(st + SWAVES * 256 + wn * 32 * NI / QBLOCK * 4);
    };
    f32x16 acc[NI][MT] = {}, s[2] = {};
    float f[MT] = {};
    i32x8 wv[2][2], av[MT][2];

    // the short block at the end of K, alone and first
    if (whole < blocks && split == splits - 1) {
        const bool in = piece * 16 < p.K - whole * QBLOCK;
#pragma unroll
        for (int k = 0; k < WLOADS + ALOADS; ++k) {
            const bool W = k < WLOADS;
            const int i = W ? k : k - WLOADS;
            const uint8_t* src = in ? (W ? w0 + off_w[i] : a0 + off_a[i]) + (int64_t)whole * QBLOCK : reinterpret_cast<const uint8_t*>(zeros16);
            const uint32_t dst = lds0 + (W ? 0 : W_B) + i * 8192 + wave * 1024;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(dst), "v"(src) : "memory");
        }
        load(whole, 0, LOADS - 1);
        wait_vmcnt<0>();
        barrier();
        scales(0);
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            const i32x8 a_lo = half(0, a_row + j * 4096, 0), a_hi = half(0, a_row + j * 4096, 1);
            const float fj = raw.a[j] * raw.w;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const f32x16 t = products<FAST>(half(0, w_row + i * 4096, 1), a_hi, products<FAST>(half(0, w_row + i * 4096, 0), a_lo, (f32x16){}));
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] += t[e] * fj;
            }
        }
        __syncthreads();
    }

    if (first < last) {
        const int steps = last - first;
        // loads of the last stage beyond the first 2 MT are left to the first step
#pragma unroll
        for (int st = 0; st < STAGES; ++st)
            if (st < steps)
#pragma unroll
                for (int k = 0; k < (st < STAGES - 1 ? LOADS : 2 * MT); ++k) load(first + st, st * STAGE, k);
        if (STAGES <= steps) wait_vmcnt<(STAGES - 2) * LOADS + 2 * MT>();
        else                 wait_vmcnt<0>();
        barrier();
#pragma unroll
        for (int q = 0; q < 2; ++q) {
#pragma unroll
            for (int j = 0; j < MT; ++j) av[j][q] = half(0, a_row + j * 4096, q);
            wv[0][q] = half(0, w_row, q);
        }
        scales(0);
        uint32_t prev = (STAGES - 1) * STAGE, cur = 0;
        Wide wide_a[MT][2], wide_w[2];                 // (on f16: each operand is widened once)
        // A step.  LOAD: of the blocks that take the place of the one before this and of this one the loads are still to be
        // sent (2), only of the former (1), of neither (0)
        auto step = [&](int kb, auto load_constant) {
            constexpr int LOAD = decltype(load_constant)::value;
            const uint32_t next = cur + STAGE == STAGES * STAGE ? 0u : cur + STAGE;
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int i = u / MT, j = u % MT;
                if (u == UNITS - MT) {
                    // this block is read (its last weights have arrived), the next one has landed
                    if constexpr (LOAD) wait_vmcnt<(STAGES - 2) * LOADS>();
                    else                wait_vmcnt<0>();
                    __builtin_amdgcn_s_waitcnt(0xC07F);               // lgkmcnt(0)
                    barrier();
                }
                __builtin_amdgcn_sched_barrier(0);
                if (j == 0) {
#pragma unroll
                    for (int q = 0; q < 2; ++q) wv[(i + 1) & 1][q] = i < NI - 1 ? half(cur, w_row + (i + 1) * 4096, q) : half(next, w_row, q);
                }
                if (u == 1) {
#pragma unroll
                    for (int t = 0; t < MT; ++t) f[t] = raw.a[t] * raw.w;
                }
                __builtin_amdgcn_sched_barrier(0);
                const int pu = (u + UNITS - 1) % UNITS;               // the unit before: its sums are scaled and added now
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const f32x16 c = q ? s[u & 1] : (f32x16){};
                    if constexpr (FAST) {
                        s[u & 1] = products<true>(wv[i & 1][q], av[j][q], c);
                    } else {
                        if (i == 0) wide_a[j][q] = widen32(av[j][q]);
                        if (j == 0) wide_w[q] = widen32(wv[i & 1][q]);
                        s[u & 1] = products(wide_w[q], wide_a[j][q], c);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    if (i == NI - 1) av[j][q] = half(next, a_row + j * 4096, q);
                    // a load per half chain from the barrier on
                    if (i == NI - 1) { if (LOAD == 2) load(first + kb + STAGES, cur, j * 2 + q); }
                    else if (LOAD && 2 * MT + u * 2 + q < LOADS) load(first + kb + STAGES - 1, prev, 2 * MT + u * 2 + q);
                    if (LOAD && LOADS > 2 * UNITS && u == 0 && q == 1) load(first + kb + STAGES - 1, prev, 2 * UNITS);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int e = 8 * q; e < 8 * q + 8; ++e) acc[pu / MT][pu % MT][e] += s[pu & 1][e] * f[pu % MT];
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (u == UNITS - 1) scales(next);
            }
            prev = cur;
            cur = next;
        };
        int kb = 0;
        for (; kb + STAGES < steps; ++kb) step(kb, std::integral_constant<int, 2>{});
        if (kb + STAGES == steps) step(kb++, std::integral_constant<int, 1>{});
        for (; kb < steps; ++kb) step(kb, std::integral_constant<int, 0>{});
        wait_vmcnt<0>();
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[NI - 1][MT - 1][e] += s[1][e] * f[MT - 1];
    }

    // Outputs: lane (h, n) holds outputs 8 r + 4 h .. + 3 of every 32, of token n.  Through LDS they leave in whole
    // lines: stored as they lie (8 bytes per token and lane) they took 10 % of the product of 32768 tokens.  16 bytes at
    // any address: rows of odd widths lie on two.
    __syncthreads();
    LDS_AS unsigned char* mine = lds + wave * 32 * PITCH;
    constexpr bool O32 = F32 || SPLIT;
    constexpr int COLS = O32 ? 64 : 32 * NI, PARTS = 32 * NI / COLS;             // outputs per pass
    constexpr int PER = O32 ? 4 : 8, LANES = COLS / PER;                         // per 16 bytes; lanes per token
    void* out = SPLIT ? static_cast<void*>(p.part + (int64_t)split * p.M * p.N) : p.out;
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
#pragma unroll
            for (int ii = 0; ii < COLS / 32; ++ii)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const f32x16& v = acc[part * (COLS / 32) + ii][j];
                    LDS_AS unsigned char* dst = mine + n * PITCH + (ii * 32 + 8 * r + 4 * h) * (O32 ? 4 : 2);
                    if constexpr (O32) *(LDS_AS f32x4*)dst = (f32x4){v[4 * r], v[4 * r + 1], v[4 * r + 2], v[4 * r + 3]};
                    else               *(LDS_AS u32x2*)dst = (u32x2){bf16_pair(v[4 * r], v[4 * r + 1]), bf16_pair(v[4 * r + 2], v[4 * r + 3])};
                }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int q = 0; q < LANES / 2; ++q) {
                const int t = q * (64 / LANES) + lane / LANES, m = m0 + wm * 32 * MT + j * 32 + t, c = n0 + wn * 32 * NI + part * COLS + lane % LANES * PER;
                const u32x4 v = *(LDS_AS u32x4*)(mine + t * PITCH + lane % LANES * 16);
                if (m >= p.M || c >= p.N) continue;
                const int64_t o = (int64_t)m * p.N + c;
                if (c + PER <= p.N) {
                    put_words_any<STREAM>(static_cast<unsigned char*>(out) + o * (O32 ? 4 : 2), v);
                } else {
#pragma unroll
                    for (int e = 0; e < PER; ++e)
                        if (c + e < p.N) {
                            if constexpr (O32) static_cast<float*>(out)[o + e] = __uint_as_float(v[e]);
                            else               static_cast<uint16_t*>(out)[o + e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
                        }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
}

// ---------------------------------------------------------------- in between

// A workgroup of eight wavefronts computes 32 NI outputs of 32 MT tokens, each wavefront all of them over every eighth block:
// what a wavefront reads from LDS it has brought there itself, in buffers of its own, so that it waits for nobody until the
// sums meet.  Up to a few hundred tokens, and for few outputs, such tiles over the whole depth beat large ones over shares
// of it, whose partial sums go through memory.
//
// What bounds it: what passes through LDS, 128 bytes a cycle read and written (64 come in), then the L2s and what is behind
// them where many CUs read; the launch and one round trip where a wavefront has few blocks.  Wavefronts of 32 x 32 that share
// the blocks of a 64 x 64 tile read each byte twice and meet at a barrier every step: 256 x 3584 x 3584 10.3 us on codes and
// 13.0 on f16, so 9.2 and 11.0; 61 x 3584 x 3584 6.7, so 5.5 (two buffers a wavefront, one for the larger tiles);
// 1024 x 576 x 4096 10.2, so 9.2.
template <int NI, int MT, int STAGES, bool FAST, bool F32>
__global__ __launch_bounds__(512, 2) void gemm_wave_tile_kernel(GemmFp8Params p, Layout tiles)
{
    constexpr int W_ROWS = 32 * NI, A_ROWS = 32 * MT, GROUPS = (W_ROWS + A_ROWS) / 8, LOADS = GROUPS + 1;
    constexpr int BLOCK_B = (W_ROWS + A_ROWS) * QBLOCK, STAGE = BLOCK_B + 256;
    constexpr int PITCH = W_ROWS + 4;                                                      // floats per token
    constexpr int LDS_B = std::max(8 * STAGES * STAGE, 8 * A_ROWS * PITCH * 4);
    static_assert((STAGES == 1 || (STAGES == 2 && MT == 1)) && MT <= 2 && LDS_B <= 160 * 1024);
    __shared__ __attribute__((aligned(1024))) unsigned char smem[LDS_B];
    LDS_AS unsigned char* lds = (LDS_AS unsigned char*)smem;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int m0, n0;
    const bool there = tiles.at(blockIdx.x, m0, n0);
    m0 *= A_ROWS;
    n0 *= W_ROWS;
    if (!there || m0 >= p.M || n0 >= p.N) return;
    const int blocks = (p.K + QBLOCK - 1) / QBLOCK;
    const uint32_t mine = (uint32_t)(uintptr_t)lds + wave * STAGES * STAGE;

    // Load k of a block: rows 8 k .. + 7 of w, then of a; 16-byte piece c of a row lies at c ^ (row >> 1 & 7).  Rows past the end
    // repeat the last
    const uint32_t row = (uint32_t)(lane >> 3) * (uint32_t)p.K, even = ((lane & 7) ^ (lane >> 4)) * 16;
    const uint32_t last_w = (uint32_t)min(W_ROWS - 1, p.N - 1 - n0) * (uint32_t)p.K, last_a = (uint32_t)min(A_ROWS - 1, p.M - 1 - m0) * (uint32_t)p.K;
    const uint8_t* w0 = p.w + (int64_t)n0 * p.K;
    const uint8_t* a0 = p.a + (int64_t)m0 * p.K;
    // Scales: of 32 tokens and, in the other half of the lanes, the weights'; of 64 tokens, and the weights' goes to a register
    // (asked for a block ahead: 1 - 4 % longer; with 32 tokens through a register: 4 - 7 %)
    const float* ws = p.w_scales + (int64_t)(n0 / QBLOCK) * blocks;
    const bool token = MT == 2 || lane < 32;
    const float* scale0 = token ? p.a_scales + min(m0 + lane, p.M - 1) : ws;
    const int64_t scale_step = token ? p.scale_pitch : 1;
    auto request = [&](int b, uint32_t stage) {
        const int64_t at = (int64_t)b * QBLOCK;
        const uint32_t row_step = 8u * (uint32_t)p.K;
        auto off = [&](int k, bool W) { return min(row + (uint32_t)(W ? k : k - W_ROWS / 8) * row_step, W ? last_w : last_a) + (even ^ (k & 1) * 64); };
        if (at + QBLOCK <= p.K) {
#pragma unroll
            for (int k = 0; k < GROUPS; ++k) {
                const bool W = k < W_ROWS / 8;
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(mine + stage + k * 1024), "v"(off(k, W)), "s"((W ? w0 : a0) + at) : "memory");
            }
        } else {                                       // columns at and past K are zeros
#pragma unroll
            for (int k = 0; k < GROUPS; ++k) {
                const bool W = k < W_ROWS / 8;
                const uint8_t* src = at + (even ^ (k & 1) * 64) < p.K ? (W ? w0 : a0) + at + off(k, W) : reinterpret_cast<const uint8_t*>(zeros16);
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(mine + stage + k * 1024), "v"(src) : "memory");
            }
        }
        const float* src = scale0 + b * scale_step;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" :: "s"(mine + stage + BLOCK_B), "v"(src) : "memory");
    };

    f32x16 acc[NI][MT] = {};
#pragma unroll
    for (int st = 0; st < STAGES; ++st)
        if (wave + 8 * st < blocks) request(wave + 8 * st, st * STAGE);
    uint32_t cur = 0;
    const int key = (n >> 1) & 7;
    LDS_AS unsigned char* own = lds + wave * STAGES * STAGE;
    for (int b = wave; b < blocks; b += 8) {
        float sw = MT == 2 ? ws[b] : 0.f;
        if (STAGES == 2 && b + 8 < blocks) wait_vmcnt<LOADS>();
        else                               wait_vmcnt<0>();
        asm volatile("" ::: "memory");
        i32x8 wv[NI][2], av[MT][2];
        float sa[MT];
        LDS_AS unsigned char* st = own + cur;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t lo = ((4 * q + h) ^ key) * 16, hi = ((4 * q + 2 + h) ^ key) * 16;
            auto half = [&](int r) {
                LDS_AS unsigned char* at = st + (r * 32 + n) * QBLOCK;
                return __builtin_shufflevector(*(LDS_AS i32x4*)(at + lo), *(LDS_AS i32x4*)(at + hi), 0, 1, 2, 3, 4, 5, 6, 7);
            };
#pragma unroll
            for (int i = 0; i < NI; ++i) wv[i][q] = half(i);
#pragma unroll
            for (int j = 0; j < MT; ++j) av[j][q] = half(NI + j);
        }
#pragma unroll
        for (int j = 0; j < MT; ++j) sa[j] = *(LDS_AS float*)(st + BLOCK_B + (j * 32 + n) * 4);
        if (MT == 1) sw = *(LDS_AS float*)(st + BLOCK_B + 32 * 4);
        __builtin_amdgcn_s_waitcnt(0xC07F);            // lgkmcnt(0): the block is in registers, the next may take its place
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        if (b + 8 * STAGES < blocks) request(b + 8 * STAGES, cur);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const f32x16 s = products<FAST>(wv[i][1], av[j][1], products<FAST>(wv[i][0], av[j][0], (f32x16){}));
                const float f = sa[j] * sw;
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] += s[e] * f;
            }
        if (STAGES == 2) cur ^= STAGE;
    }
    __syncthreads();
    // sums of the wavefronts' blocks, in their order; [wave][token][output]
    LDS_AS float* red = (LDS_AS float*)lds;
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *(LDS_AS f32x4*)(red + (wave * A_ROWS + j * 32 + n) * PITCH + i * 32 + 8 * r + 4 * h) =
                    (f32x4){acc[i][j][4 * r], acc[i][j][4 * r + 1], acc[i][j][4 * r + 2], acc[i][j][4 * r + 3]};
    __syncthreads();
    for (int i = tid; i < W_ROWS * A_ROWS / 4; i += 512) {
        const int c = i % (W_ROWS / 4) * 4, t = i / (W_ROWS / 4);                          // four outputs of a token
        const LDS_AS float* at = red + t * PITCH + c;
        f32x4 v = *(const LDS_AS f32x4*)at;
#pragma unroll
        for (int k = 1; k < 8; ++k) v += *(const LDS_AS f32x4*)(at + k * A_ROWS * PITCH);
        const int m = m0 + t, col = n0 + c;
        if (m >= p.M || col >= p.N) continue;
        const int64_t o = (int64_t)m * p.N + col;
        if (col + 4 <= p.N) {
            if constexpr (F32) *reinterpret_cast<words4_any*>(static_cast<float*>(p.out) + o) = __builtin_bit_cast(words4, v);
            else               *reinterpret_cast<words2_any*>(static_cast<uint16_t*>(p.out) + o) = (words2){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < p.N) put<F32>(p.out, o + e, v[e]);
        }
    }
}

// partial products of the shares of K, added in their order
template <bool F32>
__global__ __launch_bounds__(256) void gemm_merge_kernel(GemmFp8Params p, int splits)
{
    const int64_t size = (int64_t)p.M * p.N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < size; i += (int64_t)gridDim.x * 256) {
        float v = p.part[i];
        for (int s = 1; s < splits; ++s) v += p.part[s * size + i];
        put<F32>(p.out, i, v);
    }
}

// ---------------------------------------------------------------- choice

enum Form { ROWS, WAVE_32x32, WAVE_64x32, WAVE_64x64, TILE_128x128, TILE_256x128, TILE_256x256 };
constexpr int TILE[][2] = {{16, 16}, {32, 32}, {64, 32}, {64, 64}, {128, 128}, {256, 128}, {256, 256}};      // tokens, outputs
struct Plan {
    Form form;
    int splits;      // shares of K
    int tokens;      // of this launch; those beyond go to another
    float us;
};

// The form that a model of the times finds fastest: a launch, per round of 256 workgroups (each fills its CU) the steps over K,
// and something from a round to the next; or the time that the operands take from memory.  us per step with few workgroups;
// the fuller the rounds, the longer the steps, for power and the caches' rates (`crowded`: all CUs).  Fitted to 280 sizes of 17 to
// 32768 tokens and ten (N, K), with each kind of sums: the choice takes 0.2 % longer than the best form on average, 18 %
// at the most.
Plan one_launch(int M, int N, int K, bool fast)
{
    const int blocks = (K + QBLOCK - 1) / QBLOCK;
    // (one token by 3584 x 3584 4.5 us, 32 x 32 tiles 5.4; by 6144 x 4096, more workgroups than CUs, 7.5 and 6.9)
    if (M <= 16 && (N + 15) / 16 <= 256) return {ROWS, 1, M, 4.f};
    struct Times { float launch, step, crowded, round; };
    struct Shape { Form form; int blocks; Times fast, f16; };
    static const Shape shapes[] = {
        {WAVE_32x32, 8, {2.4f, 0.70f, 1.2f, 1.f}, {2.8f, 0.73f, 1.35f, 1.f}}, {WAVE_64x32, 8, {2.4f, 1.01f, 1.35f, 1.f}, {2.8f, 1.13f, 1.2f, 1.5f}},
        {WAVE_64x64, 8, {3.2f, 1.46f, 1.2f, 2.f}, {3.6f, 1.85f, 1.2f, 3.5f}}, {TILE_128x128, 1, {4.f, 0.336f, 1.65f, 2.f}, {4.f, 0.75f, 1.35f, 2.f}},
        {TILE_256x128, 1, {4.4f, 0.545f, 1.9f, 2.f}, {4.4f, 1.2f, 1.5f, 2.f}}, {TILE_256x256, 1, {4.4f, 1.24f, 1.35f, 2.f}, {}}};
    Plan best = {TILE_256x128, 1, M, 3e38f};
    for (const Shape& f : shapes) {
        if (f.form == TILE_256x256 && !fast) continue;                   // (its registers are taken on f16)
        const Times& t = fast ? f.fast : f.f16;
        const long tokens = TILE[f.form][0], outputs = TILE[f.form][1], tiles = ((M + tokens - 1) / tokens) * ((N + outputs - 1) / outputs);
        const int steps = (blocks + f.blocks - 1) / f.blocks;
        // shares of K, merged by a second launch
        for (int s = 1; s == 1 || (f.form == TILE_256x128 && s <= 8 && steps / s >= 4 && tiles * s <= 256); s *= 2) {
            const long rounds = (tiles * s + 255) / 256;
            const float fill = (float)(tiles * s) / (float)(rounds * 256);
            const float step = t.step * (1.f + (t.crowded - 1.f) * fill * fill);
            const float memory = ((float)N + (float)M) * (float)K / 5.5e6f;
            float us = t.launch + std::max(memory, (float)rounds * (float)((steps + s - 1) / s) * step + (float)(rounds - 1) * t.round);
            if (s > 1) us += 4.0f + (float)s * (float)M * (float)N * 8.f / 6e6f;      // (the partial sums, in the caches)
            if (us < best.us) best = {f.form, s, M, us};
        }
    }
    return best;
}

// One launch, or one whose tiles fill whole rounds and another for the tokens that are left: the last round of large tiles
// is rarely full (4000 x 5376 x 3584: 336 tiles, 82.8 us; 252 and the rest in smaller ones 74.5).
Plan plan_of(int M, int N, int K, bool fast)
{
    Plan best = one_launch(M, N, K, fast);
    if (best.form < TILE_128x128 || best.splits > 1) return best;
    const int rows = TILE[best.form][0], wide = TILE[best.form][1];
    const long across = (N + wide - 1) / wide, down = (M + rows - 1) / rows, rounds = (down * across) / 256;
    const long whole = rounds * 256 / across;                            // rows of tiles in so many rounds
    if (whole < 1 || whole >= down) return best;
    const int tokens = (int)whole * rows;
    const Plan main = one_launch(tokens, N, K, fast), rest = one_launch(M - tokens, N, K, fast);
    const float us = main.us + rest.us - 2.f;                            // (the second launch is in place when the first ends)
    return us < best.us ? Plan{main.form, main.splits, tokens, us} : best;
}

long workgroups(const Plan& plan, int N)
{
    const int* t = TILE[plan.form];
    return (long)((plan.tokens + t[0] - 1) / t[0]) * ((N + t[1] - 1) / t[1]) * plan.splits;
}

template <int WAVES, int U> void launch_rows(const GemmFp8Params& p, bool f32, hipStream_t s)
{
    const dim3 grid((unsigned)((p.N + 15) / 16)), block(WAVES * 64);
    if (f32) gemm_rows_kernel<WAVES, U, true><<<grid, block, 0, s>>>(p);
    else     gemm_rows_kernel<WAVES, U, false><<<grid, block, 0, s>>>(p);
}

// The rectangles with the fewest rows of operands, of those that take no more rounds than tiles in a row
Layout layout_of(int tiles_m, int tiles_n, int tokens, int outputs)
{
    const long per = ((long)tiles_m * tiles_n + 7) / 8, rounds = (per + 31) / 32;
    Layout best = {-1, tiles_m, (int)per, 0.f};
    long best_rows = 0;
    for (int l = 0; l <= 3; ++l) {
        const int across = 1 << l, down = 8 >> l, rows = (tiles_m + across - 1) / across, columns = (tiles_n + down - 1) / down;
        const long size = (long)rows * tokens + (long)columns * outputs;
        if (((long)rows * columns + 31) / 32 > rounds || (best.log_across >= 0 && size >= best_rows)) continue;
        best = {l, rows, columns, 1.f / (float)rows};
        best_rows = size;
    }
    return best;
}

template <int NI, int MT, int STAGES> void launch_wave_tiles(const GemmFp8Params& p, bool f32, bool fast, hipStream_t s)
{
    const Layout tiles = layout_of((p.M + 32 * MT - 1) / (32 * MT), (p.N + 32 * NI - 1) / (32 * NI), 32 * MT, 32 * NI);
    const dim3 grid((unsigned)tiles.workgroups()), block(512);
    if (fast) {
        if (f32) gemm_wave_tile_kernel<NI, MT, STAGES, true, true><<<grid, block, 0, s>>>(p, tiles);
        else     gemm_wave_tile_kernel<NI, MT, STAGES, true, false><<<grid, block, 0, s>>>(p, tiles);
    } else {
        if (f32) gemm_wave_tile_kernel<NI, MT, STAGES, false, true><<<grid, block, 0, s>>>(p, tiles);
        else     gemm_wave_tile_kernel<NI, MT, STAGES, false, false><<<grid, block, 0, s>>>(p, tiles);
    }
}

template <int NI, int MT, int WN, int STAGES, bool FAST> void launch_tiles(const GemmFp8Params& p, bool f32, int splits, hipStream_t s)
{
    constexpr int TOKENS = 32 * MT * (8 / WN), OUTPUTS = 32 * NI * WN;
    const int tm = (p.M + TOKENS - 1) / TOKENS, tn = (p.N + OUTPUTS - 1) / OUTPUTS;
    const dim3 grid((unsigned)(((long)tm * tn * splits + 7) / 8 * 8)), block(512);
    const bool stream = (int64_t)p.M * p.N * (f32 ? 4 : 2) > STREAM_BYTES;
    auto run = [&](auto is_f32, auto is_split, auto is_stream) {
        gemm_tile_kernel<NI, MT, WN, STAGES, FAST, decltype(is_f32)::value, decltype(is_split)::value, decltype(is_stream)::value>
            <<<grid, block, 0, s>>>(p, tm, tn, splits);
    };
    using std::true_type;
    using std::false_type;
    if (splits > 1) { if constexpr (OUTPUTS == 128 && TOKENS == 256) run(false_type{}, true_type{}, false_type{}); }
    else if (f32)                    stream ? run(true_type{}, false_type{}, true_type{}) : run(true_type{}, false_type{}, false_type{});
    else                             stream ? run(false_type{}, false_type{}, true_type{}) : run(false_type{}, false_type{}, false_type{});
    if (splits > 1) {
        const dim3 mg((unsigned)std::min<int64_t>(((int64_t)p.M * p.N + 255) / 256, 4096));
        if (f32) gemm_merge_kernel<true><<<mg, dim3(256), 0, s>>>(p, splits);
        else     gemm_merge_kernel<false><<<mg, dim3(256), 0, s>>>(p, splits);
    }
}

}  // namespace

// f(plan, tokens before it) for every launch of a product
template <typename F> static void each_launch(int M, int N, int K, bool fast, F f)
{
    const Plan first = plan_of(M, N, K, fast);
    f(first, 0);
    if (first.tokens < M) f(one_launch(M - first.tokens, N, K, fast), first.tokens);
}

constexpr int MOST = 1 << 30;        // tokens, outputs: sums with a tile's size stay in 32 bits

size_t gemm_fp8_workspace(int M, int N, int K)
{
    if (M > MOST || N > MOST) return 0;
    size_t most = 0;
    for (bool fast : {false, true})
        each_launch(M, N, K, fast, [&](const Plan& plan, int) {
            if (plan.splits > 1) most = std::max(most, (size_t)plan.splits * plan.tokens * N * sizeof(float));
        });
    return most;
}

bool gemm_fp8_supported(int M, int N, int K)
{
    if (M > MOST || N > MOST) return false;
    long most = 0;
    for (bool fast : {false, true}) each_launch(M, N, K, fast, [&](const Plan& plan, int) { most = std::max(most, workgroups(plan, N)); });
    return most < 1l << 22;              // (1024 threads each at most)
}

hipError_t launch_gemm_fp8(const GemmFp8Params& all, mla_dtype out, bool fast_sums, hipStream_t s)
{
    const bool f32 = out == MLA_F32;
    each_launch(all.M, all.N, all.K, fast_sums, [&](const Plan& plan, int before) {
        GemmFp8Params p = all;
        p.M = plan.tokens;
        p.a += (int64_t)before * all.K;
        p.a_scales += before;
        p.out = static_cast<char*>(all.out) + (int64_t)before * all.N * (f32 ? 4 : 2);
        switch (plan.form) {
            case ROWS:       launch_rows<16, 2>(p, f32, s); break;
            case WAVE_32x32: launch_wave_tiles<1, 1, 2>(p, f32, fast_sums, s); break;
            case WAVE_64x32: launch_wave_tiles<1, 2, 1>(p, f32, fast_sums, s); break;
            case WAVE_64x64: launch_wave_tiles<2, 2, 1>(p, f32, fast_sums, s); break;
            case TILE_128x128:
                if (fast_sums) launch_tiles<2, 1, 2, 3, true>(p, f32, 1, s);
                else           launch_tiles<2, 1, 2, 3, false>(p, f32, 1, s);
                break;
            case TILE_256x128:
                if (fast_sums) launch_tiles<2, 2, 2, 3, true>(p, f32, plan.splits, s);
                else           launch_tiles<2, 2, 2, 3, false>(p, f32, plan.splits, s);
                break;
            case TILE_256x256: launch_tiles<4, 2, 2, 2, true>(p, f32, 1, s); break;
        }
    });
    return hipGetLastError();
}

}  // namespace mla
