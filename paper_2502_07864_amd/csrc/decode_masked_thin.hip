// Masked attention over the latent cache on the matrix cores for few query rows (bf16 queries, bf16 or fp8 cache): 32 query rows per workgroup.
//
//   S^T [keys x 32] = K [keys x (d_c + 64)] . Q^T,   O^T [d_c x 32] += V^T [d_c x keys] . P^T,   V = the first d_c columns of K
//
// Few rows are bound by the stream of the cache.  The four wavefronts of a workgroup have the same 32 query rows and take the chunk's
// tiles of 32 keys in turn, each with a place of its own in the LDS and a softmax of its own: no barrier until the end, where the four
// results are joined.  A wavefront waits for its tile block by block, scores, weighs and accumulates it, and asks for its next one block by block beside the value products; while one waits the
// others compute, so that two or three tiles of a CU are on their way at any time, and a chunk of up to four tiles is one round trip.  fp8 tiles are half as
// wide: a wavefront has two places, and asks two tiles ahead; codes are widened to bf16 (exactly) where they are read, the row's scale goes to
// scores and weights.
//
// A small call is bound by round trips (length, page, tile, and one for whatever of the code comes first: what runs once is kept short,
// loops instead of their copies).
//
// Measured: 64 sequences x 32 rows under a window of 4096 70 us a call, 307 MB, 4.5 to 4.7 TB/s in the kernel (past the caches; 82 with whole tiles asked for at the end of the
// last one and through them); a window of 4096 of one sequence 16 us in the kernel, of which 4 are the join (the kernel for plain decode, whose wavefronts share every tile and
// have nothing to join, takes 8 for as many rows); 256 rows on 1000 cached ones 18, where the kernel for many rows takes 20.  fp8: 16 sequences of 64000 rows, 32
// query rows, 116 us a call, 5.1 TB/s (on the kernel for many rows 292); bf16 193 us, 6.1 TB/s.
//
// References of the exponentials, masks and keys that are not finite: as in the kernel for many rows (decode_masked.hip), but that a
// wavefront goes over its tiles again by itself where a score exceeds its reference by more than 2^64.
#include "masked_tile.h"
#include <type_traits>

namespace mla {
namespace {

typedef __attribute__((ext_vector_type(2))) int i32x2;

// ONCE: tiles that this workgroup alone reads, past the caches.  32 query rows: 64 sequences under a window of 4096 80 us without, 70 with; 16 x 64000 rows 218, 192,
// in fp8 130, 116.  Where other groups of rows read them too it costs more than it gives (256 rows on 4 x 16000: 62, 68), and where a call's rows are few
// enough to be found in a cache by the next call (16 x 4000 rows, 75 MB: 38 and 34 on six sets in turn, 33 and 34 on two; one sequence of 16000, 19 MB: 27, 29).
template <int D_C, bool FP8, bool ONCE>
__global__ __launch_bounds__(MF_THREADS, 1) void masked_thin_kernel(MaskedParams p)
{
    constexpr int ROW = D_C + 64, ROWB = FP8 ? ROW : ROW * 2, CPR = ROWB / 16;
    constexpr int TILE_B = MK_TILE * ROWB;
    constexpr int NKS = ROW / 32, NCT = D_C / 16;
    constexpr int PLACES = FP8 ? 2 : 1, PLACE_B = PLACES * TILE_B;       // of a wavefront

    __shared__ __attribute__((aligned(1024))) unsigned char smem[4 * PLACE_B];
    __shared__ __attribute__((aligned(16))) float ks_smem[FP8 ? 4 : 1][2][64];     // (fp8) scales of the rows of a tile, twice
    __shared__ uint64_t tree_smem[64];
    __shared__ float m_smem[4][32], l_smem[4][32];      // reference and normaliser of every wavefront's rows
    __shared__ __attribute__((aligned(16))) float f_smem[32][4];         // and factor
    LDS_AS unsigned char* lds = (LDS_AS unsigned char*)smem;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;

    // the groups of query rows of one chunk get linear ids 8 apart: same XCD, same time, so all but the first find the rows in its L2
    const int Z = (p.H + MK_THIN_ROWS - 1) / MK_THIN_ROWS;
    const int id = blockIdx.x, rr = id >> 3;
    const int zi = (int)((unsigned)rr % (unsigned)Z), wg = chunk_at((rr - zi) / Z, id & 7);
    if (wg >= p.B * p.num_splits) return;               // padding of the last group of 8
    const int split = (int)((unsigned)wg % (unsigned)p.num_splits), b = sequence_at(p, (int)((unsigned)wg / (unsigned)p.num_splits), lane);
    const int hb = zi * MK_THIN_ROWS, HL = min(MK_THIN_ROWS, p.H - hb);

    const bool tree = p.tree != nullptr;
    const Reach reach = reach_of(((const CONST_AS int32_t*)p.lens)[b], p.q_len, p.max_pages * p.page_size, tree, p.window, p.sinks);
    const int v0 = chunk_start(reach.tiles, split, p.num_splits), v1 = chunk_start(reach.tiles, split + 1, p.num_splits);
    auto part_of = [&](int r) { return part_index(b, hb + r, split, p.H, p.num_splits); };
    if (v0 >= v1) {                                     // nothing to see
        for (int r = wave; r < HL; r += 4) {
            if (p.num_splits == 1)
                for (int c = lane * 8; c < D_C; c += 512)
                    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.o_part) + part_of(r) * D_C + c) = (u32x4){0u, 0u, 0u, 0u};
            if (lane == 0 && p.lse_part) p.lse_part[part_of(r)] = -INFINITY;
        }
        return;
    }

    // ---- this wavefront's tiles: v0 + wave, + 4, ...; where their halves lie, 32 tiles at a time, a lane each
    const int32_t* const ptab = p.page_table + (size_t)b * p.max_pages;
    const int per_page = p.page_size / 16;
    auto ids_from = [&](int v) {
        const int k = 2 * reach.tile(min(v + 4 * (lane >> 1), v1 - 1)) + (lane & 1);
        return half_at(p, half_page(p, ptab, per_page, k), per_page, k);
    };
    LDS_AS unsigned char* const mine = lds + wave * PLACE_B;
    LDS_AS float* const my_scales = (LDS_AS float*)ks_smem[FP8 ? wave : 0][0];
    const uint32_t dst = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)mine);
    // (fp8) codes as they are, chunk c of row r at position c ^ (r >> 2 & 2), and the scales; always as many loads, so that they can be waited
    // for by count: a half that is not there is some other, which nobody sees
    constexpr int PER_TILE = FP8 ? TILE_B / 1024 + 1 : 0;
    // (bf16) in blocks of 64 columns, row r of a block behind row r - 1, its chunk c at position c ^ (r >> 1 & 7): the 16 rows of a read meet 16 different
    // units, and a block that is done with can be asked for again while the others are read
    constexpr int BLOCKS = ROW / 64, BLOCK_B = MK_TILE * 128;
    auto load16 = [&](uint32_t to, uint32_t off, const unsigned char* src) {
        if constexpr (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "s"(to), "v"(off), "s"(src) : "memory");
        else                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(to), "v"(off), "s"(src) : "memory");
    };
    auto request_block = [&](const Place& s, int c) {
        const int l = lane_again();
#pragma unroll
        for (int i = 0; i < 4; ++i) {                   // eight rows at a time
            const unsigned char* src = static_cast<const unsigned char*>(p.kv) + (size_t)max(i < 2 ? s.lo : s.hi, 0) * (TILE_B / 2) + (i & 1) * (8 * ROWB) + c * 128;
            const uint32_t off = (uint32_t)((l >> 3) * ROWB) + (uint32_t)(((l & 7) ^ ((l >> 4) + 4 * (i & 1))) << 4), to = dst + (uint32_t)(c * BLOCK_B + i * 1024);
            load16(to, off, src);
        }
    };
    auto request = [&](const Place& s, int slot) {
        const int l = lane_again();
        if constexpr (FP8) {
            const uint32_t to = dst + (uint32_t)slot * TILE_B;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const unsigned char* src = static_cast<const unsigned char*>(p.kv) + (size_t)max(h ? s.hi : s.lo, 0) * (TILE_B / 2);
#pragma unroll
                for (int k = 0; k < TILE_B / 2048; ++k) {
                    const uint32_t off = (uint32_t)(l * 16) ^ (k * 64 + l >= 8 * CPR ? 32u : 0u), at = to + (uint32_t)h * (TILE_B / 2) + (uint32_t)k * 1024u;
                    load16(at, off, src + k * 1024);
                }
            }
            const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)my_scales + (uint32_t)slot * 256u);
            const int low = s.lo, high = s.hi;
            const float* from = p.kv_scale + (size_t)max(l & 16 ? high : low, 0) * 16 + (l & 15);
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" :: "s"(at), "v"(from) : "memory");
            return;
        }
#pragma unroll 1
        for (int c = 0; c < BLOCKS; ++c) request_block(s, c);
    };
    Place at, next = Place{-1, -1};                     // of this tile, (fp8) and of the wavefront's next one
    int32_t ids;
    auto place_now = [&](int v) { return tile_place(p, (const CONST_AS int32_t*)ptab, per_page, reach.tile(v)); };
    auto start = [&]() {
        at = Place{-1, -1};
        if (v0 + wave < v1) {
            at = place_now(v0 + wave);
            request(at, 0);
        }
        if (FP8 && v0 + wave + 4 < v1) {
            next = place_now(v0 + wave + 4);
            request(next, 1);
        }
        ids = ids_from(v0 + wave);
    };
    start();

    // ---- the query rows -> registers (B operands of the scores; a negative scale changes their sign)
    bf16x8 qreg[2][NKS];
    {
        const uint16_t* qa = static_cast<const uint16_t*>(p.q_abs) + (size_t)b * p.H * D_C;
        const uint16_t* qr = static_cast<const uint16_t*>(p.q_rope) + (size_t)b * p.H * 64;
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            const size_t row = hb + min(hi * 16 + n, HL - 1);
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) {
                // (fp8: a lane reads 16 codes at a time, eight for each of two k-steps)
                const int kl = ks < D_C / 32 ? ks : ks - D_C / 32, col = FP8 ? (kl >> 1) * 64 + g * 16 + (kl & 1) * 8 : kl * 32 + g * 8;
                const u32x4 v = ks < D_C / 32 ? *reinterpret_cast<const u32x4*>(qa + row * D_C + col) : *reinterpret_cast<const u32x4*>(qr + row * 64 + col);
                qreg[hi][ks] = __builtin_bit_cast(bf16x8, v);
            }
        }
    }
    if (p.scale < 0.f) {
        asm volatile("");                               // (a branch, not 144 instructions for everybody)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
                qreg[hi][ks] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, qreg[hi][ks]) ^ (u32x4){0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u});
    }
    if (tree) {
        if (tid < p.q_len) tree_smem[tid] = tree_word(p, b, tid);
        __syncthreads();
    }
    const WholeTiles whole = whole_tiles(p, reach, hb / p.heads, (hb + HL - 1) / p.heads);
    int token[2];
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) token[hi] = (hb + min(hi * 16 + n, HL - 1)) / p.heads;

    // ---- per-lane state: this lane's queries = column n of the D tiles of the two groups
    float m_ref[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
    f32x4 oacc[2][NCT];
    const float sc = fmaxf(fabsf(p.scale) * LOG2E, 1.17549435e-38f);     // (never zero: a masked score is -inf and has to stay it)

    // keys and places of the reads: as in the kernel for many rows
    constexpr int LANE_KEYS = FP8 ? 8 : 4, BLOCK_KEYS = FP8 ? 4 : 16;         // key LANE_KEYS g + BLOCK_KEYS rb + i
    uint32_t a_base[2], t_base[4];
    if constexpr (FP8) {
        const int row = 8 * (n >> 2) + (n & 3), from = 8 * g + (n >> 1);
        a_base[0] = a_base[1] = (uint32_t)(row * ROWB) + (((uint32_t)g ^ (uint32_t)(row >> 2 & 2)) << 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) t_base[e] = (uint32_t)(from * ROWB) + (((uint32_t)e ^ (uint32_t)(from >> 2 & 2)) << 4) + (uint32_t)((n & 1) * 8);
    } else {
#pragma unroll
        for (int e = 0; e < 2; ++e) a_base[e] = (uint32_t)(n * 128) + (((uint32_t)(4 * e + g) ^ (uint32_t)(n >> 1)) << 4);
        const int r = g * 4 + (n >> 2);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            t_base[e] = (uint32_t)(r * 128) + ((((uint32_t)(2 * e) + (uint32_t)((n & 3) >> 1)) ^ (uint32_t)(r >> 1 & 7)) << 4) + (uint32_t)((n & 1) * 8);
    }
    f32x4 ksc[2];                                       // (fp8) scales of this lane's keys

    // ---- sweeps over the tiles: ACCUMULATE against the references, and where some score exceeded its own by more than FAST_GAP (rare) one
    // for the exact maxima (it accumulates too, which is not used) and one against them
    enum { ACCUMULATE, MAXIMA, ACCUMULATE_AGAIN };
    bool unset = true;
    for (int pass = ACCUMULATE;;) {
        float top[2] = {-INFINITY, -INFINITY};          // largest score of the sweep so far, this lane's keys (unscaled)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            l_run[hi] = 0.f;
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) oacc[hi][ct] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
        int turn = 0;
        if constexpr (!FP8) wait_vmcnt<0>();            // (the queries, too: else each of their registers would be waited for in the loop)
        for (int v = v0 + wave; v < v1; v += 4, ++turn) {
            if (turn && (turn & 31) == 0) ids = ids_from(v);
            if constexpr (FP8) {
                if (v + 4 < v1) wait_vmcnt<PER_TILE>();
                else            wait_vmcnt<0>();
                __builtin_amdgcn_sched_barrier(0);
            }
            LDS_AS unsigned char* const tile = mine + (FP8 ? (turn & 1) * TILE_B : 0);

            // ---- scores
            f32x4 x[2][2];
            {
                bf16x8 ka[2][NKS], kk[2][2];
                u32x4 raw[2][NKS / 2];                      // (fp8) the codes of two k-steps
                auto key_of = [&](int rb, int ks) -> bf16x8 {
                    if constexpr (FP8) return widened(raw[rb][ks / 2][ks % 2 * 2], raw[rb][ks / 2][ks % 2 * 2 + 1]);
                    else               return ka[rb][ks];
                };
                // (bf16) blocks 0 .. c are there: those behind them, four loads each, may be on their way
                auto landed = [&](int c) {
                    switch (BLOCKS - 1 - c) {
                    case 0: wait_vmcnt<0>(); break;
                    case 1: wait_vmcnt<4>(); break;
                    case 2: wait_vmcnt<8>(); break;
                    case 3: wait_vmcnt<12>(); break;
                    case 4: wait_vmcnt<16>(); break;
                    case 5: wait_vmcnt<20>(); break;
                    case 6: wait_vmcnt<24>(); break;
                    case 7: wait_vmcnt<28>(); break;
                    default: wait_vmcnt<32>();
                    }
                    __builtin_amdgcn_sched_barrier(0);
                };
                auto rk = [&](int ks) {
                    if constexpr (FP8) {
                        if (ks % 2 == 0) {
#pragma unroll
                            for (int rb = 0; rb < 2; ++rb) raw[rb][ks / 2] = *(LDS_AS u32x4*)(tile + a_base[0] + ks / 2 * 64 + rb * 4 * ROWB);
                        }
                        return;
                    }
                    if (ks % 2 == 0) landed(ks / 2);
#pragma unroll
                    for (int rb = 0; rb < 2; ++rb) ka[rb][ks] = *(LDS_AS bf16x8*)(tile + a_base[ks & 1] + (ks >> 1) * BLOCK_B + rb * 16 * 128);
                };
                static constexpr int AHEAD = 4;
                static_assert(BLOCKS == 9 || BLOCKS == 5);
#pragma unroll
                for (int ks = 0; ks < AHEAD; ++ks) rk(ks);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int ks = 0; ks < NKS; ++ks) {
                    if (ks + AHEAD < NKS) rk(ks + AHEAD);
#pragma unroll
                    for (int rb = 0; rb < 2; ++rb) {
                        kk[ks & 1][rb] = FP8 && ks ? kk[ks & 1][rb] : key_of(rb, ks);
                        if (FP8 && ks + 1 < NKS) kk[~ks & 1][rb] = key_of(rb, ks + 1);      // (widened beside the matrix instructions before)
                    }
#pragma unroll
                    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                        for (int hi = 0; hi < 2; ++hi)
                            x[rb][hi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk[ks & 1][rb], qreg[hi][ks], ks == 0 ? (f32x4){0.f, 0.f, 0.f, 0.f} : x[rb][hi], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if constexpr (FP8) {
#pragma unroll
                for (int rb = 0; rb < 2; ++rb) {
                    ksc[rb] = *(LDS_AS f32x4*)(my_scales + (turn & 1) * 64 + g * 8 + rb * 4);
#pragma unroll
                    for (int hi = 0; hi < 2; ++hi) x[rb][hi] *= ksc[rb];
                }
            }
            if (__builtin_expect(!at.whole() || !whole.holds(v), 0)) {
                bool odd = false;
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) {
                    const uint32_t sees = (at.rows() & visible_rows(p, reach, reach.tile(v) * MK_TILE, token[hi], tree ? tree_smem[token[hi]] : 0)) >> (LANE_KEYS * g);
#pragma unroll
                    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const bool bad = !(fabsf(x[rb][hi][i]) < INFINITY);
                            if (sees >> (rb * BLOCK_KEYS + i) & 1u) {
                                if (bad) l_run[hi] = __uint_as_float(QUIET_NAN);
                            } else {
                                odd |= bad;
                                x[rb][hi][i] = -INFINITY;
                            }
                        }
                }
                if (__builtin_expect(__any(odd), 0)) {      // values (fp8: or scales) that are not finite, of keys that somebody does not see
                    for (int i = lane; i < TILE_B / 16; i += 64) {
                        LDS_AS u32x4* unit = (LDS_AS u32x4*)(tile + i * 16);
                        u32x4 w = *unit;
#pragma unroll
                        for (int d = 0; d < 4; ++d) w[d] = FP8 ? finite_codes(w[d]) : finite_halves(w[d]);
                        *unit = w;
                    }
                    if constexpr (FP8) {
#pragma unroll
                        for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                            for (int i = 0; i < 4; ++i) ksc[rb][i] = fabsf(ksc[rb][i]) < INFINITY ? ksc[rb][i] : 0.f;
                    }
                }
            } else {
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) l_run[hi] = with_least(l_run[hi], x[0][hi], x[1][hi]);
            }
            // ---- weights
#pragma unroll
            for (int hi = 0; hi < 2; ++hi)
#pragma unroll
                for (int rb = 0; rb < 2; ++rb) top[hi] = max_of(max_of(top[hi], x[rb][hi][0], x[rb][hi][1]), x[rb][hi][2], x[rb][hi][3]);
            if (unset) {                                    // the reference of a query row: the maximum of its first tile with a row that it sees
                bool left = false;
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) {
                    const float t = over_groups(top[hi]);   // (no tile before had one: the maximum so far is this tile's)
                    if (m_ref[hi] == -INFINITY && t != -INFINITY) m_ref[hi] = t * sc;
                    left |= m_ref[hi] == -INFINITY;
                }
                unset = __any(left);
            }
            bf16x8 pb[2];
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                const float m_use = m_ref[hi] == -INFINITY ? 0.f : m_ref[hi];
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float e0 = fast_exp2(fmaf(x[k >> 1][hi][2 * (k & 1)], sc, -m_use)), e1 = fast_exp2(fmaf(x[k >> 1][hi][2 * (k & 1) + 1], sc, -m_use));
                    l_run[hi] += e0 + e1;
                    if constexpr (FP8) {
                        e0 *= ksc[k >> 1][2 * (k & 1)];
                        e1 *= ksc[k >> 1][2 * (k & 1) + 1];
                    }
                    w[k] = pack_bf16x2(e0, e1);
                }
                pb[hi] = __builtin_bit_cast(bf16x8, (u32x4){w[0], w[1], w[2], w[3]});
            }
            // ---- values.  (bf16) The wavefront's next tile is asked for beside them, a block as soon as it is done with, the rope part's at the end.
            const bool more = !FP8 && v + 4 < v1;
            if (more) {
                const int i = (turn + 1) & 31;
                at = Place{(int)__builtin_amdgcn_readlane(ids, 2 * i), (int)__builtin_amdgcn_readlane(ids, 2 * i + 1)};
                if (i == 0) at = place_now(v + 4);
            }
            {
                s16x4 lo[NCT], up[NCT];
                u32x2 column[NCT];
                auto rt = [&](int ct) {
                    LDS_AS unsigned char* from = tile + t_base[ct & 3] + (ct >> 2) * (FP8 ? 64 : BLOCK_B);
                    if constexpr (FP8) {
                        column[ct] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((LDS_AS i32x2*)from));
                        return;
                    }
                    lo[ct] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)from);
                    up[ct] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(from + 16 * 128));
                };
                static constexpr int AHEAD = 4;
#pragma unroll
                for (int ct = 0; ct < AHEAD; ++ct) rt(ct);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int ct = 0; ct < NCT; ++ct) {
                    if (ct + AHEAD < NCT) rt(ct + AHEAD);
                    const bf16x8 va = FP8 ? widened(column[ct][0], column[ct][1])
                                          : __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo[ct], up[ct], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int hi = 0; hi < 2; ++hi) oacc[hi][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[hi], oacc[hi][ct], 0, 0, 0);
                    if (!FP8 && ct % 4 == 3 && more) {
                        __builtin_amdgcn_sched_barrier(0);              // (behind the wait for the block's last read)
                        request_block(at, ct / 4);
                        if (ct == NCT - 1) request_block(at, BLOCKS - 1);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            // (every read of the tile has been waited for: its place is free)
            if constexpr (FP8) {
                at = next;
                if (v + 8 < v1) {
                    const int i = (turn + 2) & 31;
                    next = Place{(int)__builtin_amdgcn_readlane(ids, 2 * i), (int)__builtin_amdgcn_readlane(ids, 2 * i + 1)};
                    if (i < 2) next = place_now(v + 8);     // (not looked up yet)
                    request(next, turn & 1);
                }
            }
        }
        if (pass == ACCUMULATE_AGAIN) break;
        if (pass == ACCUMULATE) {
            // (an infinite score makes a NaN of its row either way, and no other row shall be the worse for it)
            const bool jumped = (top[0] * sc > m_ref[0] + FAST_GAP && top[0] < INFINITY) || (top[1] * sc > m_ref[1] + FAST_GAP && top[1] < INFINITY);
            if (__builtin_expect(!__any(jumped), 1)) break;
            pass = MAXIMA;
            unset = false;
        } else {
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                const float t = over_groups(top[hi]);
                m_ref[hi] = t == -INFINITY ? t : t * sc;
            }
            pass = ACCUMULATE_AGAIN;
        }
        start();
    }

    // ---- the four wavefronts joined: each one's factor for every row, then the columns in two halves through the LDS
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
        float l = l_run[hi] + __shfl_xor(l_run[hi], 16);
        l += __shfl_xor(l, 32);
        if (g == 0) {
            m_smem[wave][hi * 16 + n] = m_ref[hi];
            l_smem[wave][hi * 16 + n] = l;
        }
    }
    __syncthreads();
    if (tid < 128) {
        const int w = tid >> 5, r = tid & 31;
        const float m = fmaxf(fmaxf(m_smem[0][r], m_smem[1][r]), fmaxf(m_smem[2][r], m_smem[3][r])), ref = m == -INFINITY ? 0.f : m;
        float l = 0.f, own = 0.f;
        for (int k = 0; k < 4; ++k) {
            const float lk = l_smem[k][r], mk = m_smem[k][r];
            const float e = lk == 0.f ? 0.f : mk == -INFINITY ? 1.f : fast_exp2(mk - ref);       // (-inf with a sum: a NaN)
            if (lk != 0.f) l += lk * e;
            if (k == w) own = e;
        }
        // (an infinite score makes the sum infinite where it is not its wavefront's reference: own / l would be 0 for every wavefront, and nothing is multiplied by that)
        if (!(l < INFINITY)) l = own = __uint_as_float(QUIET_NAN);
        f_smem[r][w] = l == 0.f ? 0.f : own / l;
        if (w == 0 && r < HL && p.lse_part) p.lse_part[part_of(r)] = l == 0.f ? -INFINITY : ref * LN2 + __builtin_amdgcn_logf(l) * LN2;
    }
    constexpr int RSO = D_C * 2 + 16;                   // bytes from row to row of half the columns in fp32 (padded)
    static_assert(32 * RSO <= PLACE_B, "exchange space must fit in a tile's place");
    constexpr int LPR = D_C / 8;                        // lanes of half a row, four columns each
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (half) __syncthreads();
#pragma unroll
        for (int hi = 0; hi < 2; ++hi)
#pragma unroll
            for (int ct = 0; ct < NCT / 2; ++ct) *(LDS_AS f32x4*)(mine + (hi * 16 + n) * RSO + (ct * 16 + g * 4) * 4) = oacc[hi][half * (NCT / 2) + ct];
        __syncthreads();
        constexpr int STEP = MF_THREADS / LPR, TURNS = 32 / STEP, BATCH = 4;      // rows at a time; (all reads of a batch on their way before any is used)
        const int c = tid % LPR;
#pragma unroll 1
        for (int k0 = 0; k0 < TURNS; k0 += BATCH) {
            f32x4 part[BATCH][4];
            float f[BATCH][4];
#pragma unroll
            for (int k = 0; k < BATCH; ++k)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int r = tid / LPR + (k0 + k) * STEP;
                    part[k][w] = *(LDS_AS f32x4*)(lds + w * PLACE_B + r * RSO + c * 16);
                    f[k][w] = f_smem[r][w];
                }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int r = tid / LPR + (k0 + k) * STEP;
                f32x4 o = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < 4; ++w)             // (what a wavefront without a row that counts has is nothing, not even times zero)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = fmaf(f[k][w], f[k][w] != 0.f ? part[k][w][i] : 0.f, o[i]);
                if (r >= HL) continue;
                const size_t to = part_of(r) * D_C + half * (D_C / 2) + c * 4;
                if (p.num_splits == 1)
                    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.o_part) + to) = (u32x2){pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
                else
                    *reinterpret_cast<f32x4*>(static_cast<float*>(p.o_part) + to) = o;
            }
        }
    }
}

}  // namespace

template <int D_C, bool FP8> static void launch(const MaskedParams& p, unsigned chunks, unsigned Z, int64_t tiles, hipStream_t s)
{
    const int64_t bytes = p.B * tiles * (MK_TILE * (D_C + 64) * (FP8 ? 1 : 2));
    if (Z == 1 && bytes >= 64 << 20) masked_thin_kernel<D_C, FP8, true><<<dim3(chunks), dim3(MF_THREADS), 0, s>>>(p);
    else masked_thin_kernel<D_C, FP8, false><<<dim3(chunks * Z), dim3(MF_THREADS), 0, s>>>(p);
}

hipError_t launch_masked_thin(const MaskedParams& p, mla_dtype cache, int64_t tiles, hipStream_t s)
{
    const unsigned chunks = ((unsigned)p.B * p.num_splits + 7) / 8 * 8, Z = (unsigned)((p.H + MK_THIN_ROWS - 1) / MK_THIN_ROWS);
    if (cache == MLA_BF16 && p.d_c == 512)      launch<512, false>(p, chunks, Z, tiles, s);
    else if (cache == MLA_BF16)                 launch<256, false>(p, chunks, Z, tiles, s);
    else if (p.d_c == 512)                      launch<512, true>(p, chunks, Z, tiles, s);
    else                                        launch<256, true>(p, chunks, Z, tiles, s);
    return hipGetLastError();
}

}  // namespace mla
