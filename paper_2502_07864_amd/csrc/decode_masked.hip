// Masked attention over the latent cache on the matrix cores (bf16 queries, bf16 or fp8 cache): 128 query rows per workgroup.
//
//   S^T [keys x rows]  = K [keys x (d_c + 64)] . Q^T [(d_c + 64) x rows]
//   O^T [d_c x rows]  += V^T [d_c x keys] . P^T [keys x rows],      V = the first d_c columns of K
//
// A wavefront owns 32 query rows (two groups of 16), their queries in registers for as long as it lives, their whole outputs
// (d_c x 32 fp32 values) and a softmax of its own: no exchange of scores or weights, one workgroup barrier per tile of 32 keys.
// Both contractions run on v_mfma_f32_16x16x32_bf16 with every LDS read feeding two of them.  The second one needs the tile
// transposed: each wavefront transposes a quarter of the columns (transposing LDS reads, one 16-byte write per lane and 16
// columns) for all four, so that the values are read in plain 128-bit reads.  Transposing reads by everybody would be
// 64 x 26 cycles of LDS issue a tile and wavefront beside the 36 x 17 of the scores, more than the 2176 cycles of matrix
// instructions; so it is 68 x 17 + 16 x 26 + 8 x 17 = 1708.
//
// A step scores tile i + 1 (and weighs tile i between its matrix instructions), then accumulates tile i (and transposes tile
// i + 1), while tile i + 2 is on its way (direct-to-LDS loads).  Two slots for tiles and two for their transposes, and the queries' last k-steps, which the registers do
// not hold: 153 KB (fp8: 152) of the CU's 160 KB of LDS at d_c = 512, one workgroup per CU; at d_c = 256 a step is two tiles, 145 and 127 KB.  A bf16 tile waits for all
// loads at once; an fp8 one is half as wide, so that three slots fit and two are on their way, waited for by count.
//
// fp8 codes stay in LDS as they are and are widened to bf16, which is exact, where they are read: the keys beside the matrix instructions of the
// 32 dimensions before, the values once, when their tile is transposed.  The row's scale goes to the scores and the weights.  (Widened on the way into LDS, through
// registers, 31 tokens x 32 heads on 4 x 131072 rows took 1678 us.)
//
// Measured (whole calls of a running server; the first dozen are some 10 % slower): that case 1068 us, 1.06 PFLOP/s; 16 x 32 on 16 x 8192 bf16 rows 162 us, 0.90; 63 x 28 on
// 64 sequences of 512 .. 4096 rows at d_c = 256 361 us, 0.73; a large library product reaches 1.35.  Bound by the one wavefront per SIMD that the registers leave: matrix pipes busy 30 to
// 44 % of the cycles, the wavefronts issue 50 to 61 % of theirs, and wait for tiles, LDS and barriers 21 to 25 %.  What had most weight on the way: no
// spilled register may be read back in the loop, since the wait for it is a wait for the tiles requested before it.  Not
// taken, for they were slower: two steps unrolled (the sums move between register files), more keys read ahead, the scores' maximum beside the value products in the bf16 forms.
//
// The reference of a query row's exponentials is the maximum of the first tile with a row it sees, and nothing is rescaled; where a
// score exceeds it by more than 2^64 the chunk is done again against the exact maxima.  The normaliser sums the weights before
// their rounding to bf16 in fp32; the weights' rounding (2^-8 of each) is the price of the bf16 instructions.  Chunks' results stay in fp32.
//
// Keys that a row does not see get the score -inf, in the tiles that need it.  A key that is not finite has scores that are not: where
// a wavefront meets one that some row of its own does not see, it clears what is not finite from the transposed tile before
// it multiplies (0 times infinity would be a NaN).  The rows that do see the key end as NaN, whichever tile it lies in and whichever way its score
// goes: their sums become one, and results, log-sum-exps and merged chunks follow from those.
#include "masked_tile.h"
#include <type_traits>

namespace mla {
namespace {

typedef __attribute__((ext_vector_type(2))) int i32x2;

constexpr int MT_ROWS = MK_TALL_ROWS;        // query rows per workgroup

template <int D_C, bool FP8>
__global__ __launch_bounds__(MF_THREADS, 1) void masked_tall_kernel(MaskedParams p)
{
    constexpr int ROW = D_C + 64, ROWB = FP8 ? ROW : ROW * 2;
    constexpr int CPR = ROWB / 16;                      // 16-byte chunks per row (bf16: 72 / 40, fp8: 36 / 20)
    constexpr int TILE_B = MK_TILE * ROWB;
    constexpr int NT = D_C == 512 ? 1 : 2;              // tiles of a step (as many as fit twice into the LDS, with their transposes)
    constexpr int NRB = 2 * NT;                         // and their blocks of 16 keys
    constexpr int RING = FP8 ? 3 : 2;                   // places for a step's tiles
    constexpr int NLOAD = TILE_B / (MF_THREADS * 16);   // (bf16) 16-byte loads per thread and tile (9 / 5)
    constexpr int FLOAD = 8 * ROWB / 1024;              // (fp8) loads of 1 KB for eight rows of a tile (4 / 2), and one of half as much
    constexpr int NKS = ROW / 32;                       // k-steps of the scores (18 / 10)
    constexpr int NCT = D_C / 16;                       // column tiles of the values (32 / 16)
    constexpr int VT_B = D_C * MK_TILE * 2;             // a transposed tile
    constexpr int NQ = D_C == 256 ? NKS : FP8 ? NKS - 4 : NKS - 2;      // k-steps whose queries stay in registers; the last ones' don't fit, and lie in LDS

    constexpr int VT_AT = RING * NT * TILE_B;           // the transposes lie behind the tiles, the queries' rope parts behind them
    __shared__ __attribute__((aligned(1024))) unsigned char smem[VT_AT + 2 * NT * VT_B + (NKS - NQ) * 2 * MF_THREADS * 16];
    __shared__ __attribute__((aligned(16))) float ks_smem[FP8 ? RING : 1][NT * 2][32];     // (fp8) scales of a step's rows, the 16 of a half tile twice
    __shared__ uint64_t tree_smem[64];
    __shared__ int token_smem[MT_ROWS];
    static_assert(sizeof(smem) + sizeof(ks_smem) + sizeof(tree_smem) + sizeof(token_smem) <= 160 * 1024, "LDS of a CU");
    LDS_AS unsigned char* lds = (LDS_AS unsigned char*)smem;
    LDS_AS float* ks_lds = (LDS_AS float*)ks_smem;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 15, g = lane >> 4;

    // the groups of query rows of one chunk get linear ids 8 apart: same XCD, same time, so all but the first find the rows in its L2
    const int Z = (p.H + MT_ROWS - 1) / MT_ROWS;
    const int id = blockIdx.x, rr = id >> 3;
    const int zi = (int)((unsigned)rr % (unsigned)Z), wg = chunk_at((rr - zi) / Z, id & 7);
    if (wg >= p.B * p.num_splits) return;               // padding of the last group of 8
    const int split = (int)((unsigned)wg % (unsigned)p.num_splits), b = sequence_at(p, (int)((unsigned)wg / (unsigned)p.num_splits), lane);
    const int hb = zi * MT_ROWS, HL = min(MT_ROWS, p.H - hb);

    const bool tree = p.tree != nullptr;
    const int32_t len = ((const CONST_AS int32_t*)p.lens)[b];
    const Reach reach = reach_of(len, p.q_len, p.max_pages * p.page_size, tree, p.window, p.sinks);
    const int v0 = chunk_start(reach.tiles, split, p.num_splits), v1 = chunk_start(reach.tiles, split + 1, p.num_splits);

    const int nrow = min(32, HL - wave * 32);           // this wavefront's query rows (may be none: it still loads and transposes)
    auto part_of = [&](int r) { return part_index(b, hb + wave * 32 + r, split, p.H, p.num_splits); };
    if (v0 >= v1) {                                     // nothing to see
        for (int r = 0; r < nrow; ++r) {
            if (p.num_splits == 1)
                for (int c = lane * 8; c < D_C; c += 512)
                    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.o_part) + part_of(r) * D_C + c) = (u32x4){0u, 0u, 0u, 0u};
            if (lane == 0 && p.lse_part) p.lse_part[part_of(r)] = -INFINITY;
        }
        return;
    }

    // ---- tiles: v is a tile's number without the gap.  Where their halves lie, 32 tiles at a time, a lane each (a scalar load on every step,
    // out of order with the LDS reads, would make each of their waits a wait for everything).
    const int32_t* const ptab = p.page_table + (size_t)b * p.max_pages;
    const int per_page = p.page_size / 16;
    auto half_of = [&](int v) { return 2 * reach.tile(min(v + (lane >> 1), v1 - 1)) + (lane & 1); };
    auto pages_from = [&](int v) { return half_page(p, ptab, per_page, half_of(v)); };
    int32_t ids = 0, pages = 0;                         // the places of tiles v0 + 32 k on, and the page ids of the 32 behind them, looked at no
                                                        // sooner than they are needed (who waits for them waits for tiles)
    auto tile_at = [&](int v) -> Place {                // (v: in the order of the sweep)
        const int i = (v - v0) & 31;
        if (i == 0) {
            ids = half_at(p, pages, per_page, half_of(v));
            pages = pages_from(v + 32);
        }
        return Place{(int)__builtin_amdgcn_readlane(ids, 2 * i), (int)__builtin_amdgcn_readlane(ids, 2 * i + 1)};
    };
    auto tile_now = [&](int v) { return tile_place(p, (const CONST_AS int32_t*)ptab, per_page, reach.tile(v)); };      // (the first ones: scalar loads, which wait for no vector load)

    const uint32_t lds_base = (uint32_t)(uintptr_t)lds;
    // A wavefront loads eight rows of a tile, which lie one behind the other as they do in the pool, 64 pieces at a time; chunk c of row r at
    // position c ^ key(r).
    auto mine_of = [&](const Place& s) { return wave < 2 ? s.lo : s.hi; };
    // tile t of step u -> its place in slot u % RING
    auto request = [&](const Place& s, int u, auto tile_tag) {
        constexpr int t = decltype(tile_tag)::value;
        const int at = mine_of(s);
        if (at < 0) return;                             // a page outside the pool is never dereferenced
        const int l = lane_again();
        const unsigned char* src = static_cast<const unsigned char*>(p.kv) + (size_t)at * (TILE_B / 2) + (wave & 1) * (8 * ROWB);
        const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_base + (uint32_t)((u & 1) * (NT * TILE_B) + t * TILE_B + wave * (8 * ROWB)));
#pragma unroll
        for (int k = 0; k < NLOAD; ++k) {
            const uint32_t off = ((uint32_t)l * 16) ^ piece_key<CPR>(k, l);
            asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                         :: "s"(dst), "v"(off), "s"(src + k * 1024), "i"(k * 1024) : "memory", "scc");
        }
    };
    // Tiles of a step
    struct Places { Place at[NT]; };
    auto there = [&](const Places& s) {                 // which of their halves are, a bit each
        uint32_t bits = 0;
#pragma unroll
        for (int t = 0; t < NT; ++t) bits |= (uint32_t)(s.at[t].lo >= 0) << 2 * t | (uint32_t)(s.at[t].hi >= 0) << (2 * t + 1);
        return bits;
    };
    auto places = [&](int u, auto at) {
        Places s;
#pragma unroll
        for (int t = 0; t < NT; ++t) s.at[t] = v0 + NT * u + t < v1 ? at(v0 + NT * u + t) : Place{-1, -1};
        return s;
    };
    // (fp8) Codes as they are, chunk c of row r at position c ^ (r >> 2 & 2), which is one key for a wavefront's rows.  Every wavefront makes the same number of
    // loads on every step, so that they can be waited for by count: tiles that are not there are some tile, which nobody sees.
    constexpr int PER_STEP = NT * (FLOAD + 2);
    auto request_codes = [&](const Places& s, int u) {
        const int l = lane_again();
        const uint32_t slot = (uint32_t)u % RING, off = (uint32_t)(l * 16) ^ (uint32_t)((wave & 1) << 5);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const unsigned char* src = static_cast<const unsigned char*>(p.kv) + (size_t)max(mine_of(s.at[t]), 0) * (TILE_B / 2) + (wave & 1) * (8 * ROWB);
            const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_base + slot * (NT * TILE_B) + (uint32_t)(t * TILE_B + wave * (8 * ROWB)));
#pragma unroll
            for (int k = 0; k < FLOAD; ++k)
                asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                             :: "s"(dst), "v"(off), "s"(src + k * 1024), "i"(k * 1024) : "memory", "scc");
            // the last half of a load's bytes, and the half tile's scales (both its wavefronts bring them)
            const float* scales = p.kv_scale + (size_t)max(mine_of(s.at[t]), 0) * 16;
            const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)ks_lds + (slot * NT + (uint32_t)t) * 256u + (uint32_t)(wave >> 1) * 128u);
            if (l < 32)
                asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\t"
                             "s_mov_b32 m0, %4\n\ts_nop 0\n\tglobal_load_lds_dword %5, %6"
                             :: "s"(dst), "v"(off), "s"(src + FLOAD * 1024), "i"(FLOAD * 1024), "s"(to), "v"((uint32_t)((l & 15) * 4)), "s"(scales) : "memory", "scc");
        }
    };
    auto request_all = [&](const Places& s, int u) {
        if constexpr (FP8) {
            request_codes(s, u);
        } else {
            request(s.at[0], u, std::integral_constant<int, 0>{});
            if constexpr (NT > 1) request(s.at[1], u, std::integral_constant<int, NT - 1>{});
        }
    };
    // the tiles of the step after this one are there, (fp8) those of the one after that may be on their way
    auto wait_for_step = [&]() {
        if constexpr (FP8) {
            wait_vmcnt<PER_STEP>();
        } else {
            wait_vmcnt<0>();
        }
    };
    const int steps = (v1 - v0 + NT - 1) / NT;
    uint32_t here, next, after = 0;                     // what is there of this step's tiles, the next one's, the one's after it (fp8)
    Places second;
    auto start = [&]() {
        const Places first = places(0, tile_now);
        second = places(1, tile_now);
        here = there(first);
        next = there(second);
        request_all(first, 0);
        if constexpr (FP8) {
            request_all(second, 1);
            const Places third = places(2, tile_now);
            after = there(third);
            request_all(third, 2);
        }
        ids = half_at(p, pages_from(v0), per_page, half_of(v0));
        pages = pages_from(v0 + 32);
    };
    start();

    // ---- this wavefront's query rows -> registers (B operands of the scores).  A negative scale changes their sign: the largest score is
    // then the largest scaled one
    bf16x8 qreg[2][NQ];
    LDS_AS unsigned char* const q_lds = lds + VT_AT + 2 * NT * VT_B + wave * ((NKS - NQ) * 2 * 1024) + lane * 16;      // this lane's, written and read by it alone
    {
        const uint16_t* qa = static_cast<const uint16_t*>(p.q_abs) + (size_t)b * p.H * D_C;
        const uint16_t* qr = static_cast<const uint16_t*>(p.q_rope) + (size_t)b * p.H * 64;
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            const size_t row = hb + min(wave * 32 + hi * 16 + n, HL - 1);
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) {
                // (fp8: a lane reads 16 codes at a time, eight for each of two k-steps)
                const int kl = ks < D_C / 32 ? ks : ks - D_C / 32, col = FP8 ? (kl >> 1) * 64 + g * 16 + (kl & 1) * 8 : kl * 32 + g * 8;
                const u32x4 v = ks < D_C / 32 ? *reinterpret_cast<const u32x4*>(qa + row * D_C + col) : *reinterpret_cast<const u32x4*>(qr + row * 64 + col);
                if (ks < NQ) qreg[hi][ks] = __builtin_bit_cast(bf16x8, v);
                else         *(LDS_AS u32x4*)(q_lds + ((ks - NQ) * 2 + hi) * 1024) = v;
            }
        }
        if (p.scale < 0.f) {
            asm volatile("");                           // (a branch, not 144 instructions for everybody)
            const u32x4 sign = (u32x4){0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
#pragma unroll
            for (int hi = 0; hi < 2; ++hi)
#pragma unroll
                for (int ks = 0; ks < NKS; ++ks) {
                    if (ks < NQ) qreg[hi][ks] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, qreg[hi][ks]) ^ sign);
                    else         *(LDS_AS u32x4*)(q_lds + ((ks - NQ) * 2 + hi) * 1024) ^= sign;
                }
        }
    }
    if (tree && tid < p.q_len) tree_smem[tid] = tree_word(p, b, tid);
    if (tid < MT_ROWS) token_smem[tid] = (hb + min(tid, HL - 1)) / p.heads;        // (both are read in few tiles)
    WholeTiles whole = whole_tiles(p, reach, hb / p.heads, (hb + HL - 1) / p.heads);
    auto seen_whole = [&](int v, uint32_t halves) { return halves == 3 && whole.holds(v); };      // (halves: the tile's bits)

    // ---- per-lane state: this lane's queries = column n of the D tiles of the two groups
    float m_ref[2] = {-INFINITY, -INFINITY};   // reference of the exponentials (log2 units)
    float l_run[2] = {0.f, 0.f};               // this lane's share of the normaliser
    f32x4 oacc[2][NCT];
    // (never zero: a masked score is -inf and has to stay it)
    const float sc = fmaxf(fabsf(p.scale) * LOG2E, 1.17549435e-38f);

    // Keys: in bf16 tiles row i of a block rb of 16 scores is key 16 rb + i, so that a lane ends with keys 4g .. 4g + 3 and 16 on, as two
    // transposing reads of 16-bit values give them; in fp8 tiles key 8 (i / 4) + 4 rb + i % 4, keys 8g .. 8g + 7, as one of 8-bit values does.
    constexpr int LANE_KEYS = FP8 ? 8 : 4, BLOCK_KEYS = FP8 ? 4 : 16;         // key LANE_KEYS g + BLOCK_KEYS rb + i
    // score A operand: chunk 4 ks + g (fp8: 4 (ks / 2) + g)
    uint32_t a_base[2], t_base[4];
    if constexpr (FP8) {
        const int row = 8 * (n >> 2) + (n & 3);
        a_base[0] = a_base[1] = (uint32_t)(row * ROWB) + (((uint32_t)g ^ (uint32_t)(row >> 2 & 2)) << 4);
        // transposing reads: the lane supplies row 8g + n / 2, 8 bytes at column 16 ct + 8 (n % 2)
        const int from = 8 * g + (n >> 1);
#pragma unroll
        for (int e = 0; e < 4; ++e) t_base[e] = (uint32_t)(from * ROWB) + (((uint32_t)e ^ (uint32_t)(from >> 2 & 2)) << 4) + (uint32_t)((n & 1) * 8);
    } else {
#pragma unroll
        for (int e = 0; e < 2; ++e) a_base[e] = (uint32_t)(n * ROWB) + ((((uint32_t)(4 * e + g)) ^ (uint32_t)swz_key(n)) << 4);
        // transposing reads: the lane supplies tile row 4g + (n >> 2) (and 16 more), 8 bytes at column 16 ct + 4 (n & 3)
        const int from = g * 4 + (n >> 2);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            t_base[e] = (uint32_t)(from * ROWB) + ((((uint32_t)(2 * e) + (uint32_t)((n & 3) >> 1)) ^ (uint32_t)swz_key(from)) << 4) + (uint32_t)((n & 1) * 8);
    }
    LDS_AS unsigned char* const vt = lds + VT_AT;

    typedef f32x4 Scores[NRB][2];              // [block of 16 keys][query group]: the lane's keys of query n
    f32x4 ksc[NRB];                            // (fp8) scales of this lane's keys
    bool dirty[NT] = {};                       // one that some query of the wavefront does not see was not, in tile t of the step

    // rows of tile v (bit: row) that the lane's query of group hi sees
    auto visible = [&](int v, uint32_t halves, int hi) -> uint32_t {
        const int token = token_smem[wave * 32 + hi * 16 + (lane_again() & 15)];
        return ((halves & 1 ? 0xFFFFu : 0u) | (halves & 2 ? 0xFFFF0000u : 0u)) & visible_rows(p, reach, reach.tile(v) * MK_TILE, token, tree ? tree_smem[token] : 0);
    };
    // tile t of the step (tile v of the sequence)
    auto mask = [&](Scores& x, int t, int v, uint32_t halves) {
        bool odd = false;
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            const uint32_t sees = visible(v, halves, hi) >> (LANE_KEYS * g);
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool bad = !(fabsf(x[2 * t + rb][hi][i]) < INFINITY);
                    if (sees >> (rb * BLOCK_KEYS + i) & 1u) {
                        if (bad) l_run[hi] = __uint_as_float(QUIET_NAN);
                    } else {
                        odd |= bad;
                        x[2 * t + rb][hi][i] = -INFINITY;
                    }
                }
        }
        dirty[t] = __any(odd);
        if (FP8 && dirty[t]) {                 // (nothing is multiplied with a scale that is not finite)
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int i = 0; i < 4; ++i) ksc[2 * t + rb][i] = fabsf(ksc[2 * t + rb][i]) < INFINITY ? ksc[2 * t + rb][i] : 0.f;
        }
    };
    // (every wavefront that has to does this for itself: it does not matter who comes first)
    auto clean = [&](LDS_AS unsigned char* tile) {
        for (int i = lane; i < VT_B / 16; i += 64) {
            LDS_AS u32x4* unit = (LDS_AS u32x4*)(tile + i * 16);
            u32x4 w = *unit;
#pragma unroll
            for (int d = 0; d < 4; ++d) w[d] = finite_halves(w[d]);
            *unit = w;
        }
    };
    float top[2] = {-INFINITY, -INFINITY};     // largest score of the sweep so far, this lane's keys (unscaled)
    auto raise_top = [&](const Scores& x) {
#pragma unroll
        for (int hi = 0; hi < 2; ++hi)
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) top[hi] = max_of(max_of(top[hi], x[rb][hi][0], x[rb][hi][1]), x[rb][hi][2], x[rb][hi][3]);
    };
    // the reference of a query row: the maximum of its first tile with a row that it sees
    bool unset = true;
    auto set_reference = [&](const Scores& x) {
        bool left = false;
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            float tm = -INFINITY;
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) tm = max_of(max_of(tm, x[rb][hi][0], x[rb][hi][1]), x[rb][hi][2], x[rb][hi][3]);
            tm = over_groups(tm);
            if (m_ref[hi] == -INFINITY) m_ref[hi] = tm == -INFINITY ? tm : tm * sc;
            left |= m_ref[hi] == -INFINITY;
        }
        unset = __any(left);
    };
    // scores of step u, just made: masked.  (fp8: scaled, and their maximum taken as if all were seen, beside the products with the values.
    // 4 sequences of 128k: 1127 us with both here, 1103; in the bf16 forms it costs the registers that keep the queries.)
    float glanced[2];                          // (fp8)
    // A row that is not finite has no score that is, whatever the query (zero times infinity is a NaN); so one query group of one wavefront, another one every
    // step, meets it for everybody, and then the sweep is done again with every tile masked, which looks at all scores.  (Every wavefront on every step, as the
    // kernel for few rows does it: 3 - 4 % of a call; so it is 0 at d_c = 512, 2 % at 256.)
    float odd = 0.f;                           // not zero any more if a score of a step that everybody sees whole was not finite
    bool some = false;                         // a step that everybody sees whole was there
    auto look_at = [&](Scores& x, int u, uint32_t bits) {
        bool whole_step = true;
#pragma unroll
        for (int t = 0; t < NT; ++t) whole_step &= seen_whole(v0 + NT * u + t, bits >> 2 * t & 3);
        if (__builtin_expect(whole_step, 1)) {
            some = true;
            if constexpr (FP8) {
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) top[hi] = fmaxf(top[hi], glanced[hi]);
            }
            if ((u & 3) == wave) {
                float o[2] = {odd, 0.f};
#pragma unroll
                for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[rb & 1] = fmaf(x[rb][0][i], 0.f, o[rb & 1]);
                odd = o[0] + o[1];
            }
        } else {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (!seen_whole(v0 + NT * u + t, bits >> 2 * t & 3)) {
                    mask(x, t, v0 + NT * u + t, bits >> 2 * t & 3);
                    continue;
                }
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) l_run[hi] = with_least(l_run[hi], x[2 * t][hi], x[2 * t + 1][hi]);
            }
        }
        if (!FP8 || !whole_step) raise_top(x);
        if (unset) set_reference(x);
    };

    // ---- a step: S^T of the tiles in `keys` and the weights of those before from their scores x (PV); then their values from `values`,
    // and the transposes of the former tiles into `to`
    auto step = [&](auto pv_tag, LDS_AS unsigned char* keys, LDS_AS float* scales, LDS_AS unsigned char* values, LDS_AS unsigned char* to, const Scores& x, Scores& y) {
        constexpr bool PV = decltype(pv_tag)::value;
        static constexpr int AHEAD = NT == 1 ? 4 : 2;     // k-steps that the key reads run ahead, one wavefront per SIMD with nothing else to hide them
        static constexpr int VAHEAD = FP8 && NT == 1 ? 6 : 4;   // column tiles that the value reads do (4 x 128k: 1062 us with 4, 1051)
        static constexpr int SHARE = NT * NCT / 4;        // column tiles that this wavefront transposes (8)
        bf16x8 ka[NRB][NKS], va[NT][NCT];
        u32x4 raw[NRB][NKS / 2];               // (fp8) the codes of two k-steps
        float m_use[2];
        uint32_t w[2][4 * NT];
        auto key_of = [&](int rb, int ks) -> bf16x8 {
            if constexpr (FP8) return widened(raw[rb][ks / 2][ks % 2 * 2], raw[rb][ks / 2][ks % 2 * 2 + 1]);
            else               return ka[rb][ks];
        };
        auto rk = [&](int ks) {
            if constexpr (FP8) {
                if (ks % 2 == 0) {
#pragma unroll
                    for (int rb = 0; rb < NRB; ++rb)
                        raw[rb][ks / 2] = *(LDS_AS u32x4*)(keys + a_base[0] + ks / 2 * 64 + (rb >> 1) * TILE_B + (rb & 1) * 4 * ROWB);
                }
                return;
            }
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) ka[rb][ks] = *(LDS_AS bf16x8*)(keys + a_base[ks & 1] + (ks >> 1) * 128 + rb * 16 * ROWB);
        };
        bf16x8 kk[2][NRB];
        bf16x8 qa[NKS - NQ + 1][2];            // (one more: an array may not be empty)
        auto rq = [&](int ks) {
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) qa[ks - NQ][hi] = *(LDS_AS bf16x8*)(q_lds + ((ks - NQ) * 2 + hi) * 1024);
        };
        auto rv = [&](int ct) {
#pragma unroll
            for (int t = 0; t < NT; ++t) va[t][ct] = *(LDS_AS bf16x8*)(values + t * VT_B + ct * 1024 + lane * 16);
        };
        auto weigh = [&](int j) {              // pair j of 8 NT: query group j / (4 NT), keys 2 (j % (4 NT)) and the one after
            const int hi = j / (4 * NT), k = j % (4 * NT), rb = k >> 1, i = 2 * (k & 1);
            float e0 = fast_exp2(fmaf(x[rb][hi][i], sc, -m_use[hi])), e1 = fast_exp2(fmaf(x[rb][hi][i + 1], sc, -m_use[hi]));
            l_run[hi] += e0 + e1;
            if constexpr (FP8) { e0 *= ksc[rb][i]; e1 *= ksc[rb][i + 1]; }
            w[hi][k] = pack_bf16x2(e0, e1);
        };
        s16x4 lo[SHARE], up[SHARE];
        u32x2 column[SHARE];
        auto rt = [&](int k) {                 // column tile wave * NCT / 4 + k of a tile, the next tile's behind them
            LDS_AS unsigned char* at = keys + (k / (NCT / 4)) * TILE_B + t_base[k & 3] + ((wave * (NCT / 4) + k % (NCT / 4)) >> 2) * (FP8 ? 64 : 128);
            if constexpr (FP8) {
                column[k] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((LDS_AS i32x2*)at));
                return;
            }
            lo[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)at);
            up[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(at + 16 * ROWB));
        };
        auto wt = [&](int k) {
            const bf16x8 v = FP8 ? widened(column[k][0], column[k][1]) : __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo[k], up[k], 0, 1, 2, 3, 4, 5, 6, 7));
            *(LDS_AS bf16x8*)(to + (k / (NCT / 4)) * VT_B + (wave * (NCT / 4) + k % (NCT / 4)) * 1024 + lane * 16) = v;
        };
        auto glance = [&](int k) {             // block k / 2 of the scores just made, query group k % 2: scaled (fp8), and their maximum
            const int rb = k >> 1, hi = k & 1;
            y[rb][hi] *= ksc[rb];
            if (rb == 0) glanced[hi] = max_of(max_of(y[rb][hi][0], y[rb][hi][0], y[rb][hi][1]), y[rb][hi][2], y[rb][hi][3]);
            else         glanced[hi] = max_of(max_of(glanced[hi], y[rb][hi][0], y[rb][hi][1]), y[rb][hi][2], y[rb][hi][3]);
        };
        if constexpr (PV) {
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) m_use[hi] = m_ref[hi] == -INFINITY ? 0.f : m_ref[hi];
        }
#pragma unroll
        for (int ks = 0; ks < AHEAD; ++ks) rk(ks);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
            if (ks + AHEAD < NKS) rk(ks + AHEAD);
            if (NQ < NKS && ks + 2 >= NQ && ks + 2 < NKS) rq(ks + 2);
            if (PV && ks + AHEAD >= NKS) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (2 * (ks + AHEAD - NKS) + i < VAHEAD) rv(2 * (ks + AHEAD - NKS) + i);
            }
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) {
                kk[ks & 1][rb] = FP8 && ks ? kk[ks & 1][rb] : key_of(rb, ks);
                if (FP8 && ks + 1 < NKS) kk[~ks & 1][rb] = key_of(rb, ks + 1);      // (widened beside the matrix instructions before)
            }
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                for (int hi = 0; hi < 2; ++hi)
                    y[rb][hi] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk[ks & 1][rb], ks < NQ ? qreg[hi][ks < NQ ? ks : 0] : qa[ks < NQ ? 0 : ks - NQ][hi],
                                                                        ks == 0 ? (f32x4){0.f, 0.f, 0.f, 0.f} : y[rb][hi], 0, 0, 0);
            if constexpr (PV) {
                if (NT == 2 && ks < 8) {
                    weigh(2 * ks);
                    weigh(2 * ks + 1);
                }
                if (NT == 1 && ks < 16 && ks % 2 == 0) weigh(ks / 2);
#pragma unroll
                for (int i = 0; i < 2 * NRB; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);   // an LDS read
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);     // a matrix instruction
                    __builtin_amdgcn_sched_group_barrier(0x2, FP8 ? 4 : 3, 0);     // vector instructions in its shadow
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        bf16x8 pb[NT][2];
        if constexpr (FP8) {                   // (the weights have theirs)
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) ksc[rb] = *(LDS_AS f32x4*)(scales + (rb >> 1) * 64 + (g >> 1) * 32 + (g & 1) * 8 + (rb & 1) * 4);
        }
        if constexpr (PV) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) pb[t][hi] = __builtin_bit_cast(bf16x8, (u32x4){w[hi][4 * t], w[hi][4 * t + 1], w[hi][4 * t + 2], w[hi][4 * t + 3]});
        }
        constexpr int EVERY = NCT / SHARE;     // a column tile is transposed beside so many (4 / 2)
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) {
            if (PV && ct + VAHEAD < NCT) rv(ct + VAHEAD);
            if (ct % EVERY == 0) rt(ct / EVERY);
            if (ct >= EVERY + EVERY / 2 && (ct - EVERY / 2) % EVERY == 0) wt((ct - EVERY / 2) / EVERY - 1);
            if (FP8 && ct >= NCT / 2 && ct < NCT / 2 + 2 * NRB) glance(ct - NCT / 2);
            if constexpr (PV) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int hi = 0; hi < 2; ++hi) oacc[hi][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[t][ct], pb[t][hi], oacc[hi][ct], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        wt(SHARE - 1);
    };
    using Yes = std::true_type;
    using No = std::false_type;

    // ---- sweeps over the tiles.  ACCUMULATE against the references (set on the way where they are not yet); if some score exceeded its
    // reference by more than FAST_GAP (rare), a sweep for the exact maxima (it accumulates too, which is not used) and the
    // accumulation again against them; if one was not finite (rare), the accumulation again.
    enum { ACCUMULATE, MAXIMA, ACCUMULATE_AGAIN };
    auto slot = [&](int u) { return lds + (int)((unsigned)u % RING) * (NT * TILE_B); };
    auto scales_of = [&](int u) { return ks_lds + (FP8 ? (int)((unsigned)u % RING) * (NT * 64) : 0); };
    auto turned = [&](int u) { return vt + (u & 1) * (NT * VT_B); };
    for (int pass = ACCUMULATE;;) {
        Scores x, y;
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            l_run[hi] = 0.f;
            top[hi] = -INFINITY;
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) oacc[hi][ct] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
        // bf16: step 0 is there, step 1 is asked for; fp8: steps 0 to 2 are
        wait_vmcnt<0>();
        __syncthreads();
        if constexpr (!FP8) request_all(second, 1);
        step(No{}, slot(0), scales_of(0), turned(0), turned(0), x, x);
        look_at(x, 0, here);
        for (int u = 0; u < steps; ++u) {
            const Places wanted = places(u + (FP8 ? 3 : 2), tile_at);
            if constexpr (FP8) {
                if (u) wait_for_step();
            } else {
                wait_for_step();
            }
            __syncthreads();     // the tiles of step u + 1 and the transposes of those of step u are there; everybody is done with what lay before
            request_all(wanted, u + (FP8 ? 3 : 2));
            const uint32_t last = there(wanted);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < NT; ++t)
                if (__builtin_expect(dirty[t], 0)) {
                    clean(turned(u) + t * VT_B);
                    dirty[t] = false;
                }
            step(Yes{}, slot(u + 1), scales_of(u + 1), turned(u), turned(u + 1), x, y);
            if (u + 1 < steps) look_at(y, u + 1, next);
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) x[rb][hi] = y[rb][hi];
            next = FP8 ? after : last;
            after = last;
        }
        if (pass == ACCUMULATE_AGAIN) break;
        if (pass == ACCUMULATE) {
            // (an infinite score makes a NaN of its row either way, and no other row shall be the worse for it)
            const bool jumped = (top[0] * sc > m_ref[0] + FAST_GAP && top[0] < INFINITY) || (top[1] * sc > m_ref[1] + FAST_GAP && top[1] < INFINITY);
            wait_vmcnt<0>();     // (fp8: nothing is on its way to the places that are asked for again)
            const bool strange = !(odd == 0.f);
            if (__builtin_expect(!__syncthreads_or(jumped || strange), 1)) break;
            if (__syncthreads_or(strange)) whole = WholeTiles{0, 0, 0};
            pass = __syncthreads_or(jumped) ? MAXIMA : ACCUMULATE_AGAIN;      // (against the same references: no bit changes)
            unset = false;
        } else {
            wait_vmcnt<0>();
            __syncthreads();
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                const float tm = over_groups(top[hi]);
                m_ref[hi] = tm == -INFINITY ? tm : tm * sc;
            }
            pass = ACCUMULATE_AGAIN;
        }
        start();
    }
    wait_vmcnt<0>();             // (fp8: what was asked for beyond the last step)
    __syncthreads();             // everybody is done with the tiles

    // ---- normalise, and transpose through LDS (a lane holds 4 consecutive columns of its query per column tile) for whole rows.
    // fp32 partials go in two halves of the columns, which the space takes.
    float lt[2], inv[2];
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
        float l = l_run[hi] + __shfl_xor(l_run[hi], 16);
        lt[hi] = l + __shfl_xor(l, 32);
        // (an infinite query whose scores are all -inf: a sum of zero, though there are rows that it sees)
        if (!(lt[hi] < INFINITY) || (some && lt[hi] == 0.f)) lt[hi] = __uint_as_float(QUIET_NAN);
        inv[hi] = lt[hi] == 0.f ? 0.f : 1.f / lt[hi];
    }
    constexpr int RSO = D_C * 2 + 32;           // row stride of the transposed block (padded)
    static_assert(4 * 32 * RSO <= sizeof(smem), "exchange space must fit");
    LDS_AS unsigned char* mine = lds + wave * (32 * RSO);
    if (p.num_splits == 1) {
#pragma unroll
        for (int hi = 0; hi < 2; ++hi)
#pragma unroll
            for (int ct = 0; ct < NCT; ++ct) {
                const f32x4 o = oacc[hi][ct] * inv[hi];
                *(LDS_AS u32x2*)(mine + (hi * 16 + n) * RSO + (ct * 16 + g * 4) * 2) = (u32x2){pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
            }
        constexpr int LPR = D_C / 8;            // lanes of a row (64 / 32)
        for (int r = lane / LPR; r < nrow; r += 64 / LPR) {
            const int c = lane % LPR;
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.o_part) + part_of(r) * D_C + c * 8) = *(LDS_AS u32x4*)(mine + r * RSO + c * 16);
        }
    } else {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int hi = 0; hi < 2; ++hi)
#pragma unroll
                for (int ct = 0; ct < NCT / 2; ++ct)
                    *(LDS_AS f32x4*)(mine + (hi * 16 + n) * RSO + (ct * 16 + g * 4) * 4) = oacc[hi][half * (NCT / 2) + ct] * inv[hi];
            constexpr int LPR = D_C / 8;        // lanes of half a row in fp32
            for (int r = lane / LPR; r < nrow; r += 64 / LPR) {
                const int c = lane % LPR;
                *reinterpret_cast<u32x4*>(static_cast<float*>(p.o_part) + part_of(r) * D_C + half * (D_C / 2) + c * 4) = *(LDS_AS u32x4*)(mine + r * RSO + c * 16);
            }
        }
    }
    if (g == 0 && p.lse_part) {
#pragma unroll
        for (int hi = 0; hi < 2; ++hi)
            if (hi * 16 + n < nrow)
                p.lse_part[part_of(hi * 16 + n)] = lt[hi] == 0.f ? -INFINITY : (m_ref[hi] == -INFINITY ? 0.f : m_ref[hi]) * LN2 + __builtin_amdgcn_logf(lt[hi]) * LN2;
    }
}

// ---- chunks merged: lse = log sum_s e^{lse_s}, o = sum_s e^{lse_s - lse} o_s.  A wavefront per query row and 256 columns; lane s
// holds the log-sum-exp of chunk s (at most 64).  8192 rows in 4 chunks, 67 MB: 13 us, 5.2 TB/s; 64 rows 4 us.  The partials are fp32: rounded to bf16 they would be off by as much again as the
// result's own rounding.
template <bool BF16>
__global__ __launch_bounds__(256) void masked_merge_kernel(MaskedParams p, void* o_lat, float* lse)
{
    const int lane = threadIdx.x & 63, blocks = (p.d_c + 255) / 256;
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w >= (int64_t)p.B * p.H * blocks) return;
    const int64_t row = w / blocks;
    const int c = (int)(w % blocks) * 256 + lane * 4, S = p.num_splits;
    const float ls = lane < S ? p.lse_part[row * S + lane] : -INFINITY;
    const bool in = c < p.d_c;
    const float* src = static_cast<const float*>(p.o_part) + row * S * p.d_c + (in ? c : 0);
    constexpr int BATCH = 8;
    float4 v[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) v[i] = *reinterpret_cast<const float4*>(src + (int64_t)min(i, S - 1) * p.d_c);
    const float m = wave_max(ls), ref = m == -INFINITY ? 0.f : m;
    const float e = expf(ls - ref), z = wave_sum(e);           // (a NaN stays one)
    const float wt = z == 0.f ? 0.f : e / z;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < S; s0 += BATCH) {
        if (s0) {
#pragma unroll
            for (int i = 0; i < BATCH; ++i) v[i] = *reinterpret_cast<const float4*>(src + (int64_t)min(s0 + i, S - 1) * p.d_c);
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const float k = s0 + i < S ? lane_value(wt, s0 + i) : 0.f;
            const bool live = k != 0.f;                        // (rows of empty chunks were never written)
            acc.x = fmaf(k, live ? v[i].x : 0.f, acc.x); acc.y = fmaf(k, live ? v[i].y : 0.f, acc.y);
            acc.z = fmaf(k, live ? v[i].z : 0.f, acc.z); acc.w = fmaf(k, live ? v[i].w : 0.f, acc.w);
        }
    }
    if (in) {
        if (BF16)
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(o_lat) + row * p.d_c + c) = make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
        else
            *reinterpret_cast<float4*>(static_cast<float*>(o_lat) + row * p.d_c + c) = acc;
    }
    if (lse && c == 0) lse[row] = z == 0.f ? -INFINITY : m == -INFINITY ? z : m + logf(z);
}

}  // namespace

bool masked_tall_supported(const MaskedParams& p, mla_dtype io, mla_dtype cache)
{
    auto on16 = [](const void* q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
    return io == MLA_BF16 && (cache == MLA_BF16 || cache == MLA_FP8_E4M3) && p.d_rope == 64 && masked_tall_width(p.d_c) &&
           p.page_size % 16 == 0 && (int64_t)p.num_pages * (p.page_size / 16) <= 0x7FFFFFFF && on16(p.q_abs) && on16(p.q_rope) && on16(p.kv);
}

hipError_t launch_masked_tall(const MaskedParams& p, mla_dtype cache, hipStream_t s)
{
    const unsigned chunks = ((unsigned)p.B * p.num_splits + 7) / 8 * 8, Z = (unsigned)((p.H + MT_ROWS - 1) / MT_ROWS);
    const dim3 grid(chunks * Z), block(MF_THREADS);
    if (cache == MLA_BF16 && p.d_c == 512)      masked_tall_kernel<512, false><<<grid, block, 0, s>>>(p);
    else if (cache == MLA_BF16)                 masked_tall_kernel<256, false><<<grid, block, 0, s>>>(p);
    else if (p.d_c == 512)                      masked_tall_kernel<512, true><<<grid, block, 0, s>>>(p);
    else                                        masked_tall_kernel<256, true><<<grid, block, 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_masked_merge(const MaskedParams& p, void* o_lat, float* lse, mla_dtype io, hipStream_t s)
{
    const int64_t waves = (int64_t)p.B * p.H * ((p.d_c + 255) / 256);
    const dim3 grid((unsigned)((waves + 3) / 4)), block(256);
    if (io == MLA_BF16) masked_merge_kernel<true><<<grid, block, 0, s>>>(p, o_lat, lse);
    else                masked_merge_kernel<false><<<grid, block, 0, s>>>(p, o_lat, lse);
    return hipGetLastError();
}

}  // namespace mla
