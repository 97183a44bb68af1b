// Rows of a paged cache moved within their sequences (the accepted path of a drafted tree to the places behind the committed rows).
//
// A workgroup takes eight units (of 16 bytes, or as many as row width and address allow) of all rows that a sequence moves, a unit
// per thread: everything is read before the barrier and written behind it, and no two workgroups share a byte, so sources and
// destinations may overlap.  Bound by latency: a round trip for positions, one for page ids, one for the row, and the launch: 3 rows of one sequence 2.4 us on
// the GPU, 8 rows of 64 sequences in fp8 2.6.
#include "layer_internal.h"
#include "mfma_tile.h"

namespace mla {
namespace {

constexpr int UNITS = 8;      // of a row, per workgroup

template <typename U>
__global__ __launch_bounds__(UNITS * MAX_MOVES) void cache_move_kernel(MoveParams p)
{
    const int b = blockIdx.x, i = threadIdx.x / UNITS, c = blockIdx.y * UNITS + threadIdx.x % UNITS;
    const int units = p.row_bytes / (int)sizeof(U);
    auto place = [&](int pos) -> int64_t {
        if (pos < 0 || pos >= p.max_pages * p.page_size) return -1;
        const int page = p.page_table[(int64_t)b * p.max_pages + pos / p.page_size];
        return page < 0 || page >= p.num_pages ? -1 : (int64_t)page * p.page_size + pos % p.page_size;
    };
    int64_t from = -1, to = -1;
    if (i < p.n) {
        const int64_t at = (int64_t)b * p.n + i;
        from = place(p.src[at]);
        to = place(p.dst[at]);
    }
    const bool moves = from >= 0 && to >= 0 && from != to;
    // (the scales of the rows: one more unit, behind the last)
    const bool unit = moves && c < units, scale = moves && c == units && p.kv_scale;
    U v;
    float s = 0.f;
    if (unit) v = static_cast<const U*>(p.kv)[from * units + c];
    if (scale) s = p.kv_scale[from];
    wait_vmcnt<0>();          // (the rows themselves, not only the requests for them, before anybody writes)
    __syncthreads();
    if (unit) static_cast<U*>(p.kv)[to * units + c] = v;
    if (scale) p.kv_scale[to] = s;
}

template <typename U> void run(const MoveParams& p, hipStream_t s)
{
    const int units = p.row_bytes / (int)sizeof(U) + (p.kv_scale != nullptr);
    const dim3 grid((unsigned)p.B, (unsigned)((units + UNITS - 1) / UNITS)), block((unsigned)((p.n * UNITS + 63) / 64 * 64));
    cache_move_kernel<U><<<grid, block, 0, s>>>(p);
}

}  // namespace

hipError_t launch_cache_move(const MoveParams& p, hipStream_t s)
{
    const uintptr_t at = reinterpret_cast<uintptr_t>(p.kv) | (uintptr_t)p.row_bytes;
    if (at % 16 == 0)     run<uint4>(p, s);
    else if (at % 4 == 0) run<uint32_t>(p, s);
    else if (at % 2 == 0) run<uint16_t>(p, s);
    else                  run<uint8_t>(p, s);
    return hipGetLastError();
}

}  // namespace mla
