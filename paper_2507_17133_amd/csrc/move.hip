// Keys and values of accepted tokens move to the positions that they have in the sequence.
//
// Sources increase and none lies before its target, so a thread that takes its 16 bytes of a head through the list, eight entries read before any of
// them is written, moves them as if all had been read first.  Each entry is two dependent loads (list, block table) of one address for the whole block, then
// the row: latency, of a few accepted tokens (5 of one request, 8 heads of 128, bf16: 4.5 us) as of many (up to 9 of each of 256, e4m3: 9.7 us in a row of calls, 9.4 MB
// read and written).  Every thread walks the list and divides for itself, and the time goes by the entries: up to 1, 2, 4, 8, 9 and 16 of each of 256 take 4.0, 4.7, 5.9, 8.4, 9.9 and 14.6 us.  Trips
// cost little beside that from eight entries on: up to 9 with 4 at a time 20.6 us, with 12 9.4, with 16 10.1, the one request 0.1 and 0.6 us more.
#include "draft.h"

namespace bmoe {
namespace {

constexpr int kMoveThreads = 256, kAhead = 8;

struct MoveArgs {
    char *k, *v;
    int64_t page_stride, token_stride, head_stride;       // bytes
    const int32_t *pages, *row_of;
    int64_t row_stride;
    int n_rows, max_pages, n_pages, page_size;
    const int32_t *sources, *start, *count;
    int64_t sources_stride;
    int max_moves, pieces, units;                         // pieces of 16 bytes of a head; of k and v of a position
};

__global__ void __launch_bounds__(kMoveThreads) move_kernel(MoveArgs p)
{
    const int b = blockIdx.x, unit = blockIdx.y * kMoveThreads + threadIdx.x;
    const int row = p.row_of ? p.row_of[b] : b, n = min(p.count[b], p.max_moves);
    const int64_t start = p.start[b];
    if ((unsigned)row >= (unsigned)p.n_rows || n <= 0) return;
    const int32_t *pages = p.pages + (int64_t)row * p.row_stride, *sources = p.sources + (int64_t)b * p.sources_stride;
    auto place = [&](int64_t pos) -> int64_t {            // bytes from the cache's base, or -1
        if (pos < 0 || pos >= (int64_t)p.max_pages * p.page_size) return -1;
        const int at = (int)((unsigned)pos / (unsigned)p.page_size), page = pages[at];
        if ((unsigned)page >= (unsigned)p.n_pages) return -1;
        return (int64_t)page * p.page_stride + (pos - (int64_t)at * p.page_size) * p.token_stride;
    };
    const int half = p.units / 2, of = unit < half ? unit : unit - half, head = of / p.pieces;
    char* base = (unit < half ? p.k : p.v) + head * p.head_stride + (int64_t)(of - head * p.pieces) * 16;
    int last = -1;                                        // the largest source so far
    for (int j0 = 0; j0 < n; j0 += kAhead) {
        uint4 held[kAhead];
        int64_t to[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int j = j0 + i, source = j < n ? sources[j] : -1;
            const bool follows = source > last && source >= start + j;
            last = max(last, source);
            const int64_t from = follows && source != start + j ? place(source) : -1;
            to[i] = from >= 0 ? place(start + j) : -1;
            if (to[i] >= 0 && unit < p.units) held[i] = *reinterpret_cast<const uint4*>(base + from);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (to[i] >= 0 && unit < p.units) *reinterpret_cast<uint4*>(base + to[i]) = held[i];
    }
}

}  // namespace

hipError_t launch_move(const moe_kv_cache& c, const moe_block_table& t, const int32_t* sources, int64_t sources_stride, int max_moves, const int32_t* start,
                       const int32_t* count, int n_seqs, hipStream_t s)
{
    const int size = c.type == MOE_KV_E4M3 ? 1 : 2;
    MoveArgs p;
    p.k = static_cast<char*>(c.k); p.v = static_cast<char*>(c.v);
    p.page_stride = c.page_stride * size; p.token_stride = c.token_stride * size; p.head_stride = c.head_stride * size;
    p.pages = t.pages; p.row_of = t.token_row; p.row_stride = t.row_stride;
    p.n_rows = t.n_rows; p.max_pages = t.max_pages; p.n_pages = c.n_pages; p.page_size = c.page_size;
    p.sources = sources; p.start = start; p.count = count; p.sources_stride = sources_stride;
    p.max_moves = max_moves;
    p.pieces = c.head_dim * size / 16;
    p.units = 2 * c.n_kv_heads * p.pieces;
    hipLaunchKernelGGL(move_kernel, dim3(n_seqs, ceil_div(p.units, kMoveThreads)), dim3(kMoveThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace bmoe
