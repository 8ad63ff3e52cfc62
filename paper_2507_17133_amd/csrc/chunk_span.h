// Which positions a tile of chunk attention's rows goes through.  Whole numbers only: a host compiler takes it as well.
#pragma once

namespace bmoe {

// The positions of a tile of rows: the first `sinks`, then those from lo on, n in all.
struct Span {
    int sinks, lo, n;

    // Rows of the new tokens j0 to j1 of `fresh` behind `context` positions; `cap`: positions of the sequence's row of the block table, 0 if it has none.
    __host__ __device__ Span(int context, int fresh, int j0, int j1, bool tree, int window, int most_sinks, int cap)
    {
        const int end = context + (tree ? fresh : j1 + 1), hi = end < cap ? end : cap;
        const int from = window > 0 ? context + (tree ? 0 : j0) + 1 - window : 0;
        lo = from < 0 ? 0 : from < hi ? from : hi;
        sinks = most_sinks < lo ? most_sinks : lo;
        n = hi - lo + sinks;
        if (n == 0) lo = 0;                               // all it sees lies behind the table's last position
    }
    // The position that place i of a step reads, `most` of them counting: beyond the last one that one, and where there is none 0, which every table has.
    __host__ __device__ int read(int i, int most) const
    {
        const int in = i < most ? i : most - 1, k = in > 0 ? in : 0;
        return k < sinks ? k : k - sinks + lo;
    }
};

}  // namespace bmoe
