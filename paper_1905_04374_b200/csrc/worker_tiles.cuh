// Which tile of a product a running number stands for (worker_linear.cu): whole numbers only, for the kernels and, in
// plain C++, for the host.
#pragma once
#ifdef __CUDACC__
#define GAR_TILES_FN __host__ __device__ __forceinline__
#else
#define GAR_TILES_FN inline
#endif

namespace gar {
namespace worker {

// What the mapping goes by.  mt * nt * splits < 2^30 and 1 <= group_m <= mt: all products below stay under 2^30.
struct Tiling {
    int mt, nt, splits;       // (pair) row tiles, column tiles, parts of the contraction (OUTER: workers)
    int group_m;              // row tiles that go round a column tile together
    int steps;                // of the whole contraction
};
struct Place {
    int m, n, split, first, steps;
};

// Row tiles that go round a column tile together: B is read from memory once for each such group of rows of A, which
// should stay in L2: 32 MB of them, of the row tiles that there are.  8192 rows, 4096 x 8192 gated: 785 us in groups of 8, 772 of 16
// (32 MB), 785 of 24, 829 of 32; 2048 x 32000: 775 of 8, 755 of 16, 744 of 32 (32 MB).
GAR_TILES_FN int group_rows(int steps, int mt) {
    const int fits = steps < 128 ? 1024 / steps : 8;
    return fits < mt ? fits : mt;
}

template <bool OUTER>
GAR_TILES_FN Place place_in(const Tiling& a, unsigned index) {
    Place t;
    unsigned split = 0;
    if (OUTER) {                         // one worker after the other
        const unsigned per = unsigned(a.mt) * unsigned(a.nt);
        split = index / per;
        index -= split * per;
    } else if (a.splits > 1) {
        split = index % unsigned(a.splits);
        index /= unsigned(a.splits);
    }
    const unsigned group_m = unsigned(a.group_m), per_group = group_m * unsigned(a.nt), g = index / per_group, in_group = index - g * per_group;
    const unsigned left = unsigned(a.mt) - g * group_m, rows = group_m < left ? group_m : left;
    t.n = int(in_group / rows);
    t.m = int(g * group_m + in_group - unsigned(t.n) * rows);
    t.split = int(split);
    t.first = 0;
    t.steps = a.steps;
    if (!OUTER && a.splits > 1) {
        const int part = (a.steps + a.splits - 1) / a.splits;
        t.first = int(split) * part;
        t.steps = part < a.steps - t.first ? part : a.steps - t.first;
    }
    return t;
}

}  // namespace worker
}  // namespace gar
