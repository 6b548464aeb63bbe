// disco_launch.h -- how threads of the token kernels map to their work, where
// host and device have to agree on it.  Plain C++: the host tests walk it.
#pragma once
#include <cstdint>

namespace disco {

constexpr int kAttendThreads = 256;

// The workgroups of a launch as rows of a grid: HIP takes fewer than 2^32
// threads along an axis.  Whole rows of a multiple of eight keep the workgroups'
// turn over the XCDs; the last row's surplus has no work.
struct Grid {
    uint32_t x, y;
};
constexpr uint32_t kGridRow = 1u << 21;  // times 1024 threads at most
constexpr Grid grid_of(uint32_t groups) {
    return groups <= kGridRow ? Grid{groups, 1} : Grid{kGridRow, (groups - 1) / kGridRow + 1};
}

// Joining the parts of attention rows: `lanes` threads hold four entries each
// of a row, `slices` such groups share its parts, `rows` rows go to a workgroup.
struct Join {
    int lanes, slices, rows;
    constexpr int lane(int thread) const { return thread % lanes; }
    constexpr int slice(int thread) const { return thread / lanes % slices; }
    constexpr int row(int thread) const { return thread / (lanes * slices); }
    // Whether the thread holds a part of one of the `left` rows from the
    // workgroup's first on.  Where lanes * slices does not divide the
    // workgroup, its last threads hold none.
    constexpr bool live(int thread, int64_t left) const { return row(thread) < rows && row(thread) < left; }
    // Whether the thread adds up the slices' sums, from its own on every `lanes`-th.
    constexpr bool adds(int thread, int64_t left) const { return live(thread, left) && slice(thread) == 0; }
};

inline Join join_of(int dim, int splits, int64_t all) {
    Join g{(dim + 3) / 4, 1, 0};
    while (2 * g.slices <= splits && 2 * g.slices * g.lanes <= kAttendThreads && all * g.lanes * g.slices < 65536)
        g.slices *= 2;
    g.rows = kAttendThreads / (g.lanes * g.slices);
    return g;
}

}  // namespace disco
