// Walks the thread maps of disco_launch.h on the CPU (tests/test_token_launch_host.py).
#include <cstdio>
#include <cstring>
#include <initializer_list>

#include "disco_launch.h"

using namespace disco;

static int failures = 0;

// Every index that a thread of the join reads or writes in the workgroup's
// shared sums lies in them, every part of a live row is added once, by the
// thread that writes the row.
static void join() {
    for (int dim = 1; dim <= 128; ++dim)
        for (int splits : {2, 3, 4, 7, 16, 33, 64, 128, 256})
            for (int64_t all : {int64_t(1), int64_t(2), int64_t(5), int64_t(64), int64_t(300), int64_t(70000)}) {
                const Join g = join_of(dim, splits, all);
                const int64_t groups = (all + g.rows - 1) / g.rows;
                bool good = g.rows >= 1 && 4 * g.lanes >= dim;
                for (int64_t wg : {int64_t(0), groups - 1}) {
                    const int64_t left = all - wg * g.rows;
                    int added[kAttendThreads] = {0};
                    for (int t = 0; t < kAttendThreads; ++t)
                        for (int s = 0; g.adds(t, left) && s < g.slices; ++s) {
                            const int at = t + s * g.lanes;
                            if (at >= kAttendThreads) good = false;
                            else ++added[at];
                        }
                    for (int t = 0; t < kAttendThreads; ++t) good = good && added[t] == (g.live(t, left) ? 1 : 0);
                }
                if (!good && failures++ < 10)
                    std::printf("join: dim %d splits %d rows %lld: lanes %d slices %d rows %d\n", dim, splits, (long long)all,
                                g.lanes, g.slices, g.rows);
            }
}

// Every workgroup of a launch has a place, no axis has 2^32 threads or 2^16 rows.
static void grid() {
    for (uint64_t groups : {uint64_t(1), uint64_t(7), uint64_t(2048), uint64_t(1) << 21, (uint64_t(1) << 21) + 1, uint64_t(1) << 24,
                            // rows of 2^31 / 4 (norm and rotation, 64 lanes a row), of 2^35 / 128 and 2^19 pairs of item and head
                            // (attention), rounded up to eight runs
                            (uint64_t(1) << 29) + 1, (uint64_t(1) << 28) + (uint64_t(1) << 19) + 4096, uint64_t(0x7fffffff)}) {
        const Grid g = grid_of((uint32_t)groups);
        const uint64_t all = uint64_t(g.x) * g.y;
        const bool good = uint64_t(g.x) * 1024 < (uint64_t(1) << 32) && g.y <= 65535 && all >= groups && all - groups < kGridRow &&
                          all < (uint64_t(1) << 32) && (g.y == 1 || g.x % 8 == 0);
        if (!good && failures++ < 10) std::printf("grid: %llu groups as %u x %u\n", (unsigned long long)groups, g.x, g.y);
    }
}

int main(int argc, char** argv) {
    const char* what = argc > 1 ? argv[1] : "";
    if (!std::strcmp(what, "join")) join();
    else if (!std::strcmp(what, "grid")) grid();
    else return 2;
    std::printf("%s: %d failures\n", what, failures);
    return failures != 0;
}
