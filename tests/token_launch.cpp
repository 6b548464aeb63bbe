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

int main(int argc, char** argv) {
    const char* what = argc > 1 ? argv[1] : "";
    if (!std::strcmp(what, "join")) join();
    else return 2;
    std::printf("%s: %d failures\n", what, failures);
    return failures != 0;
}
