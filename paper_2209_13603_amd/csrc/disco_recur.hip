// disco_recur.hip -- the gated linear recurrence along time, forward.
//
//   h_t = a_t h_(t-1) + c_t x_t,  y_t = h_t, or h_t sigmoid(z_t)
//
// Bound by the memory: x and the gates in, y out.  With channels enough to fill
// the card each thread walks its channels' steps alone, sixteen loads ahead of the
// arithmetic.  Otherwise a workgroup takes 64 channels (a 128-byte line of bf16) and its
// threads hold the runs of a tile of 256 steps: each finds its run's map, the
// maps are joined in a fixed order, and the run is taken from the state before
// it, all from registers, so that x and the gates are read once.  Where that
// leaves CUs idle the time axis is split: k_recur_maps finds the splits' maps
// first, at the price of a second read.  States and maps are fp32 throughout.
//
// Measured (kernel traces), bf16: 16384 channels of 2048 steps with an output gate 70 us (scan, 268 MB, 3.8 TB/s: the
// loads of a tile wait for its one barrier); 1048576 of 24 steps 33 us (walk, 151 MB, 4.5 TB/s); one series of 131072 x
// 768 without an output gate 96 us the maps (403 MB, 4.2 TB/s) and 134 us the states (604 MB, 4.5 TB/s, of which the
// first third is still in the caches).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "disco_internal.h"
#include "disco_recur.h"

namespace disco {

namespace {

constexpr int V = kRecurChannels;

// What a thread reads for a run.
template <typename T, bool Z>
struct Inputs {
    Part<T> g[kRun], x[kRun], z[Z ? kRun : 1];
};

// AHEAD: the next tile's loads are out while this one is worked on (fp32 has no
// registers for that; without an output gate the smaller tiles of two workgroups a CU cover each other,
// and it gained nothing; their 128 registers are asked for: left to itself the compiler takes up to 150 in bf16,
// and one series of 131072 x 768 takes 165 us instead of 133).
template <typename T, bool EVEN, bool Z, int GAIN, bool SCAN>
__global__ __launch_bounds__((Lane<V, SCAN>::kThreads), (SCAN && !Z && sizeof(T) == 2 ? 4 : 1)) void k_recur(RecurArgs a, RecurCut cut) {
    typedef Lane<V, SCAN> L;
    constexpr bool AHEAD = SCAN && sizeof(T) == 2 && Z;
    __shared__ float maps[SCAN ? 2 : 1][L::kWaves][L::kLanes][2 * V];
    const L ln(a, cut);
    const int64_t C = a.channels, at = ln.state_at(a), runs = (a.steps + kRun - 1) / kRun;
    float h[V];
    load_state(cut.splits > 1 ? cut.entry : a.state, at, ln.c, C, ln.live, h);
    if constexpr (SCAN) through_splits<V, false>(a, cut, ln.split, at, ln.c, ln.live, h);
    auto load = [&](int t) {
        Inputs<T, Z> in;
        const Run r(a, ((int64_t)t * L::kSlots + ln.slot) * kRun, ln.count);
        ln.template load<T, EVEN>(a.g, r, t, in.g);
        ln.template load<T, EVEN>(a.x, r, t, in.x);
        if constexpr (Z) ln.template load<T, EVEN>(a.z, r, t, in.z);
        return in;
    };
    Inputs<T, Z> next;
    if constexpr (AHEAD)
        if (ln.t0 < ln.t1) next = load(ln.t0);
    for (int t = ln.t0; t < ln.t1; ++t) {
        const int64_t run = (int64_t)t * L::kSlots + ln.slot, s0 = run * kRun;
        const Run r(a, s0, ln.count);
        Inputs<T, Z> in;
        if constexpr (AHEAD) {
            in = next;
            if (t + 1 < ln.t1) next = load(t + 1);
        } else {
            in = load(t);
        }
        r.take_out(in.x);
        r.hold(in.g);
        float mine[V];
        T* y = ln.template at<T>(a.y) + s0 * a.y.st;
        auto out = [&](int i, float state, int j) { return Z ? state * sigmoid(in.z[Z ? i : 0].at(j)) : state; };
        // Writes step i of the run; e(j): its states.
        auto finish = [&](auto&& e) {
            if (r.whole) {
                if (ln.live) {
                    char* to = SCAN ? ln.template tile<T>(a.y, t) : nullptr;
                    const uint32_t off = SCAN ? ln.template offset<T>(a.y) : 0;
#pragma unroll
                    for (int i = 0; i < kRun; ++i) {
                        float v[V];
#pragma unroll
                        for (int j = 0; j < V; ++j) v[j] = out(i, e(i, j), j);
                        if constexpr (SCAN) {
                            store_part<T, EVEN>((T*)(to + off), ln.next, v);
                            move_all(to, a.y.st * (int64_t)sizeof(T));
                        } else {
                            store_part<T, EVEN>(y, ln.next, v);
                            move(y, a.y.st);
                        }
                    }
                }
                return;
            }
#pragma unroll
            for (int k = 0; k < kRun; k += kGroup)
                if (r.stores(k)) {
#pragma unroll
                    for (int i = k; i < k + kGroup; ++i) {
                        float v[V];
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            v[j] = out(i, e(i, j), j);
                            v[j] = i < r.left ? v[j] : 0.0f;
                        }
                        if (ln.live && i < r.steps) store_part<T, EVEN>(y, ln.next, v);
                        move(y, a.y.st);
                    }
                }
        };
        if constexpr (SCAN) {
            // the run's map step by step; the states are one multiply-add from it
            float A[kRun][V], B[kRun][V], qa[V], qb[V];
            Product P[V];
            float state[V] = {0.0f};
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const Step<T> step(in.g[i].at(j));
                    step.onto(P[j]);
                    state[j] = step.template advance<GAIN>(state[j], in.x[i].at(j));
                    A[i][j] = P[j].a;
                    B[i][j] = state[j];
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                qa[j] = P[j].gate();
                qb[j] = state[j];
            }
            JoinMaps<V, SCAN, false>::run(qa, qb, h, mine, maps, t & 1);
            if (a.carries) store_state(a.carries, (ln.b * runs + run) * C + ln.c, ln.c, C, ln.live && run < runs, mine);
            finish([&](int i, int j) { return fmaf(A[i][j], mine[j], B[i][j]); });
        } else {
            if (a.carries) store_state(a.carries, (ln.b * runs + run) * C + ln.c, ln.c, C, ln.live, h);
            finish([&](int i, int j) {
                const float q = gate_of(in.g[i].at(j));
                return h[j] = advance<GAIN>(h[j], q, in.x[i].at(j));
            });
        }
    }
    if (a.last && ln.slot == 0 && ln.split == cut.splits - 1) store_state(a.last, at, ln.c, C, ln.live, h);
}

// The maps of all splits but the last.
template <typename T, bool EVEN, int GAIN>
__global__ __launch_bounds__(kScanBlock) void k_recur_maps(RecurArgs a, RecurCut cut) {
    typedef Lane<V, true> L;
    __shared__ float maps[2][L::kWaves][L::kLanes][2 * V];
    const L ln(a, cut);
    SplitMap<V> all;
    struct Pair {
        Part<T> g[kRun], x[kRun];
    };
    auto load = [&](int t) {
        Pair in;
        const Run r(a, ((int64_t)t * L::kSlots + ln.slot) * kRun, ln.count);
        ln.template load<T, EVEN>(a.g, r, t, in.g);
        ln.template load<T, EVEN>(a.x, r, t, in.x);
        return in;
    };
    for (int t = ln.t1 - 1; t >= ln.t0; --t) {
        const Run r(a, ((int64_t)t * L::kSlots + ln.slot) * kRun, ln.count);
        Pair in = load(t);
        r.take_out(in.x);
        r.hold(in.g);
        float qa[V], qb[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            Product P;
            float state = 0.0f;
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                const Step<T> step(in.g[i].at(j));
                step.onto(P);
                state = step.template advance<GAIN>(state, in.x[i].at(j));
            }
            qa[j] = P.gate();
            qb[j] = state;
        }
        JoinMaps<V, true, false>::all(qa, qb, maps, t & 1);
        if (ln.slot == 0) all.before(qa, qb);
    }
    if (ln.slot != 0 || !ln.live) return;
    if (ln.split == 0) keep_entry(ln, a, cut, a.state);
    all.store(ln, a, cut);
}

}  // namespace

hipError_t launch_recur(const RecurArgs& a, float* ws) {
    RecurCut cut = recur_cut(a);
    recur_ws(&cut, a, ws);
    if (cut.splits > 1) {
        const int tk = timing_begin("recurrence_maps", a.stream);
        const uint32_t groups = cut.groups / cut.splits * (cut.splits - 1);
        const hipError_t e = recur_dispatch(a, [&](auto t, auto even, auto) {
            return by_gain(a.gain, [&](auto gain) {
                hipLaunchKernelGGL((k_recur_maps<decltype(t), decltype(even)::value, decltype(gain)::value>), grid_dim(groups),
                                   dim3(kScanBlock), 0, a.stream, a, cut);
                return hipGetLastError();
            });
        });
        timing_end(tk, a.stream);
        if (e != hipSuccess) return e;
    }
    const int tk = timing_begin("recurrence", a.stream);
    const hipError_t e = recur_dispatch(a, [&](auto t, auto even, auto z) {
        return by_gain(a.gain, [&](auto gain) {
            auto go = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid_dim(cut.groups), dim3(cut.blocks ? kScanBlock : kWalkBlock), 0, a.stream, a, cut);
            };
            if (cut.blocks) go(k_recur<decltype(t), decltype(even)::value, decltype(z)::value, decltype(gain)::value, true>);
            else go(k_recur<decltype(t), decltype(even)::value, decltype(z)::value, decltype(gain)::value, false>);
            return hipGetLastError();
        });
    });
    timing_end(tk, a.stream);
    return e;
}

}  // namespace disco
