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
#include <hip/hip_runtime.h>

#include <cstdint>

#include "disco_internal.h"
#include "disco_recur.h"

namespace disco {

namespace {

constexpr int V = kRecurChannels;

template <typename T, bool WIDE, bool Z, int GAIN, bool SCAN>
__global__ __launch_bounds__(kRecurThreads) void k_recur(RecurArgs a, RecurCut cut) {
    typedef Lane<V, SCAN> L;
    __shared__ float maps[SCAN ? 2 : 1][L::kWaves][L::kLanes][2 * V];
    const L ln(a, cut);
    const int64_t C = a.channels, at = ln.state_at(a), runs = (a.steps + kRun - 1) / kRun;
    float h[V];
    load_state(cut.splits > 1 ? cut.entry : a.state, at, ln.c, C, ln.live, h);
    if constexpr (SCAN) through_splits<V, false>(a, cut, ln.split, at, ln.c, ln.live, h);
    for (int t = ln.t0; t < ln.t1; ++t) {
        const int64_t run = (int64_t)t * L::kSlots + ln.slot, s0 = run * kRun;
        const Run r(a, s0, ln.count);
        Part<T, V> x[kRun], z[kRun];
        float q[kRun][V];
        {
            Part<T, V> g[kRun];
            r.template load<T, V, WIDE>(ln.template at<const T>(a.g), a.g.st, ln.c, C, g);
            r.template load<T, V, WIDE>(ln.template at<const T>(a.x), a.x.st, ln.c, C, x);
            if constexpr (Z) r.template load<T, V, WIDE>(ln.template at<const T>(a.z), a.z.st, ln.c, C, z);
#pragma unroll
            for (int i = 0; i < kRun; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) q[i][j] = gate_of((float)g[i].v[j]);
            take_out(r, q);
        }
        float mine[V];
        if constexpr (SCAN) {
            Product P[V];
            float A[V], B[V];
#pragma unroll
            for (int j = 0; j < V; ++j) B[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < kRun; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    P[j].take(q[i][j]);
                    B[j] = advance<GAIN>(B[j], q[i][j], (float)x[i].v[j]);
                }
#pragma unroll
            for (int j = 0; j < V; ++j) A[j] = P[j].gate();
            JoinMaps<V, SCAN, false>::run(A, B, h, mine, maps, t & 1);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) mine[j] = h[j];
        }
        if (a.carries) store_state(a.carries, (ln.b * runs + run) * C + ln.c, ln.c, C, ln.live && run < runs, mine);
        T* y = ln.template at<T>(a.y) + s0 * a.y.st;
#pragma unroll
        for (int i = 0; i < kRun; ++i, y += a.y.st) {
            float e[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                mine[j] = advance<GAIN>(mine[j], q[i][j], (float)x[i].v[j]);
                e[j] = Z ? mine[j] * sigmoid((float)z[i].v[j]) : mine[j];
                e[j] = i < r.left ? e[j] : 0.0f;
            }
            if (ln.live && i < r.steps) store_part<T, V, WIDE>(y, ln.c, C, e);
        }
        if constexpr (!SCAN) {
#pragma unroll
            for (int j = 0; j < V; ++j) h[j] = mine[j];
        }
    }
    if (a.last && ln.slot == 0 && ln.split == cut.splits - 1) store_state(a.last, at, ln.c, C, ln.live, h);
}

// The maps of all splits but the last: each slot takes a stretch of the split's
// runs, and the slots' maps are joined in their order.
template <typename T, bool WIDE, int GAIN>
__global__ __launch_bounds__(kRecurThreads) void k_recur_maps(RecurArgs a, RecurCut cut) {
    typedef Lane<V, true> L;
    __shared__ float maps[L::kSlots][L::kLanes][2 * V];
    const L ln(a, cut);
    const int64_t C = a.channels;
    const int n = ln.t1 - ln.t0;
    Product P[V];
    float A[V], B[V];
#pragma unroll
    for (int j = 0; j < V; ++j) B[j] = 0.0f;
    for (int t = 0; t < n; ++t) {
        const int64_t s0 = ((int64_t)ln.t0 * L::kSlots + (int64_t)ln.slot * n + t) * kRun;
        const Run r(a, s0, ln.count);
        Part<T, V> x[kRun], g[kRun];
        r.template load<T, V, WIDE>(ln.template at<const T>(a.g), a.g.st, ln.c, C, g);
        r.template load<T, V, WIDE>(ln.template at<const T>(a.x), a.x.st, ln.c, C, x);
        float q[kRun][V];
#pragma unroll
        for (int i = 0; i < kRun; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) q[i][j] = gate_of((float)g[i].v[j]);
        take_out(r, q);
#pragma unroll
        for (int i = 0; i < kRun; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                P[j].take(q[i][j]);
                B[j] = advance<GAIN>(B[j], q[i][j], (float)x[i].v[j]);
            }
    }
    const int col = threadIdx.x % L::kLanes;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        A[j] = P[j].gate();
        maps[ln.slot][col][j] = A[j];
        maps[ln.slot][col][V + j] = B[j];
    }
    __syncthreads();
    if (ln.slot != 0 || !ln.live) return;
    if (ln.split == 0) keep_entry(ln, a, cut, a.state);
    for (int s = 1; s < L::kSlots; ++s)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            B[j] = decay(B[j], maps[s][col][j]) + maps[s][col][V + j];
            A[j] = joined(A[j], maps[s][col][j]);
        }
    float* out = cut.maps + 2 * ((int64_t)ln.split * a.batch * C + ln.state_at(a));
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (ln.c + j < C) {
            out[2 * j] = A[j];
            out[2 * j + 1] = B[j];
        }
}

}  // namespace

hipError_t launch_recur(const RecurArgs& a, float* ws) {
    RecurCut cut = recur_cut(a);
    recur_ws(&cut, a, ws);
    if (cut.splits > 1) {
        const int tk = timing_begin("recurrence_maps", a.stream);
        const uint32_t groups = cut.groups / cut.splits * (cut.splits - 1);
        const hipError_t e = recur_dispatch(a, [&](auto t, auto wide, auto) {
            return by_gain(a.gain, [&](auto gain) {
                hipLaunchKernelGGL((k_recur_maps<decltype(t), decltype(wide)::value, decltype(gain)::value>), grid_dim(groups),
                                   dim3(kRecurThreads), 0, a.stream, a, cut);
                return hipGetLastError();
            });
        });
        timing_end(tk, a.stream);
        if (e != hipSuccess) return e;
    }
    const int tk = timing_begin("recurrence", a.stream);
    const hipError_t e = recur_dispatch(a, [&](auto t, auto wide, auto z) {
        return by_gain(a.gain, [&](auto gain) {
            auto go = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid_dim(cut.groups), dim3(kRecurThreads), 0, a.stream, a, cut);
            };
            if (cut.blocks) go(k_recur<decltype(t), decltype(wide)::value, decltype(z)::value, decltype(gain)::value, true>);
            else go(k_recur<decltype(t), decltype(wide)::value, decltype(z)::value, decltype(gain)::value, false>);
            return hipGetLastError();
        });
    });
    timing_end(tk, a.stream);
    return e;
}

}  // namespace disco
