// disco_recur_grad.hip -- gradients of the gated linear recurrence.
//
//   D_t = o_t dy_t + a_(t+1) D_(t+1)  (the last one: + dlast),  o = sigmoid(z) or 1,
//   dx_t = c_t D_t,  dg_t = D_t (h_(t-1) + x_t dc/da) a (1 - a),
//   dz_t = dy_t h_t o (1 - o),  dstate = a_0 D_0
//
// the states h recomputed in fp32, run by run, from those that the forward call
// left before every run of 16 steps (1/8 of a bf16 tensor's bytes a call, instead of
// a tensor of states): the pass reads x, the gates and dy once and writes the
// gradients.  The same walk, scan and splits as forward, from the end to the start.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "disco_internal.h"
#include "disco_recur.h"

namespace disco {

namespace {

constexpr int V = kRecurChannels;

// dc/da times a (1 - a).
template <int GAIN>
__device__ __forceinline__ float gain_slope(float q) {
    const float s = fabsf(q);
    if (GAIN == kGainMean) return -fmaf(-s, s, s);
    if (GAIN == kGainOne) return 0.0f;
    const float a = closed(q) ? s : 1.0f - s, rest = closed(q) ? 1.0f - s : s;
    return -a * a * __builtin_amdgcn_sqrtf(rest * __builtin_amdgcn_rcpf(1.0f + a));
}

template <typename T, bool WIDE, bool Z, int GAIN, bool SCAN>
__global__ __launch_bounds__(kRecurThreads) void k_recur_grad(RecurArgs a, RecurCut cut) {
    typedef Lane<V, SCAN> L;
    __shared__ float maps[SCAN ? 2 : 1][L::kWaves][L::kLanes][2 * V];
    const L ln(a, cut);
    const int64_t C = a.channels, at = ln.state_at(a), runs = (a.steps + kRun - 1) / kRun;
    float G[V];  // what the steps behind pass to the state
    load_state(cut.splits > 1 ? cut.entry : a.dlast, at, ln.c, C, ln.live, G);
    if constexpr (SCAN) through_splits<V, true>(a, cut, ln.split, at, ln.c, ln.live, G);
    for (int t = ln.t1 - 1; t >= ln.t0; --t) {
        const int64_t run = (int64_t)t * L::kSlots + ln.slot, s0 = run * kRun;
        const Run r(a, s0, ln.count);
        Part<T, V> x[kRun], dy[kRun];
        float q[kRun][V], qz[Z ? kRun : 1][V], h[V];
        load_state(a.carries, (ln.b * runs + run) * C + ln.c, ln.c, C, ln.live && run < runs, h);
        {
            Part<T, V> g[kRun], z[kRun];
            r.template load<T, V, WIDE>(ln.template at<const T>(a.g), a.g.st, ln.c, C, g);
            r.template load<T, V, WIDE>(ln.template at<const T>(a.x), a.x.st, ln.c, C, x);
            r.template load<T, V, WIDE>(ln.template at<const T>(a.dy), a.dy.st, ln.c, C, dy);
            if constexpr (Z) r.template load<T, V, WIDE>(ln.template at<const T>(a.z), a.z.st, ln.c, C, z);
#pragma unroll
            for (int i = 0; i < kRun; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    q[i][j] = gate_of((float)g[i].v[j]);
                    if constexpr (Z) qz[i][j] = gate_of((float)z[i].v[j]);
                }
            take_out(r, q);
        }
        // the gradient that the output of step i brings to its state
        auto brought = [&](int i, int j) {
            const float d = (float)dy[i].v[j];
            if constexpr (!Z) return d;
            const float s = fabsf(qz[Z ? i : 0][j]);
            return d * (closed(qz[Z ? i : 0][j]) ? s : 1.0f - s);
        };
        float mine[V];
        if constexpr (SCAN) {
            Product P[V];
            float A[V], B[V];
#pragma unroll
            for (int j = 0; j < V; ++j) B[j] = 0.0f;
#pragma unroll
            for (int i = kRun - 1; i >= 0; --i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    P[j].take(q[i][j]);
                    B[j] = decay(B[j] + brought(i, j), q[i][j]);
                }
#pragma unroll
            for (int j = 0; j < V; ++j) A[j] = P[j].gate();
            JoinMaps<V, SCAN, true>::run(A, B, G, mine, maps, t & 1);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) mine[j] = G[j];
        }
        float before[kRun + 1][V];
#pragma unroll
        for (int j = 0; j < V; ++j) before[0][j] = h[j];
#pragma unroll
        for (int i = 0; i < kRun; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) before[i + 1][j] = advance<GAIN>(before[i][j], q[i][j], (float)x[i].v[j]);
        T* to_x = ln.template at<T>(a.dx) + (s0 + kRun - 1) * a.dx.st;
        T* to_g = ln.template at<T>(a.dg) + (s0 + kRun - 1) * a.dg.st;
        T* to_z = ln.template at<T>(a.dz) + (s0 + kRun - 1) * a.dz.st;
#pragma unroll
        for (int i = kRun - 1; i >= 0; --i, to_x -= a.dx.st, to_g -= a.dg.st, to_z -= a.dz.st) {
            float dx[V], dg[V], dz[V];
            const bool inside = i < r.left;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float D = mine[j] + brought(i, j), s = fabsf(q[i][j]), slope = fmaf(-s, s, s);
                dx[j] = inside ? gain_of<GAIN>(q[i][j]) * D : 0.0f;
                if (GAIN == kGainMean) dg[j] = D * slope * (before[i][j] - (float)x[i].v[j]);
                else dg[j] = D * fmaf(gain_slope<GAIN>(q[i][j]), (float)x[i].v[j], slope * before[i][j]);
                dg[j] = inside ? dg[j] : 0.0f;
                if constexpr (Z) {
                    const float u = fabsf(qz[Z ? i : 0][j]);
                    dz[j] = inside ? (float)dy[i].v[j] * before[i + 1][j] * fmaf(-u, u, u) : 0.0f;
                }
                mine[j] = decay(D, q[i][j]);
            }
            if (ln.live && i < r.steps) {
                if (a.dx.p) store_part<T, V, WIDE>(to_x, ln.c, C, dx);
                if (a.dg.p) store_part<T, V, WIDE>(to_g, ln.c, C, dg);
                if constexpr (Z)
                    if (a.dz.p) store_part<T, V, WIDE>(to_z, ln.c, C, dz);
            }
        }
        if constexpr (!SCAN) {
#pragma unroll
            for (int j = 0; j < V; ++j) G[j] = mine[j];
        }
    }
    if (a.dstate && ln.slot == 0 && ln.split == 0) store_state(a.dstate, at, ln.c, C, ln.live, G);
}

// The maps of all splits but the first, from their ends.
template <typename T, bool WIDE, bool Z>
__global__ __launch_bounds__(kRecurThreads) void k_recur_grad_maps(RecurArgs a, RecurCut cut) {
    typedef Lane<V, true> L;
    __shared__ float maps[L::kSlots][L::kLanes][2 * V];
    const L ln(a, cut, 1);
    const int64_t C = a.channels;
    const int n = ln.t1 - ln.t0;
    Product P[V];
    float A[V], B[V];
#pragma unroll
    for (int j = 0; j < V; ++j) B[j] = 0.0f;
    for (int t = n - 1; t >= 0; --t) {
        const int64_t s0 = ((int64_t)ln.t0 * L::kSlots + (int64_t)ln.slot * n + t) * kRun;
        const Run r(a, s0, ln.count);
        Part<T, V> g[kRun], dy[kRun], z[kRun];
        r.template load<T, V, WIDE>(ln.template at<const T>(a.g), a.g.st, ln.c, C, g);
        r.template load<T, V, WIDE>(ln.template at<const T>(a.dy), a.dy.st, ln.c, C, dy);
        if constexpr (Z) r.template load<T, V, WIDE>(ln.template at<const T>(a.z), a.z.st, ln.c, C, z);
        float q[kRun][V];
#pragma unroll
        for (int i = 0; i < kRun; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) q[i][j] = gate_of((float)g[i].v[j]);
        take_out(r, q);
#pragma unroll
        for (int i = kRun - 1; i >= 0; --i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = (float)dy[i].v[j];
                P[j].take(q[i][j]);
                B[j] = decay(B[j] + (Z ? d * sigmoid((float)z[i].v[j]) : d), q[i][j]);
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
    if (ln.slot != L::kSlots - 1 || !ln.live) return;
    if (ln.split == 1) keep_entry(ln, a, cut, a.dlast);
    for (int s = L::kSlots - 2; s >= 0; --s)
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

size_t recur_ws_bytes(const RecurArgs& a) {
    const RecurCut cut = recur_cut(a);
    return cut.splits > 1 ? ((size_t)cut.splits * 2 + 1) * a.batch * a.channels * sizeof(float) : 0;
}

hipError_t launch_recur_grad(const RecurArgs& a, float* ws) {
    RecurCut cut = recur_cut(a);
    recur_ws(&cut, a, ws);
    if (cut.splits > 1) {
        const int tk = timing_begin("recurrence_grad_maps", a.stream);
        const uint32_t groups = cut.groups / cut.splits * (cut.splits - 1);
        const hipError_t e = recur_dispatch(a, [&](auto t, auto wide, auto z) {
            hipLaunchKernelGGL((k_recur_grad_maps<decltype(t), decltype(wide)::value, decltype(z)::value>), grid_dim(groups),
                               dim3(kRecurThreads), 0, a.stream, a, cut);
            return hipGetLastError();
        });
        timing_end(tk, a.stream);
        if (e != hipSuccess) return e;
    }
    const int tk = timing_begin("recurrence_grad", a.stream);
    const hipError_t e = recur_dispatch(a, [&](auto t, auto wide, auto z) {
        return by_gain(a.gain, [&](auto gain) {
            auto go = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid_dim(cut.groups), dim3(kRecurThreads), 0, a.stream, a, cut);
            };
            if (cut.blocks) go(k_recur_grad<decltype(t), decltype(wide)::value, decltype(z)::value, decltype(gain)::value, true>);
            else go(k_recur_grad<decltype(t), decltype(wide)::value, decltype(z)::value, decltype(gain)::value, false>);
            return hipGetLastError();
        });
    });
    timing_end(tk, a.stream);
    return e;
}

}  // namespace disco
