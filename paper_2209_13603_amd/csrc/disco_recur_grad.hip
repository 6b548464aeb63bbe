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
//
// Measured (kernel traces), bf16, with an output gate 16384 channels of 2048 steps 114 us (scan, 478 MB, 4.2 TB/s); without
// one 1048576 of 24 steps 54 us (walk, 260 MB, 4.8 TB/s).  The scan holds 171 to 256 registers, one workgroup a CU; with an
// output gate over an odd number of channels in bf16 it spills 8.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "disco_internal.h"
#include "disco_recur.h"

namespace disco {

namespace {

constexpr int V = kRecurChannels;

// Nothing is moved over it: the steps of a run have much to do ahead of the chain
// that links them, which taken all at once does not fit the registers.
__device__ __forceinline__ void apart() { __builtin_amdgcn_sched_barrier(0); }

// dc/da times a (1 - a).
template <int GAIN>
__device__ __forceinline__ float gain_slope(float q) {
    const float s = fabsf(q);
    if (GAIN == kGainMean) return -fmaf(-s, s, s);
    if (GAIN == kGainOne) return 0.0f;
    const float a = closed(q) ? s : 1.0f - s, rest = closed(q) ? 1.0f - s : s;
    return -a * a * __builtin_amdgcn_sqrtf(rest * __builtin_amdgcn_rcpf(1.0f + a));
}

// What a thread reads for a run.
template <typename T, bool Z>
struct Inputs {
    Part<T> g[kRun], x[kRun], dy[kRun], z[Z ? kRun : 1];
    float before[V];
};

// AHEAD: the next tile's loads are out while this one is worked on.
template <typename T, bool EVEN, bool Z, int GAIN, bool SCAN>
__global__ __launch_bounds__((Lane<V, SCAN>::kThreads)) void k_recur_grad(RecurArgs a, RecurCut cut) {
    typedef Lane<V, SCAN> L;
    constexpr bool AHEAD = SCAN && sizeof(T) == 2;
    __shared__ float maps[SCAN ? 2 : 1][L::kWaves][L::kLanes][2 * V];
    // The states before the steps of a thread's run (in registers they would leave no room for the
    // next tile).
    struct alignas(4 * V) Pair {
        float v[V];
    };
    __shared__ Pair before[kRun][L::kThreads];
    const L ln(a, cut);
    const int64_t C = a.channels, at = ln.state_at(a), runs = (a.steps + kRun - 1) / kRun;
    float G[V];  // what the steps behind pass to the state
    load_state(cut.splits > 1 ? cut.entry : a.dlast, at, ln.c, C, ln.live, G);
    if constexpr (SCAN) through_splits<V, true>(a, cut, ln.split, at, ln.c, ln.live, G);
    auto load = [&](int t) {
        Inputs<T, Z> in;
        const int64_t run = (int64_t)t * L::kSlots + ln.slot;
        const Run r(a, run * kRun, ln.count);
        load_state(a.carries, (ln.b * runs + run) * C + ln.c, ln.c, C, ln.live && run < runs, in.before);
        ln.template load<T, EVEN>(a.g, r, t, in.g);
        ln.template load<T, EVEN>(a.dy, r, t, in.dy);
        if constexpr (Z) ln.template load<T, EVEN>(a.z, r, t, in.z);
        ln.template load<T, EVEN>(a.x, r, t, in.x);
        return in;
    };
    Inputs<T, Z> next;
    if constexpr (AHEAD)
        if (ln.t0 < ln.t1) next = load(ln.t1 - 1);
    for (int t = ln.t1 - 1; t >= ln.t0; --t) {
        const int64_t run = (int64_t)t * L::kSlots + ln.slot, s0 = run * kRun;
        const Run r(a, s0, ln.count);
        Inputs<T, Z> in;
        if constexpr (AHEAD) {
            in = next;
            if (t > ln.t0) next = load(t - 1);
        } else {
            in = load(t);
        }
        r.take_out(in.x);
        r.take_out(in.dy);
        if constexpr (Z) r.take_out(in.z);
        float q[kRun][V], qz[Z ? kRun : 1][V];
#pragma unroll
        for (int i = 0; i < kRun; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                q[i][j] = gate_of(in.g[i].at(j));
                if constexpr (Z) qz[i][j] = gate_of(in.z[i].at(j));
            }
        r.take_out(q);
        // the gradient that the output of step i brings to its state
        auto brought = [&](int i, int j) {
            const float d = in.dy[i].at(j);
            if constexpr (!Z) return d;
            const float s = fabsf(qz[Z ? i : 0][j]);
            return d * (closed(qz[Z ? i : 0][j]) ? s : 1.0f - s);
        };
        float mine[V];
        if constexpr (SCAN) {
            float qa[V], qb[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                Product P;
                float D = 0.0f;
#pragma unroll
                for (int i = kRun - 1; i >= 0; --i) {
                    P.take(q[i][j]);
                    D = decay(D + brought(i, j), q[i][j]);
                    if (i % kGroup == 0) apart();
                }
                qa[j] = P.gate();
                qb[j] = D;
            }
            JoinMaps<V, SCAN, true>::run(qa, qb, G, mine, maps, t & 1);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) mine[j] = G[j];
        }
        anew(q);
        if constexpr (Z) anew(qz);
#pragma unroll
        for (int i = 0; i < kRun; ++i) in.dy[i].anew();
        {
            float h[V];
#pragma unroll
            for (int j = 0; j < V; ++j) h[j] = in.before[j];
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                Pair p;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    p.v[j] = h[j];
                    h[j] = advance<GAIN>(h[j], q[i][j], in.x[i].at(j));
                }
                before[i][threadIdx.x] = p;
                in.x[i].anew();
                if (i % kGroup == kGroup - 1) apart();
            }
#pragma unroll
            for (int j = 0; j < V; ++j) in.before[j] = h[j];  // the state behind the run
        }
        anew(q);
        const int64_t last = s0 + kRun - 1;
        T *to_x = ln.template at<T>(a.dx) + last * a.dx.st, *to_g = ln.template at<T>(a.dg) + last * a.dg.st,
          *to_z = ln.template at<T>(a.dz) + last * a.dz.st;
        // (as the loads: a place that the workgroup shares, and the thread's from there)
        const int64_t behind = (int64_t)(kRun - 1) * (int64_t)sizeof(T);
        char *tile_x = nullptr, *tile_g = nullptr, *tile_z = nullptr;
        uint32_t off_x = 0, off_g = 0, off_z = 0;
        if constexpr (SCAN) {
            tile_x = ln.template tile<T>(a.dx, t) + behind * a.dx.st;
            tile_g = ln.template tile<T>(a.dg, t) + behind * a.dg.st;
            tile_z = ln.template tile<T>(a.dz, t) + behind * a.dz.st;
            off_x = ln.template offset<T>(a.dx), off_g = ln.template offset<T>(a.dg), off_z = ln.template offset<T>(a.dz);
        }
        auto step = [&](int i, bool inside, bool stored, auto every) {
            float dx[V], dg[V], dz[V];
            const Pair p = before[i][threadIdx.x];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float D = mine[j] + brought(i, j), s = fabsf(q[i][j]), slope = fmaf(-s, s, s);
                dx[j] = inside ? gain_of<GAIN>(q[i][j]) * D : 0.0f;
                if (GAIN == kGainMean) dg[j] = D * slope * (p.v[j] - in.x[i].at(j));
                else dg[j] = D * fmaf(gain_slope<GAIN>(q[i][j]), in.x[i].at(j), slope * p.v[j]);
                dg[j] = inside ? dg[j] : 0.0f;
                if constexpr (Z) {
                    const float u = fabsf(qz[Z ? i : 0][j]);
                    dz[j] = inside ? in.dy[i].at(j) * in.before[j] * fmaf(-u, u, u) : 0.0f;
                }
                mine[j] = decay(D, q[i][j]);
                in.before[j] = p.v[j];
            }
            if constexpr (SCAN && every) {
                store_part<T, EVEN>((T*)(tile_x + off_x), ln.next, dx);
                store_part<T, EVEN>((T*)(tile_g + off_g), ln.next, dg);
                if constexpr (Z) store_part<T, EVEN>((T*)(tile_z + off_z), ln.next, dz);
                move_all(tile_x, -a.dx.st * (int64_t)sizeof(T));
                move_all(tile_g, -a.dg.st * (int64_t)sizeof(T));
                if constexpr (Z) move_all(tile_z, -a.dz.st * (int64_t)sizeof(T));
            } else {
                if (stored) {
                    if (every || a.dx.p) store_part<T, EVEN>(to_x, ln.next, dx);
                    if (every || a.dg.p) store_part<T, EVEN>(to_g, ln.next, dg);
                    if constexpr (Z)
                        if (every || a.dz.p) store_part<T, EVEN>(to_z, ln.next, dz);
                }
                move(to_x, -a.dx.st);
                move(to_g, -a.dg.st);
                if constexpr (Z) move(to_z, -a.dz.st);
            }
            if (i % kGroup == 0) apart();
        };
        // (every: all gradients are asked for)
        if (r.whole && a.dx.p && a.dg.p && (!Z || a.dz.p)) {
            if (ln.live) {
#pragma unroll
                for (int i = kRun - 1; i >= 0; --i) step(i, true, true, std::true_type{});
            }
        } else {
#pragma unroll
            for (int k = kRun - kGroup; k >= 0; k -= kGroup) {
                if (r.stores(k)) {
#pragma unroll
                    for (int i = k + kGroup - 1; i >= k; --i) step(i, i < r.left, ln.live && i < r.steps, std::false_type{});
                } else {
                    to_x -= kGroup * a.dx.st;
                    to_g -= kGroup * a.dg.st;
                    to_z -= kGroup * a.dz.st;
                }
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
template <typename T, bool EVEN, bool Z>
__global__ __launch_bounds__(kScanBlock) void k_recur_grad_maps(RecurArgs a, RecurCut cut) {
    typedef Lane<V, true> L;
    __shared__ float maps[2][L::kWaves][L::kLanes][2 * V];
    const L ln(a, cut, 1);
    SplitMap<V> all;
    for (int t = ln.t0; t < ln.t1; ++t) {
        const Run r(a, ((int64_t)t * L::kSlots + ln.slot) * kRun, ln.count);
        Part<T> g[kRun], dy[kRun], z[kRun];
        ln.template load<T, EVEN>(a.g, r, t, g);
        ln.template load<T, EVEN>(a.dy, r, t, dy);
        if constexpr (Z) ln.template load<T, EVEN>(a.z, r, t, z);
        r.take_out(dy);
        if constexpr (Z) r.take_out(z);
        float qa[V], qb[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            Product P;
            float D = 0.0f;
#pragma unroll
            for (int i = kRun - 1; i >= 0; --i) {
                float q = gate_of(g[i].at(j));
                if (!r.whole) q = i < r.left ? q : 0.0f;
                const float d = dy[i].at(j);
                P.take(q);
                D = decay(D + (Z ? d * sigmoid(z[i].at(j)) : d), q);
            }
            qa[j] = P.gate();
            qb[j] = D;
        }
        JoinMaps<V, true, true>::all(qa, qb, maps, t & 1);
        if (ln.slot == 0) all.before(qa, qb);
    }
    if (ln.slot != 0 || !ln.live) return;
    if (ln.split == 1) keep_entry(ln, a, cut, a.dlast);
    all.store(ln, a, cut);
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
        const hipError_t e = recur_dispatch(a, [&](auto t, auto even, auto z) {
            hipLaunchKernelGGL((k_recur_grad_maps<decltype(t), decltype(even)::value, decltype(z)::value>), grid_dim(groups),
                               dim3(kScanBlock), 0, a.stream, a, cut);
            return hipGetLastError();
        });
        timing_end(tk, a.stream);
        if (e != hipSuccess) return e;
    }
    const int tk = timing_begin("recurrence_grad", a.stream);
    const hipError_t e = recur_dispatch(a, [&](auto t, auto even, auto z) {
        return by_gain(a.gain, [&](auto gain) {
            auto go = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid_dim(cut.groups), dim3(cut.blocks ? kScanBlock : kWalkBlock), 0, a.stream, a, cut);
            };
            if (cut.blocks) go(k_recur_grad<decltype(t), decltype(even)::value, decltype(z)::value, decltype(gain)::value, true>);
            else go(k_recur_grad<decltype(t), decltype(even)::value, decltype(z)::value, decltype(gain)::value, false>);
            return hipGetLastError();
        });
    });
    timing_end(tk, a.stream);
    return e;
}

}  // namespace disco
