// disco_recur.h -- parts shared by the kernels of the gated recurrence and of its
// gradients.
//
//   h_t = a_t h_(t-1) + c_t x_t,  a = sigmoid(g),  c = 1 - a (mean), sqrt(1 - a^2)
//   (power) or 1 (one).
//
// A gate is held as q: |q| is the smaller of a and 1 - a, its sign bit is set where
// that is a.  A state multiplied by an a near 1 is taken as h - (1 - a) h, so
// that 1 - a keeps all its bits however long the memory is.
//
// A thread holds a run of 16 steps of V channels.  The map of states over some steps
// is h -> A h + B, and a run's is joined with the others' without knowing the state
// before it.  A is held as a gate is: over a long memory the products that
// round near 1 alike would drift (gates of 12, 40000 steps: 6e-5; so 1e-7).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <numeric>
#include <type_traits>

#include "disco_blocks.h"

namespace disco {

constexpr int kWalkBlock = 256;  // threads of a workgroup whose threads walk alone
constexpr int kScanBlock = 512;  // of one that scans
constexpr int kRecurBlock = 64;  // channels of a workgroup that scans along time
constexpr int kMaxSplits = 64;

constexpr int kRecurChannels = 2;  // of a thread: see Part

// How a call is cut.  scan: workgroups of 64 channels whose threads hold
// consecutive runs and join their maps, `splits` of them share the time axis;
// otherwise a thread walks all runs of its V channels by itself.
struct RecurCut {
    uint32_t columns;   // groups of V channels; of items too far apart (scan) with the empty ones that fill up the last block
    uint32_t blocks;    // of 32 groups, over all items (scan)
    uint32_t groups;    // workgroups
    int32_t splits, tiles;  // tiles of all runs; a split takes every tiles / splits
    Divisor by_columns;
    float* maps;   // [splits][batch][channels][2]
    float* entry;  // [batch][channels]: the state that the call is given, which its result may overwrite
};

__device__ __forceinline__ float gate_of(float g) {
    const float e = __builtin_amdgcn_exp2f(-1.44269504f * fabsf(g));
    const float q = e * __builtin_amdgcn_rcpf(1.0f + e);
    return __uint_as_float(__float_as_uint(q) | (__float_as_uint(g) & 0x80000000u));
}
__device__ __forceinline__ bool closed(float q) { return __float_as_int(q) < 0; }  // a is the smaller
__device__ __forceinline__ float decay(float h, float q) { return fmaf(-q, h, closed(q) ? 0.0f : h); }
// A product A of a's step by step, and 1 - A as the sum of what each step takes.  The sum is
// asked for only where A is not below 1/2, that is where no a was: a step with an a below 1/2 need not
// be right in it.
struct Product {
    float a = 1.0f, rest = 0.0f;
    __device__ __forceinline__ void take(float q) {
        rest = fmaf(fabsf(q), a, rest);
        a = decay(a, q);
    }
    // As a gate.
    __device__ __forceinline__ float gate() const { return a < 0.5f ? -a : rest; }
};
// The product of two such.
__device__ __forceinline__ float joined(float p, float q) {
    const float s = fabsf(p), r = fabsf(q);
    if (!closed(p) && !closed(q)) {
        const float rest = fmaf(r, 1.0f - s, s);
        return rest <= 0.5f ? rest : rest - 1.0f;
    }
    return -((closed(p) ? s : 1.0f - s) * (closed(q) ? r : 1.0f - r));
}
template <int GAIN>
__device__ __forceinline__ float gain_of(float q) {
    const float s = fabsf(q);
    if (GAIN == kGainMean) return closed(q) ? 1.0f - s : s;
    if (GAIN == kGainPower) return __builtin_amdgcn_sqrtf(closed(q) ? fmaf(-s, s, 1.0f) : s * (2.0f - s));
    return 1.0f;
}
template <int GAIN>
__device__ __forceinline__ float advance(float h, float q, float x) {
    if (GAIN == kGainMean) {  // the one of h and x that weighs more, and the other's share
        const float s = fabsf(q), p = closed(q) ? x : h, o = closed(q) ? h : x;
        return fmaf(s, o, fmaf(-s, p, p));
    }
    if (GAIN == kGainPower) return fmaf(gain_of<GAIN>(q), x, decay(h, q));
    return decay(h, q) + x;
}
__device__ __forceinline__ float sigmoid(float z) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * z));
}

// A step of a run that is scanned.  fp32 takes a gate as above; bf16, where the vector operations
// show in the time (half of the cycles issue one), as a and 1 - a, each with a relative error of fp32 however small
// it is: over the 16 steps of a run the roundings of an a near 1 come to 16 x 2^-25 of a state at most, and from run to run the
// map has 1 - A as a sum.  One series of 131072 x 768 takes 250 us as fp32 takes it and 238 so.
template <typename T>
struct Step;
template <>
struct Step<float> {
    float q;
    __device__ __forceinline__ explicit Step(float g) : q(gate_of(g)) {}
    __device__ __forceinline__ void onto(Product& p) const { p.take(q); }
    template <int GAIN>
    __device__ __forceinline__ float advance(float h, float x) const { return disco::advance<GAIN>(h, q, x); }
};
template <>
struct Step<__bf16> {
    float a, rest;
    __device__ __forceinline__ explicit Step(float g) {
        const float e = __builtin_amdgcn_exp2f(-1.44269504f * fabsf(g));
        const float most = __builtin_amdgcn_rcpf(1.0f + e), least = e * most;
        a = g < 0.0f ? least : most;
        rest = g < 0.0f ? most : least;
    }
    __device__ __forceinline__ void onto(Product& p) const {
        p.rest = fmaf(rest, p.a, p.rest);
        p.a *= a;
    }
    template <int GAIN>
    __device__ __forceinline__ float advance(float h, float x) const {
        if (GAIN == kGainMean) return fmaf(a, h, rest * x);
        if (GAIN == kGainPower) return fmaf(a, h, __builtin_amdgcn_sqrtf(fmaf(-rest, rest, rest + rest)) * x);
        return fmaf(a, h, x);
    }
};

// Two neighbouring channels as they lie: bf16 in one register (as single values, once
// branches meet, they take one each).
template <typename T>
struct Part;
template <>
struct Part<__bf16> {
    uint32_t u;
    __device__ __forceinline__ float at(int j) const { return __uint_as_float(j ? u & 0xffff0000u : u << 16); }
    __device__ __forceinline__ void clear_unless(bool in) { u = in ? u : 0u; }
    __device__ __forceinline__ void hold_unless(bool in) { u = in ? u : 0x7f807f80u; }
    // A new value to the compiler: what is converted is then converted again, instead of kept.
    __device__ __forceinline__ void anew() { asm("" : "+v"(u)); }
};
template <>
struct Part<float> {
    float v[2];
    __device__ __forceinline__ float at(int j) const { return v[j]; }
    __device__ __forceinline__ void clear_unless(bool in) { v[0] = in ? v[0] : 0.0f, v[1] = in ? v[1] : 0.0f; }
    __device__ __forceinline__ void hold_unless(bool in) { v[0] = in ? v[0] : HUGE_VALF, v[1] = in ? v[1] : HUGE_VALF; }
    __device__ __forceinline__ void anew() {}
};
// A thread's two channels of a row.  EVEN: rows have an even number of channels, and the
// two go together; otherwise one by one, the second `next` entries from the first: 1, or 0
// in the thread of the last channel, which is alone.
template <typename T, bool EVEN>
__device__ __forceinline__ Part<T> load_part(const T* p, int next) {
    Part<T> r;
    if constexpr (sizeof(T) == 2) {
        if constexpr (EVEN) {
            r.u = *(const Any1*)p;
        } else {
            const uint32_t lo = *(const uint16_t*)p, hi = *(const uint16_t*)(p + next);
            r.u = lo | hi << 16;
        }
    } else if constexpr (EVEN) {
        const Any2f v = *(const Any2f*)p;
        r.v[0] = v[0], r.v[1] = v[1];
    } else {
        r.v[0] = p[0], r.v[1] = p[next];
    }
    return r;
}
template <typename T, bool EVEN>
__device__ __forceinline__ void store_part(T* p, int next, const float (&v)[2]) {
    if constexpr (!EVEN) {
        p[0] = (T)v[0];
        p[next] = (T)(next ? v[1] : v[0]);
    } else if constexpr (sizeof(T) == 2) {
        typedef float F __attribute__((ext_vector_type(2)));
        typedef __bf16 B __attribute__((ext_vector_type(2)));
        *(Any1*)p = __builtin_bit_cast(uint32_t, __builtin_convertvector((F{v[0], v[1]}), B));
    } else {
        *(Any2f*)p = Any2f{v[0], v[1]};
    }
}

// The gates as new values: what is derived from them is then derived again, instead
// of kept from one pass over a run to the next (conditions too, in scalar registers).
template <int N, int V>
__device__ __forceinline__ void anew(float (&q)[N][V]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) asm("" : "+v"(q[i][j]));
}

// The next step's place.  (A new value each time: sums of the first place and multiples
// of the stride, made ahead, take two registers a step.)
template <typename T>
__device__ __forceinline__ void move(T*& p, int64_t by) {
    p += by;
    asm("" : "+v"(p));
}

// The same for a place that all threads share, in bytes.
template <typename P>
__device__ __forceinline__ void move_all(P& p, int64_t by) {
    p += by;
    asm("" : "+s"(p));
}

// The run of a thread: 16 steps from s0 on, of which the item has `left` and the
// tensors `steps`.  Whole runs go without conditions; of the others a wave takes
// the groups of four steps in which one of its threads has any.  Their loads stop at the item's last
// step (an item without any reads its first, which memory has); what lies beyond is
// taken out.
constexpr int kGroup = 4;
struct Run {
    int64_t first;  // step that the loads begin at
    int left, steps;
    bool whole;     // of all the wave's threads
    __device__ __forceinline__ Run() {}
    __device__ __forceinline__ Run(const RecurArgs& a, int64_t s0, int64_t count) {
        const int64_t n = count - s0, m = a.steps - s0;
        left = n < 0 ? 0 : n > kRun ? kRun : (int)n;
        steps = m < 0 ? 0 : m > kRun ? kRun : (int)m;
        first = left > 0 ? s0 : count > 0 ? count - 1 : 0;
        whole = __all(left == kRun);
    }
    __device__ __forceinline__ bool stores(int i) const { return whole || __any(i < steps); }
    // Of whole runs `from`, a workgroup's first step, goes on through scalar registers, `off` (bytes) is
    // the thread's place from there (scan); otherwise p is its own.
    template <typename T, bool EVEN, bool SCAN>
    __device__ __forceinline__ void load(const T* p, const char* from, uint32_t off, int64_t st, int next,
                                         Part<T> (&v)[kRun]) const {
        if (whole) {
            if constexpr (SCAN) {
#pragma unroll
                for (int i = 0; i < kRun; ++i) {
                    v[i] = load_part<T, EVEN>((const T*)(from + off), next);
                    move_all(from, st * (int64_t)sizeof(T));
                }
            } else {
                p += first * st;
#pragma unroll
                for (int i = 0; i < kRun; ++i) {
                    v[i] = load_part<T, EVEN>(p, next);
                    move(p, st);
                }
            }
            return;
        }
        p += first * st;
#pragma unroll
        for (int k = 0; k < kRun; k += kGroup) {
            if (__any(k < left)) {
#pragma unroll
                for (int i = k; i < k + kGroup; ++i) {
                    v[i] = load_part<T, EVEN>(p, next);
                    move(p, i + 1 < left ? st : 0);
                }
            } else {
#pragma unroll
                for (int i = k; i < k + kGroup; ++i) v[i] = Part<T>{};
            }
        }
    }
    // Zeros for the steps that the item has not.
    template <typename T>
    __device__ __forceinline__ void take_out(Part<T> (&v)[kRun]) const {
        if (whole) return;
#pragma unroll
        for (int i = 0; i < kRun; ++i) v[i].clear_unless(i < left);
    }
    // Their gates leave a state as it is: +inf before the sigmoid, q = 0 behind it.
    template <typename T>
    __device__ __forceinline__ void hold(Part<T> (&g)[kRun]) const {
        if (whole) return;
#pragma unroll
        for (int i = 0; i < kRun; ++i) g[i].hold_unless(i < left);
    }
    template <int V>
    __device__ __forceinline__ void take_out(float (&q)[kRun][V]) const {
        if (whole) return;
#pragma unroll
        for (int i = 0; i < kRun; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) q[i][j] = i < left ? q[i][j] : 0.0f;
    }
};

// Where a thread works: its channels, and the runs it takes.
template <int V, bool SCAN>
struct Lane {
    static constexpr int kThreads = SCAN ? kScanBlock : kWalkBlock;
    static constexpr int kLanes = kRecurBlock / V;              // threads of a step (scan)
    static constexpr int kSlots = SCAN ? kThreads / kLanes : 1; // runs of a tile
    static constexpr int kInWave = 64 / kLanes;                 // of them in a wave
    static constexpr int kWaves = kThreads / 64;
    uint32_t b, b0;  // batch item; of the workgroup's first thread (scan)
    int64_t c;       // first channel
    int next;        // see load_part
    int slot, split;
    bool live;       // has channels
    int64_t count;   // steps of this item
    int t0, t1;      // tiles
    __device__ __forceinline__ Lane(const RecurArgs& a, const RecurCut& cut, int first_split = 0) {
        const uint32_t all = cut.columns * a.batch;
        uint32_t column;
        if constexpr (SCAN) {
            const uint32_t id = group_index(), block = id % cut.blocks;
            split = first_split + (int)(id / cut.blocks);
            slot = threadIdx.x / kLanes;
            b0 = cut.by_columns.quotient(block * kLanes);
            column = block * kLanes + threadIdx.x % kLanes;
            live = column < all && split < cut.splits;
            t0 = (int)((int64_t)cut.tiles * split / cut.splits);
            t1 = split < cut.splits ? (int)((int64_t)cut.tiles * (split + 1) / cut.splits) : t0;
        } else {
            column = group_index() * kThreads + threadIdx.x;
            live = column < all;
            slot = split = 0;
            t0 = 0;
            t1 = live ? cut.tiles : 0;
        }
        column = min(column, all - 1);  // threads without channels read the last ones and write nothing
        b = cut.by_columns.quotient(column);
        if constexpr (!SCAN) b0 = b;
        c = (int64_t)(column - b * cut.columns) * V;
        if (SCAN && c >= a.channels) {  // reads the last ones and writes nothing
            live = false;
            c = (a.channels - 1) / V * V;
        }
        next = c + 1 < a.channels ? 1 : 0;
        count = a.steps;
        if (a.lengths) {
            const int64_t n = a.lengths[b];
            count = n < 0 ? 0 : n < count ? n : count;
        }
    }
    template <typename T>
    __device__ __forceinline__ T* at(const Rows& r) const {
        return (T*)r.p + b * r.sb + c;
    }
    // The first step of tile t in a tensor, of the workgroup's first item, and the thread's place from there
    // in bytes (scan).
    template <typename T>
    __device__ __forceinline__ char* tile(const Rows& r, int t) const {
        return (char*)((T*)r.p + (int64_t)b0 * r.sb + (int64_t)t * kSlots * kRun * r.st);
    }
    template <typename T>
    __device__ __forceinline__ uint32_t offset(const Rows& r) const {
        return ((b - b0) * (uint32_t)r.sb + slot * kRun * (uint32_t)r.st + (uint32_t)c) * (uint32_t)sizeof(T);
    }
    template <typename T, bool EVEN>
    __device__ __forceinline__ void load(const Rows& r, const Run& run, int t, Part<T> (&v)[kRun]) const {
        run.template load<T, EVEN, SCAN>(at<const T>(r), SCAN ? tile<T>(r, t) : nullptr, SCAN ? offset<T>(r) : 0, r.st, next, v);
    }
    // The place of this thread's channels in a [batch][channels] array.
    __device__ __forceinline__ int64_t state_at(const RecurArgs& a) const { return (int64_t)b * a.channels + c; }
};

// fp32 values of a thread's channels (one by one: channels may be odd).
template <int V>
__device__ __forceinline__ void load_state(const float* p, int64_t at, int64_t c, int64_t n, bool live, float (&h)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = p && live && c + j < n ? p[at + j] : 0.0f;
}
template <int V>
__device__ __forceinline__ void store_state(float* p, int64_t at, int64_t c, int64_t n, bool live, const float (&h)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (live && c + j < n) p[at + j] = h[j];
}

// Joins the maps of a workgroup's runs: gives each thread the state before
// its own (after its own, looking backwards) from that before the tile, `h`, and leaves in h the
// state behind the tile.  One barrier a tile; the buffers take turns.
template <int V, bool SCAN, bool BACK>
struct JoinMaps {
    typedef Lane<V, SCAN> L;
    __device__ __forceinline__ static void run(float (&A)[V], float (&B)[V], float (&h)[V], float (&mine)[V],
                                               float (*maps)[L::kWaves][L::kLanes][2 * V], int turn) {
        in_wave(A, B, maps, turn);
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = threadIdx.x % L::kLanes;
        const int order = BACK ? L::kInWave - 1 - lane / L::kLanes : lane / L::kLanes;
        // of the runs before this one in the wave
        float ea[V], eb[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int from = BACK ? lane + L::kLanes : lane - L::kLanes;
            const float a = __shfl(A[j], from), b = __shfl(B[j], from);
            ea[j] = order ? a : 0.0f;
            eb[j] = order ? b : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < L::kWaves; ++k) {
            const int w = BACK ? L::kWaves - 1 - k : k;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (w == wave) mine[j] = decay(h[j], ea[j]) + eb[j];
                h[j] = decay(h[j], maps[turn][w][col][j]) + maps[turn][w][col][V + j];
            }
        }
    }
    // The tile's own map, in the first wave's threads.
    __device__ __forceinline__ static void all(float (&A)[V], float (&B)[V], float (*maps)[L::kWaves][L::kLanes][2 * V], int turn) {
        in_wave(A, B, maps, turn);
        __syncthreads();
        if (threadIdx.x >= 64) return;
        const int col = threadIdx.x % L::kLanes;
#pragma unroll
        for (int k = 0; k < L::kWaves; ++k) {
            const int w = BACK ? L::kWaves - 1 - k : k;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float a = maps[turn][w][col][j], b = maps[turn][w][col][V + j];
                B[j] = k ? decay(B[j], a) + b : b;
                A[j] = k ? joined(A[j], a) : a;
            }
        }
    }

private:
    // Joins the maps of a wave's runs with those before them in it, and leaves the wave's.
    __device__ __forceinline__ static void in_wave(float (&A)[V], float (&B)[V], float (*maps)[L::kWaves][L::kLanes][2 * V], int turn) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = threadIdx.x % L::kLanes;
        const int at = lane / L::kLanes;  // place in the wave
        const int order = BACK ? L::kInWave - 1 - at : at;
#pragma unroll
        for (int d = 1; d < L::kInWave; d *= 2) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int from = BACK ? lane + d * L::kLanes : lane - d * L::kLanes;
                const float a = __shfl(A[j], from), b = __shfl(B[j], from);
                if (order >= d) {
                    B[j] += decay(b, A[j]);
                    A[j] = joined(A[j], a);
                }
            }
        }
        if (order == L::kInWave - 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                maps[turn][wave][col][j] = A[j];
                maps[turn][wave][col][V + j] = B[j];
            }
        }
    }
};

// Where a call has splits, the first kernel keeps the given state for the second.
template <typename L>
__device__ __forceinline__ void keep_entry(const L& ln, const RecurArgs& a, const RecurCut& cut, const float* given) {
    float h[kRecurChannels];
    load_state(given, ln.state_at(a), ln.c, a.channels, ln.live, h);
    store_state(cut.entry, ln.state_at(a), ln.c, a.channels, ln.live, h);
}

// A split's map from those of its tiles, taken in the order opposite to that in which the
// call then goes through them, so that it finds the last read ones in the caches.
template <int V>
struct SplitMap {
    float A[V] = {0.0f}, B[V] = {0.0f};
    // The map of a tile that comes before those taken so far.
    __device__ __forceinline__ void before(const float (&a)[V], const float (&b)[V]) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            B[j] += decay(b[j], A[j]);
            A[j] = joined(A[j], a[j]);
        }
    }
    template <typename L>
    __device__ __forceinline__ void store(const L& ln, const RecurArgs& a, const RecurCut& cut) const {
        float* out = cut.maps + 2 * ((int64_t)ln.split * a.batch * a.channels + ln.state_at(a));
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (ln.c + j < a.channels) {
                out[2 * j] = A[j];
                out[2 * j + 1] = B[j];
            }
    }
};

// The state before split `split` (behind it, looking backwards) from that at the
// ends of the series.
template <int V, bool BACK>
__device__ __forceinline__ void through_splits(const RecurArgs& a, const RecurCut& cut, int split, int64_t at, int64_t c,
                                               bool live, float (&h)[V]) {
    const int64_t all = (int64_t)a.batch * a.channels;
    const int n = BACK ? cut.splits - 1 - split : split;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const int s = BACK ? cut.splits - 1 - i : i;
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (live && c + j < a.channels) {
                const float* m = cut.maps + 2 * (s * all + at + j);
                h[j] = decay(h[j], m[0]) + m[1];
            }
    }
}

// Whether a workgroup's threads reach all that they scan with 32-bit offsets from its first item's channels: `steps`
// steps and `items` items on.
inline bool within_reach(const RecurArgs& a, int64_t steps, int64_t items) {
    const int64_t most = ((int64_t)1 << 31) / (a.bf16 ? 2 : 4);
    for (const Rows* t : {&a.x, &a.g, &a.z, &a.y, &a.dy, &a.dx, &a.dg, &a.dz}) {
        if (!t->p) continue;
        if (t->st > most / steps || (items > 0 && t->sb > most / items) || t->st * steps + t->sb * items + a.channels > most) return false;
    }
    return true;
}

// Whether threads walk alone: where there are enough of them, few steps, or steps so far
// apart that a tile has no 32-bit offsets.  A tile of 256 steps is half idle on 80 steps, but a
// walk's runs wait for each other.  Forward and gradients, walking and scanning: 3221 x 76 x 16 18 + 27 and
// 20 + 39 us; 64 x 48 x 512 11 + 16 and 12 + 25; 1024 x 64 x 16 13 + 19 and 9 + 14; 100 x 128 x 512 24 + 37
// and 18 + 36; 32 x 128 x 512 20 + 34 and 9 + 15.  At the border of 65536 threads, whole steps of 256 x T x 512 in bf16:
// T = 100 65 and 94 us, 128 80 and 95, 512 308 and 284 (412 and 412 with an output gate, 427 and 445 in fp32), 2048 1231 and 992:
// from some hundred steps on the scan is ahead there; with four times the threads the walk still is (1024 x 512 x 512 870
// and 1032).
constexpr uint32_t kWalkThreads = 65536;
constexpr int64_t kTileSteps = (int64_t)kScanBlock / (kRecurBlock / kRecurChannels) * kRun;
inline bool walks(const RecurArgs& a) {
    const int64_t all = a.batch * ((a.channels + kRecurChannels - 1) / kRecurChannels);
    return a.steps <= 2 * kRun || all >= kWalkThreads || (a.steps <= 5 * kRun && all >= kWalkThreads / 4) ||
           !within_reach(a, kTileSteps, 0);
}
constexpr uint32_t kScanGroups = 512;
inline RecurCut recur_cut(const RecurArgs& a) {
    constexpr uint32_t v = kRecurChannels, lanes = kRecurBlock / v, slots = kScanBlock / lanes;
    RecurCut c{};
    c.columns = (uint32_t)((a.channels + v - 1) / v);
    const int64_t runs = (a.steps + kRun - 1) / kRun;
    const bool walk = walks(a);
    // Blocks begin at multiples of gcd(columns, lanes) within an item.  Of items that a block would span beyond its reach each
    // takes blocks of its own.
    const int64_t spans = (c.columns - std::gcd(c.columns, lanes) + lanes - 1) / c.columns;
    if (!walk && !within_reach(a, kTileSteps, std::min<int64_t>(a.batch - 1, spans))) c.columns = (c.columns + lanes - 1) / lanes * lanes;
    c.by_columns = divisor(c.columns);
    const int64_t all = (int64_t)c.columns * a.batch;
    c.splits = 1;
    if (walk) {
        c.tiles = (int32_t)runs;
        c.groups = (uint32_t)((all + kWalkBlock - 1) / kWalkBlock);
        return c;
    }
    c.tiles = (int32_t)((runs + slots - 1) / slots);
    c.blocks = (uint32_t)((all + lanes - 1) / lanes);
    // Split, at the price of the second read, into as many workgroups as the forward call without an output gate holds: two a
    // CU by its registers (768 gained nothing).  The gated forward call and all gradients hold one a CU, so that between 129 and 191
    // blocks their parts go in two rounds.  Whole steps of B x 2048 x 960, in bf16 without and with an output gate and in fp32, as it is and
    // unsplit: 105 blocks 95 and 107, 129 and 142, 148 and 150 us; 135 123 and 113; 150 127 and 116, 172 and 153; 180 153 and
    // 123, 212 and 159, 228 and 181: from some 130 blocks on a call would be better left whole.
    if (c.blocks < 192)
        c.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>({(int64_t)(kScanGroups / c.blocks), (int64_t)c.tiles, (int64_t)kMaxSplits}));
    c.groups = c.blocks * (uint32_t)c.splits;
    return c;
}

// Calls f with the storage type, whether rows have an even number of channels, and
// whether there is an output gate.
template <typename F>
hipError_t recur_dispatch(const RecurArgs& a, F&& f) {
    auto gated = [&](auto t, auto even) {
        return a.z.p ? f(t, even, std::true_type{}) : f(t, even, std::false_type{});
    };
    auto type = [&](auto t) { return a.channels % 2 == 0 ? gated(t, std::true_type{}) : gated(t, std::false_type{}); };
    return a.bf16 ? type(__bf16{}) : type(float{});
}

inline void recur_ws(RecurCut* cut, const RecurArgs& a, float* ws) {
    cut->maps = ws;
    cut->entry = ws ? ws + (int64_t)cut->splits * a.batch * a.channels * 2 : nullptr;
}

template <typename F>
hipError_t by_gain(int gain, F&& f) {
    if (gain == kGainMean) return f(std::integral_constant<int, kGainMean>{});
    if (gain == kGainPower) return f(std::integral_constant<int, kGainPower>{});
    return f(std::integral_constant<int, kGainOne>{});
}

}  // namespace disco
