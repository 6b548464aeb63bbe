// disco_residual.hip -- the residual sum of a block with the norms before and
// after it, its gate and dropout, and its gradients.
//
//   n1 = f / rms(f),  u = w1 n1 (or f),  d = drop(u),  h = scale x + gate d,
//   n2 = h / rms(h),  y = w2 n2,         rms(v) = sqrt(mean v^2 + eps);
//   t = w2 dy,  D = dh + (t - n2 mean(t n2)) / rms(h),  dx = scale D,
//   du = drop(gate D),  t = w1 du,  df = (t - n1 mean(t n1)) / rms(f),
//   dw1 = sum du n1,  dgate = sum D d,  dw2 = sum dy n2.
//
// A few operations an entry: the bound is the memory's rate, so every tensor is
// read or written once and a row stays in registers from its loads to its stores.
// The gradients recompute h and both norms from x and f, which costs no byte more
// than reading a stored h, and leaves h and y without a rounding between them:
// y is taken from h before its rounding to bf16.  Rows of up to 512 entries in the
// gradients (2048 forward) lie in one wave, whose lanes share the sums by shuffles;
// longer ones in a workgroup.  A thread holds chunks of eight entries, the
// share of one block of the dropout's generator.  All sums are fp32.
//
// The gradients of the weights are summed in a fixed order: each workgroup walks
// a run of rows and leaves one partial row a sum (one an item for weights of
// [batch, channels]), which k_residual_join adds.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "disco_blocks.h"
#include "disco_internal.h"

namespace disco {

namespace {

constexpr int kThreads = 256;
constexpr int kWave = 64;

// lanes: threads of a row (a power of two; beyond a wave the whole workgroup);
// nv: chunks of a thread; slots: rows of a workgroup at a time.
struct Shape {
    int lanes, nv, threads, slots;
    uint32_t rows, items, groups, per_group;  // per_group: rows of a workgroup's run (gradients)
    Divisor tokens;
};

// Sum over a row's threads.  Within a wave by shuffles, beyond through `red`, two
// buffers in turn.
__device__ __forceinline__ float row_sum(float v, int lanes, float (*red)[1024 / kWave], int& turn) {
    const int within = min(lanes, kWave);
    for (int m = 1; m < within; m <<= 1) v += __shfl_xor(v, m);
    if (lanes <= kWave) return v;
    turn ^= 1;
    if ((threadIdx.x & (kWave - 1)) == 0) red[turn][threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0f;
    for (int i = 0; i < lanes / kWave; ++i) v += red[turn][i];
    return v;
}

// A row's values, brought into the range whose squares fp32 holds, and what they
// are multiplied by to be normed.
template <int N>
__device__ __forceinline__ float norm_factor(float (&e)[N], const ResidualArgs& a, float ss, int lanes,
                                             float (*red)[1024 / kWave], int& turn, float* up) {
    const float inv = 1.0f / (float)a.channels;
    float eps = a.eps;
    const float f = row_scale(ss, inv, eps);
    *up = f;
    if (__any(f != 1.0f)) {  // (the same in all waves of a row)
        ss = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            e[i] *= f;
            ss = fmaf(e[i], e[i], ss);
        }
        ss = row_sum(ss, lanes, red, turn);
        eps = f > 1.0f ? a.eps_up : a.eps * f * f;
    }
    return rsqrtf(fmaf(ss, inv, eps));
}

template <int N>
__device__ __forceinline__ float squares(const float (&e)[N]) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = fmaf(e[i], e[i], s);
    return s;
}

template <typename T>
__device__ __forceinline__ T* row_of(const Rows& t, uint32_t b, uint32_t tok) {
    return (T*)t.p + b * t.sb + tok * t.st;
}

// What is not there is taken as zeros (or ones): the arithmetic has no branches but
// around sums over a row.
template <typename T, int W>
__device__ __forceinline__ Raw<T> load_part(const Rows& t, uint32_t b, uint32_t tok, int c, int n) {
    return load_raw<T, W>(row_of<const T>(t, b, tok), c, t.p ? n : 0);
}
template <typename T, int W>
__device__ __forceinline__ Raw<T> load_weight(const void* w, int64_t sb, uint32_t b, int c, int n) {
    return load_raw<T, W>((const T*)w + b * sb, c, w ? n : 0, 1.0f);
}

template <typename T, int NV, int W>
__global__ __launch_bounds__(kThreads) void k_residual(ResidualArgs a, Shape s) {
    __shared__ float red[2][1024 / kWave];
    const int lane = threadIdx.x & (s.lanes - 1), slot = threadIdx.x / s.lanes, C = a.channels;
    int turn = 0;
    const uint64_t offset = a.dropped ? drop_offset(a.drop) : 0;
    for (uint64_t first = (uint64_t)blockIdx.x * s.slots; first < s.rows; first += (uint64_t)s.groups * s.slots) {
        const bool live = first + slot < s.rows;
        const uint32_t row = live ? (uint32_t)(first + slot) : 0;
        const uint32_t b = s.tokens.quotient(row), tok = row - b * s.tokens.d;
        const int n = live ? C : 0;
        Raw<T> x[NV];
        float e[NV * kChunk];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (lane + s.lanes * j) * kChunk;
            const Raw<T> f = load_part<T, W>(a.f, b, tok, c, n);
            x[j] = load_part<T, W>(a.x, b, tok, c, n);
#pragma unroll
            for (int i = 0; i < kChunk; ++i) e[j * kChunk + i] = (float)f.v[i];
        }
        float r = 1.0f, up;
        if (a.post) r = norm_factor(e, a, row_sum(squares(e), s.lanes, red, turn), s.lanes, red, turn, &up);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int chunk = lane + s.lanes * j, c = chunk * kChunk;
            float* u = e + j * kChunk;
            float v[kChunk];
            const Raw<T> w = load_weight<T, W>(a.post_w, a.post_sb, b, c, n);
            const Raw<T> g = load_weight<T, W>(a.gate, a.gate_sb, b, c, n);
            const uint32_t keep = a.dropped ? kept(a.drop, offset, row, chunk) : 0xffu;
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                const float d = keep >> i & 1 ? u[i] * r * (float)w.v[i] * a.drop.factor : 0.0f;
                u[i] = fmaf(a.scale, (float)x[j].v[i], d * (float)g.v[i]);
                v[i] = u[i];
            }
            if (a.h.p) store_row<T, W>(row_of<T>(a.h, b, tok), c, n, v);
        }
        if (!a.y.p) continue;
        r = norm_factor(e, a, row_sum(squares(e), s.lanes, red, turn), s.lanes, red, turn, &up);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (lane + s.lanes * j) * kChunk;
            const Raw<T> w = load_weight<T, W>(a.next_w, a.next_sb, b, c, n);
            float v[kChunk];
#pragma unroll
            for (int i = 0; i < kChunk; ++i) v[i] = e[j * kChunk + i] * r * (float)w.v[i];
            store_row<T, W>(row_of<T>(a.y, b, tok), c, n, v);
        }
    }
}

// The three sums over rows.
enum { kPost, kGate, kNext, kSums };
// Where a sum's partial rows go: rows of C floats from `at` on.  One a workgroup
// where the weight is shared; otherwise the run's part of item b is row
// workgroup + b (both only grow along the rows, so no two parts share one).
struct Partial {
    float* at;
    bool per_item;
};
struct Partials {
    Partial p[kSums];
    bool any_item;
};

// (A row's chunk a thread: with two, 138 registers spill.)
template <typename T, int W, int THREADS>
__global__ __launch_bounds__(THREADS) void k_residual_grad(ResidualArgs a, Shape s, Partials ps) {
    __shared__ float red[2][1024 / kWave];
    __shared__ float sums[kThreads * kChunk];
    constexpr int N = kChunk;
    const int lane = threadIdx.x & (s.lanes - 1), slot = threadIdx.x / s.lanes, C = a.channels, c = lane * kChunk;
    const float inv = 1.0f / (float)C;
    int turn = 0;
    const uint64_t offset = a.dropped ? drop_offset(a.drop) : 0;
    float acc[kSums][N];
#pragma unroll
    for (int k = 0; k < kSums; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) acc[k][i] = 0.0f;
    // Leaves the workgroup's sum k in a partial row, the slots' in slot order.
    auto flush = [&](int k, uint32_t at) {
        float* out = ps.p[k].at + (int64_t)at * C;
        if (s.slots == 1) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (c + i < C) out[c + i] = acc[k][i];
        } else {
            const int per = s.lanes * N;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) sums[slot * per + c + i] = acc[k][i];
            __syncthreads();
            for (int d = threadIdx.x; d < min(per, C); d += s.threads) {
                float v = 0.0f;
                for (int sl = 0; sl < s.slots; ++sl) v += sums[sl * per + d];
                out[d] = v;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) acc[k][i] = 0.0f;
    };
    const uint64_t begin = (uint64_t)blockIdx.x * s.per_group, end = min(begin + s.per_group, (uint64_t)s.rows);
    for (uint64_t seg = begin; seg < end;) {
        const uint32_t item = s.tokens.quotient((uint32_t)seg);
        const uint64_t stop = ps.any_item ? min(end, (uint64_t)(item + 1) * s.tokens.d) : end;
        for (uint64_t first = seg; first < stop; first += s.slots) {
            const bool live = first + slot < stop;
            const uint32_t row = live ? (uint32_t)(first + slot) : (uint32_t)first;
            const uint32_t b = s.tokens.quotient(row), tok = row - b * s.tokens.d;
            const int n = live ? C : 0;
            const Raw<T> f = load_part<T, W>(a.f, b, tok, c, n), x = load_part<T, W>(a.x, b, tok, c, n);
            const Raw<T> dh = load_part<T, W>(a.dh, b, tok, c, n), dy = load_part<T, W>(a.dy, b, tok, c, n);
            float n1[N], h[N], D[N];
#pragma unroll
            for (int i = 0; i < N; ++i) n1[i] = (float)f.v[i];
            float r1 = 1.0f, up1 = 1.0f;
            if (a.post) {
                r1 = norm_factor(n1, a, row_sum(squares(n1), s.lanes, red, turn), s.lanes, red, turn, &up1);
#pragma unroll
                for (int i = 0; i < N; ++i) n1[i] *= r1;
                r1 *= up1;
            }
            const Raw<T> w = load_weight<T, W>(a.post_w, a.post_sb, b, c, n);
            const Raw<T> g = load_weight<T, W>(a.gate, a.gate_sb, b, c, n);
            const uint32_t keep = a.dropped ? kept(a.drop, offset, row, lane) : 0xffu;
            auto drop = [&](float v, int i) { return keep >> i & 1 ? v * a.drop.factor : 0.0f; };
#pragma unroll
            for (int i = 0; i < N; ++i) {
                h[i] = fmaf(a.scale, (float)x.v[i], drop(n1[i] * (float)w.v[i], i) * (float)g.v[i]);
            }
            if (a.dy.p) {
                float up2, m = 0.0f;
                const float r = norm_factor(h, a, row_sum(squares(h), s.lanes, red, turn), s.lanes, red, turn, &up2);
                const Raw<T> w2 = load_weight<T, W>(a.next_w, a.next_sb, b, c, n);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    h[i] *= r;  // n2
                    acc[kNext][i] = fmaf((float)dy.v[i], h[i], acc[kNext][i]);
                    m = fmaf((float)dy.v[i] * (float)w2.v[i], h[i], m);
                }
                m = row_sum(m, s.lanes, red, turn) * inv;
                const float r2 = r * up2;
#pragma unroll
                for (int i = 0; i < N; ++i) D[i] = fmaf(r2, fmaf(-m, h[i], (float)dy.v[i] * (float)w2.v[i]), (float)dh.v[i]);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) D[i] = (float)dh.v[i];
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                acc[kGate][i] = fmaf(D[i], drop(n1[i] * (float)w.v[i], i), acc[kGate][i]);
                h[i] = a.scale * D[i];
                D[i] = drop(D[i] * (float)g.v[i], i);  // du
            }
            if (a.dx.p) store_row<T, W>(row_of<T>(a.dx, b, tok), c, n, h);
            if (a.post) {
                float m = 0.0f;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    acc[kPost][i] = fmaf(D[i], n1[i], acc[kPost][i]);
                    D[i] *= (float)w.v[i];
                    m = fmaf(D[i], n1[i], m);
                }
                m = row_sum(m, s.lanes, red, turn) * inv;
#pragma unroll
                for (int i = 0; i < N; ++i) D[i] = r1 * fmaf(-m, n1[i], D[i]);
            }
            if (a.df.p) store_row<T, W>(row_of<T>(a.df, b, tok), c, n, D);
        }
#pragma unroll
        for (int k = 0; k < kSums; ++k)
            if (ps.p[k].at && ps.p[k].per_item) flush(k, blockIdx.x + item);
        seg = stop;
    }
#pragma unroll
    for (int k = 0; k < kSums; ++k)
        if (ps.p[k].at && !ps.p[k].per_item) flush(k, blockIdx.x);
}

struct SumJoin {
    const float* from;
    void* to;
    bool per_item;
};
struct Joins {
    SumJoin j[kSums];
};
constexpr int kJoinColumns = 16, kJoinSlices = 64;

// Adds the partial rows of a weight's gradient in a fixed order.  grid: (columns /
// 16, items, sums); 16 columns x 64 slices of the rows.
template <typename T>
__global__ __launch_bounds__(1024) void k_residual_join(Joins js, Shape s, int C) {
    __shared__ float red[kJoinSlices][kJoinColumns + 1];
    const SumJoin j = js.j[blockIdx.z];
    if (!j.to || (blockIdx.y > 0 && !j.per_item)) return;
    const int col = threadIdx.x % kJoinColumns, slice = threadIdx.x / kJoinColumns, c = blockIdx.x * kJoinColumns + col;
    for (uint32_t item = blockIdx.y; item < (j.per_item ? s.items : 1); item += gridDim.y) {
        uint32_t lo = 0, hi = s.groups;
        if (j.per_item) {  // rows workgroup + item of the runs that reach into the item
            const uint64_t r0 = (uint64_t)item * s.tokens.d;
            lo = (uint32_t)(r0 / s.per_group) + item;
            hi = s.rows ? (uint32_t)((r0 + s.tokens.d - 1) / s.per_group) + item + 1 : lo;
        }
        float v = 0.0f;
        if (c < C)
            for (uint32_t r = lo + slice; r < hi; r += kJoinSlices) v += j.from[(int64_t)r * C + c];
        __syncthreads();
        red[slice][col] = v;
        for (int m = kJoinSlices / 2; m > 0; m >>= 1) {
            __syncthreads();
            if (slice < m) red[slice][col] += red[slice + m][col];
        }
        if (slice == 0 && c < C) ((T*)j.to)[(int64_t)item * C + c] = (T)red[0][col];
    }
}

int width(const ResidualArgs& a) {
    const size_t e = a.bf16 ? 2 : 4;
    int w = a.bf16 ? 8 : 4;
    auto fits = [&](int v) {
        if (a.channels % v) return false;
        for (const void* p : {a.post_w, a.gate, a.next_w})
            if ((uintptr_t)p % (v * e)) return false;
        for (const Rows* t : {&a.x, &a.f, &a.h, &a.y, &a.dh, &a.dy, &a.dx, &a.df})
            if (!rows_fit(*t, v, e)) return false;
        return true;
    };
    while (w > 1 && !fits(w)) w /= 2;
    return w;
}

// most: chunks a thread holds at most; in a wave as few idle lanes as can be.
Shape shape_of(const ResidualArgs& a, int most) {
    Shape s{};
    const int chunks = (a.channels + kChunk - 1) / kChunk;
    if (chunks <= kWave * most) {
        int best = 0;
        for (int nv = 1; nv <= most; ++nv) {
            int lanes = 1;
            while (lanes * nv < chunks) lanes *= 2;
            if (lanes > kWave || (best && lanes * nv >= best)) continue;
            best = lanes * nv;
            s.lanes = lanes;
            s.nv = nv;
        }
        s.threads = kThreads;
    } else {
        s.lanes = 2 * kWave;
        while (s.lanes * most < chunks) s.lanes *= 2;
        s.nv = (chunks + s.lanes - 1) / s.lanes;
        s.threads = s.lanes;
    }
    s.slots = s.threads / s.lanes;
    s.rows = (uint32_t)(a.batch * a.tokens);
    s.items = a.batch;
    s.tokens = divisor((uint32_t)std::max<int64_t>(a.tokens, 1));
    return s;
}

constexpr int kForwardChunks = 4, kGradChunks = 1;
constexpr uint32_t kForwardThreads = 256 * 2048, kGradThreads = 256 * 1024;  // of a launch

Shape grad_shape(const ResidualArgs& a) {
    Shape s = shape_of(a, kGradChunks);
    const uint32_t most = kGradThreads / (uint32_t)s.threads;
    const uint32_t runs = std::max(1u, std::min((s.rows + s.slots - 1) / s.slots, most));
    s.per_group = std::max(1u, ((s.rows + runs - 1) / runs + s.slots - 1) / s.slots * s.slots);
    s.groups = std::max(1u, (s.rows + s.per_group - 1) / s.per_group);
    return s;
}

template <typename F>
hipError_t dispatch(const ResidualArgs& a, int nv, F&& f) {
    auto width_of = [&](auto t, auto n) {
        switch (width(a)) {
            case 8: return f(t, n, std::integral_constant<int, (sizeof(t) == 2 ? 8 : 4)>{});
            case 4: return f(t, n, std::integral_constant<int, 4>{});
            case 2: return f(t, n, std::integral_constant<int, 2>{});
            default: return f(t, n, std::integral_constant<int, 1>{});
        }
    };
    auto type = [&](auto n) { return a.bf16 ? width_of(__bf16{}, n) : width_of(float{}, n); };
    switch (nv) {
        case 1: return type(std::integral_constant<int, 1>{});
        case 2: return type(std::integral_constant<int, 2>{});
        case 3: return type(std::integral_constant<int, 3>{});
        default: return type(std::integral_constant<int, 4>{});
    }
}

struct Sum {
    const void* weight;
    void* to;
    int64_t sb;
};
void sums_of(const ResidualArgs& a, Sum (&s)[kSums]) {
    s[kPost] = Sum{a.post_w, a.dpost, a.post_sb};
    s[kGate] = Sum{a.gate, a.dgate, a.gate_sb};
    s[kNext] = Sum{a.next_w, a.dnext, a.next_sb};
}
// Partial rows of a weight's gradient.
size_t partial_rows(const ResidualArgs& a, const Shape& s, const Sum& u) { return (size_t)s.groups + (u.sb ? a.batch : 0); }

}  // namespace

hipError_t launch_residual(const ResidualArgs& a) {
    Shape s = shape_of(a, kForwardChunks);
    s.groups = std::min((s.rows + s.slots - 1) / s.slots, kForwardThreads / (uint32_t)s.threads);
    const int tk = timing_begin("residual_norm", a.stream);
    const hipError_t e = dispatch(a, s.nv, [&](auto t, auto n, auto w) {
        hipLaunchKernelGGL((k_residual<decltype(t), decltype(n)::value, decltype(w)::value>), dim3(s.groups),
                           dim3((unsigned)s.threads), 0, a.stream, a, s);
        return hipGetLastError();
    });
    timing_end(tk, a.stream);
    return e;
}

size_t residual_grad_ws_bytes(const ResidualArgs& a) {
    const Shape s = grad_shape(a);
    Sum u[kSums];
    sums_of(a, u);
    size_t rows = 0;
    for (const Sum& k : u)
        if (k.weight) rows += partial_rows(a, s, k);
    return rows * a.channels * sizeof(float);
}

hipError_t launch_residual_grad(const ResidualArgs& a, float* ws) {
    const Shape s = grad_shape(a);
    Sum u[kSums];
    sums_of(a, u);
    Partials ps{};
    Joins js{};
    bool any = false;
    for (int k = 0; k < kSums; ++k) {
        if (!u[k].to) continue;
        ps.p[k] = Partial{ws, u[k].sb != 0};
        js.j[k] = SumJoin{ws, u[k].to, u[k].sb != 0};
        ws += partial_rows(a, s, u[k]) * a.channels;
        ps.any_item = ps.any_item || u[k].sb != 0;
        any = true;
    }
    int tk = timing_begin("residual_norm_grad", a.stream);
    hipError_t e = dispatch(a, s.nv, [&](auto t, auto n, auto w) {
        if constexpr (decltype(n)::value == kGradChunks) {
            auto go = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3(s.groups), dim3((unsigned)s.threads), 0, a.stream, a, s, ps);
            };
            if (s.threads <= 512) go(k_residual_grad<decltype(t), decltype(w)::value, 512>);
            else go(k_residual_grad<decltype(t), decltype(w)::value, 1024>);
        }
        return hipGetLastError();
    });
    timing_end(tk, a.stream);
    if (e != hipSuccess || !any) return e;
    tk = timing_begin("residual_norm_join", a.stream);
    const unsigned items = ps.any_item ? (unsigned)std::min<uint32_t>(a.batch, 65535) : 1;
    const dim3 grid((unsigned)((a.channels + kJoinColumns - 1) / kJoinColumns), items, kSums);
    if (a.bf16) hipLaunchKernelGGL(k_residual_join<__bf16>, grid, dim3(1024), 0, a.stream, js, s, a.channels);
    else hipLaunchKernelGGL(k_residual_join<float>, grid, dim3(1024), 0, a.stream, js, s, a.channels);
    timing_end(tk, a.stream);
    return hipGetLastError();
}

}  // namespace disco
