// disco_rotate.hip -- the norm of every head with the rotation to its token's
// position in the same pass, and its gradients.
//
// A row is one head of one token, D <= 128 entries.  With r = (mean x^2 +
// eps)^-1/2 and n = r x:
//   y = T (w n),  T the rotation of R / 2 pairs by the angles of the token;
//   g = T^-1 dy,  dw = sum of g n over the rows that share w,
//   dx = r (t - n mean(t n)) with t = w g.
// All of it is a few operations an entry: the bound is the memory's rate, so x
// (and dy) are read once and y (dx) written once, and r is recomputed in the
// gradient instead of stored.  A lane holds V pairs of one row (two loads of V
// entries, V the widest that sizes, strides and addresses allow), so that
// rotation stays within the lane in both layouts, and entries beyond R come in
// the same 2 V to a lane; the lanes of a row, a power of two of them, share the
// sums of squares by shuffles.  Rows of all heads of all tokens follow each
// other over the lanes; angles and weight come from the caches (together 14 of
// 58 us).  Statistics and sums are fp32, of rows brought into its range where their
// squares leave it; y, dx and dw are rounded once.
// Measured, 4 x 32768 tokens, 8 heads of 64, bf16: forward 62 us (268 MB, 4.3
// TB/s; two heads a thread took 3 % off, four 5 % on), gradients 93 us (403 MB, 4.3 TB/s) and 7 us
// for the weight's.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "disco_heads.h"
#include "disco_internal.h"

namespace disco {

namespace {

constexpr int kThreads = 256;

template <typename T, int V>
using Vec = T __attribute__((ext_vector_type(V)));

template <typename T, int V>
__device__ __forceinline__ void load(const T* p, float* f) {
    const Vec<T, V> v = *(const Vec<T, V>*)p;
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = (float)v[i];
}
template <typename T, int V>
__device__ __forceinline__ void store(T* p, const float* f) {
    Vec<float, V> v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = f[i];
    *(Vec<T, V>*)p = __builtin_convertvector(v, Vec<T, V>);
}

// lanes: of a row; slots: rows of a workgroup's pass; rows: of one grid column
// (all heads of all tokens, or the tokens of head blockIdx.y with per_head).
struct Shape {
    int items, rot_items, lanes, slots, gx, gy;
    uint32_t rows;
    bool per_head;
    Divisor heads, tokens;
};

// The part of a row that a lane holds: entries [a, a + V) and [b, b + V).
struct Item {
    int a, b;
    bool rot, has_a, has_b;
};
template <int V, bool INTER>
__device__ __forceinline__ Item item_of(int item, const Shape& s, int R, int D) {
    Item it;
    it.rot = item < s.rot_items;
    if (it.rot) {
        it.a = INTER ? 2 * V * item : V * item;
        it.b = INTER ? it.a + V : it.a + R / 2;
        it.has_a = it.has_b = true;
    } else {
        it.a = R + (item - s.rot_items) * 2 * V;
        it.b = it.a + V;
        it.has_a = it.a < D;
        it.has_b = it.b < D;
    }
    return it;
}

// Turns the V pairs e of a lane by (c, s); `back` turns the other way.
template <int V, bool INTER>
__device__ __forceinline__ void turn(float* e, const float* c, const float* s, float sign) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int ia = INTER ? 2 * j : j, ib = INTER ? 2 * j + 1 : V + j;
        const float a = e[ia], b = e[ib], sn = sign * s[j];
        e[ia] = a * c[j] - b * sn;
        e[ib] = a * sn + b * c[j];
    }
}

__device__ __forceinline__ float lane_sum(float v, int lanes) {
    for (int m = 1; m < lanes; m <<= 1) v += __shfl_xor(v, m);
    return v;
}

// Cosines and sines of the token's pairs; false where its position is no row
// of the tables.
template <int V>
__device__ __forceinline__ bool load_angles(const RotateArgs& a, int64_t b, int64_t tok, int item, bool rot, float* c,
                                            float* s) {
#pragma unroll
    for (int j = 0; j < V; ++j) c[j] = 1.0f, s[j] = 0.0f;
    if (a.rotary == 0) return true;
    const int64_t pos = a.positions ? (int64_t)a.positions[b * a.pos_sb + tok] : a.pos0 + tok;
    if (pos < 0 || pos >= a.rows) return false;
    if (rot) {
        const int64_t o = pos * (a.rotary / 2) + V * item;
        load<float, V>(a.cosines + o, c);
        load<float, V>(a.sines + o, s);
    }
    return true;
}

// eps beside the squares of a row that was multiplied by f.
__device__ __forceinline__ float scaled_eps(const RotateArgs& a, float f) { return f > 1.0f ? a.eps_up : a.eps * f * f; }

// Token and head of a row.
struct Place {
    int64_t b, tok;
    int h;
};
__device__ __forceinline__ Place place_of(const RotateArgs& a, const Shape& s, uint32_t row) {
    Place p;
    uint32_t t = row;
    if (s.per_head) {
        p.h = blockIdx.y;
    } else {
        t = s.heads.quotient(row);
        p.h = (int)(row - t * s.heads.d);
    }
    const uint32_t b = s.tokens.quotient(t);
    p.b = b;
    p.tok = t - b * s.tokens.d;
    return p;
}
template <typename T>
__device__ __forceinline__ T* row_at(const Heads& t, const Place& p) {
    return (T*)t.p + p.b * t.sb + p.tok * t.st + p.h * t.sh;
}

// A row's part for each thread: one load or two, and as many stores.
template <typename T, int V, bool INTER>
__global__ __launch_bounds__(kThreads) void k_rotate(RotateArgs a, Shape sh) {
    const int item = threadIdx.x % sh.lanes, slot = threadIdx.x / sh.lanes;
    const uint32_t row = group_index() * (uint32_t)sh.slots + slot;
    if (row >= sh.rows) return;  // whole rows: the sums below stay within one
    const Item it = item_of<V, INTER>(item, sh, a.rotary, a.dim);
    const Place p = place_of(a, sh, row);
    float e[2 * V], w[2 * V], c[V], s[V];
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) e[i] = 0.0f, w[i] = 1.0f;
    const T* x = row_at<const T>(a.x, p);
    if (it.has_a) load<T, V>(x + it.a, e);
    if (it.has_b) load<T, V>(x + it.b, e + V);
    float r = load_angles<V>(a, p.b, p.tok, item, it.rot, c, s) ? 1.0f : __builtin_nanf("");
    if (a.weight) {
        const T* wp = (const T*)a.weight + p.h * a.weight_sh;
        if (it.has_a) load<T, V>(wp + it.a, w);
        if (it.has_b) load<T, V>(wp + it.b, w + V);
    }
    if (a.norm) {
        const float inv_d = 1.0f / (float)a.dim;
        auto squares = [&] {
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) ss = fmaf(e[i], e[i], ss);
            return lane_sum(ss, sh.lanes);
        };
        float ss = squares(), eps = a.eps;
        const float f = row_scale(ss, inv_d, eps);
        if (__any(f != 1.0f)) {
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) e[i] *= f;
            ss = squares();
            eps = scaled_eps(a, f);
        }
        r *= rsqrtf(fmaf(ss, inv_d, eps));
    }
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) e[i] = e[i] * r * w[i];
    if (it.rot) turn<V, INTER>(e, c, s, 1.0f);
    T* y = row_at<T>(a.y, p);
    if (it.has_a) store<T, V>(y + it.a, e);
    if (it.has_b) store<T, V>(y + it.b, e + V);
}

// Gradients.  Each workgroup walks the runs of rows with the grid's stride and
// leaves its sum of g n in partial[(blockIdx.y, blockIdx.x)][D].
template <typename T, int V, bool INTER>
__global__ __launch_bounds__(kThreads) void k_rotate_grad(RotateArgs a, Shape sh, float* __restrict__ partial) {
    __shared__ float red[kThreads * 2 * V];
    const int item = threadIdx.x % sh.lanes, slot = threadIdx.x / sh.lanes;
    const Item it = item_of<V, INTER>(item, sh, a.rotary, a.dim);
    const float inv_d = 1.0f / (float)a.dim;
    float w[2 * V], dw[2 * V];
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) w[i] = 1.0f, dw[i] = 0.0f;
    auto load_weight = [&](int h) {
        const T* wp = (const T*)a.weight + h * a.weight_sh;
        if (it.has_a) load<T, V>(wp + it.a, w);
        if (it.has_b) load<T, V>(wp + it.b, w + V);
    };
    if (a.weight && (a.weight_sh == 0 || sh.per_head)) load_weight(sh.per_head ? blockIdx.y : 0);
    for (uint64_t row = (uint64_t)blockIdx.x * sh.slots + slot; row < sh.rows; row += (uint64_t)sh.gx * sh.slots) {
        const Place p = place_of(a, sh, (uint32_t)row);
        float e[2 * V], g[2 * V], c[V], s[V];
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) e[i] = g[i] = 0.0f;
        const T* dy = row_at<const T>(a.dy, p);
        if (it.has_a) load<T, V>(dy + it.a, g);
        if (it.has_b) load<T, V>(dy + it.b, g + V);
        if (a.norm) {
            const T* x = row_at<const T>(a.x, p);
            if (it.has_a) load<T, V>(x + it.a, e);
            if (it.has_b) load<T, V>(x + it.b, e + V);
        }
        const float poison = load_angles<V>(a, p.b, p.tok, item, it.rot, c, s) ? 1.0f : __builtin_nanf("");
        if (a.weight && a.weight_sh && !sh.per_head) load_weight(p.h);
        if (it.rot) turn<V, INTER>(g, c, s, -1.0f);
        if (a.norm) {
            float ss, tx, eps = a.eps;
            auto sums = [&] {
                ss = tx = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) {
                    ss = fmaf(e[i], e[i], ss);
                    tx = fmaf(w[i] * g[i], e[i], tx);
                }
                ss = lane_sum(ss, sh.lanes);
                tx = lane_sum(tx, sh.lanes);
            };
            sums();
            const float f = row_scale(ss, inv_d, eps);
            const bool any = __any(f != 1.0f);
            if (any) {
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) e[i] *= f;
                sums();
                eps = scaled_eps(a, f);
            }
            const float r = poison * rsqrtf(fmaf(ss, inv_d, eps));
            const float m = r * r * tx * inv_d;  // mean(t n) r
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) {
                dw[i] = fmaf(g[i] * r, e[i], dw[i]);
                g[i] = r * fmaf(-m, e[i], w[i] * g[i]);
            }
            if (any) {
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) g[i] *= f;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) g[i] *= poison;
        }
        if (a.dx.p) {
            T* dx = row_at<T>(a.dx, p);
            if (it.has_a) store<T, V>(dx + it.a, g);
            if (it.has_b) store<T, V>(dx + it.b, g + V);
        }
    }
    if (!partial) return;
    // The slots' sums in slot order.
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) red[(slot * sh.lanes + item) * 2 * V + i] = dw[i];
    __syncthreads();
    const int per = sh.lanes * 2 * V;
    float* out = partial + ((int64_t)blockIdx.y * sh.gx + blockIdx.x) * a.dim;
    for (int i = threadIdx.x; i < per; i += kThreads) {
        const Item li = item_of<V, INTER>(i / (2 * V), sh, a.rotary, a.dim);
        const int j = i % (2 * V), d = j < V ? li.a + j : li.b + j - V;
        if (i / (2 * V) >= sh.items || !(j < V ? li.has_a : li.has_b)) continue;
        float v = 0.0f;
        for (int sl = 0; sl < sh.slots; ++sl) v += red[sl * per + i];
        out[d] = v;
    }
}

// dw[group][D] = sum of the group's `rows` partial rows, in a fixed order.
// grid: (ceil(D / 16), groups); block: 16 entries x 64 slices of the rows.
template <typename T>
__global__ __launch_bounds__(1024) void k_rotate_dw(const float* __restrict__ partial, int rows, int D,
                                                    T* __restrict__ dw) {
    __shared__ float red[64][17];
    const int col = threadIdx.x % 16, slice = threadIdx.x / 16, d = blockIdx.x * 16 + col;
    float v = 0.0f;
    if (d < D)
        for (int r = slice; r < rows; r += 64) v += partial[((int64_t)blockIdx.y * rows + r) * D + d];
    red[slice][col] = v;
    for (int m = 32; m > 0; m >>= 1) {
        __syncthreads();
        if (slice < m) red[slice][col] += red[slice + m][col];
    }
    if (slice == 0 && d < D) dw[(int64_t)blockIdx.y * D + d] = (T)red[0][col];
}

bool fits(const Heads& t, int v, size_t elem) {
    return !t.p || ((uintptr_t)t.p % (v * elem) == 0 && t.sb % v == 0 && t.st % v == 0 && t.sh % v == 0);
}

// The widest load: it divides the pairs, the entries beyond them, every stride
// and address.
int width(const RotateArgs& a) {
    const size_t e = a.bf16 ? 2 : 4;
    for (int v = a.bf16 ? 8 : 4; v > 1; v /= 2) {
        if ((a.rotary / 2) % v || (a.dim - a.rotary) % v) continue;
        if (a.weight && (uintptr_t)a.weight % (v * e)) continue;
        if (!fits(a.x, v, e) || !fits(a.y, v, e) || !fits(a.dy, v, e) || !fits(a.dx, v, e)) continue;
        // cosines and sines come in fp32: at most 16 bytes a load
        const uintptr_t al = 4 * (uintptr_t)std::min(v, 4);
        if (a.rotary && ((uintptr_t)a.cosines % al || (uintptr_t)a.sines % al)) continue;
        return v;
    }
    return 1;
}

// per_head: a grid column for each head; blocks: the most workgroups (0: a
// thread for every part of a row).
Shape shape_of(const RotateArgs& a, int v, bool per_head, int blocks) {
    Shape s;
    s.rot_items = a.rotary / 2 / v;
    s.items = s.rot_items + (a.dim - a.rotary + 2 * v - 1) / (2 * v);
    s.lanes = 1;
    while (s.lanes < s.items) s.lanes *= 2;
    s.slots = kThreads / s.lanes;
    s.per_head = per_head;
    s.heads = divisor((uint32_t)std::max(a.heads, 1));
    s.tokens = divisor((uint32_t)std::max<int64_t>(a.tokens, 1));
    s.gy = per_head ? std::max(a.heads, 1) : 1;
    s.rows = (uint32_t)((int64_t)a.batch * a.tokens * (per_head ? 1 : a.heads));
    const int64_t gx = std::max<int64_t>(1, ((int64_t)s.rows + s.slots - 1) / s.slots);
    s.gx = (int)std::min<int64_t>(gx, blocks > 0 ? std::max(1, blocks / s.gy) : gx);
    return s;
}

// Workgroups of the gradient when it sums dw, each of which leaves one partial
// row, and otherwise (as many as one axis of a grid takes).
constexpr int kGradBlocks = 1024, kGradRowBlocks = kGridRow;

// Calls f with the kernels' types for the storage type, width and layout.
template <typename F>
hipError_t dispatch(const RotateArgs& a, int v, F&& f) {
    auto layout = [&](auto t, auto vv) {
        return a.interleaved ? f(t, vv, std::true_type{}) : f(t, vv, std::false_type{});
    };
    auto type = [&](auto vv) {
        if (a.bf16) return layout(__bf16{}, vv);
        return layout(float{}, std::integral_constant<int, (decltype(vv)::value > 4 ? 4 : decltype(vv)::value)>{});
    };
    switch (v) {
        case 8: return type(std::integral_constant<int, 8>{});
        case 4: return type(std::integral_constant<int, 4>{});
        case 2: return type(std::integral_constant<int, 2>{});
        default: return type(std::integral_constant<int, 1>{});
    }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a) {
    const int v = width(a);
    const Shape s = shape_of(a, v, false, 0);
    const int tk = timing_begin("norm_rotate", a.stream);
    const hipError_t e = dispatch(a, v, [&](auto t, auto vv, auto inter) {
        hipLaunchKernelGGL((k_rotate<decltype(t), decltype(vv)::value, decltype(inter)::value>), grid_dim(s.gx),
                           dim3(kThreads), 0, a.stream, a, s);
        return hipGetLastError();
    });
    timing_end(tk, a.stream);
    return e;
}

size_t rotate_grad_ws_bytes(const RotateArgs& a) { return (size_t)(kGradBlocks + 4096) * a.dim * sizeof(float); }

hipError_t launch_rotate_grad(const RotateArgs& a, float* ws) {
    const int v = width(a);
    const Shape s = shape_of(a, v, a.weight && a.weight_sh != 0 && a.dweight, a.dweight ? kGradBlocks : kGradRowBlocks);
    int tk = timing_begin("norm_rotate_grad", a.stream);
    hipError_t e = dispatch(a, v, [&](auto t, auto vv, auto inter) {
        hipLaunchKernelGGL((k_rotate_grad<decltype(t), decltype(vv)::value, decltype(inter)::value>),
                           dim3((unsigned)s.gx, (unsigned)s.gy), dim3(kThreads), 0, a.stream, a, s,
                           a.dweight ? ws : nullptr);
        return hipGetLastError();
    });
    timing_end(tk, a.stream);
    if (e != hipSuccess || !a.dweight) return e;
    const int groups = a.weight_sh ? a.heads : 1, rows = s.gx * s.gy / groups;
    tk = timing_begin("norm_rotate_dw", a.stream);
    const dim3 grid((unsigned)((a.dim + 15) / 16), (unsigned)groups);
    if (a.bf16)
        hipLaunchKernelGGL(k_rotate_dw<__bf16>, grid, dim3(1024), 0, a.stream, ws, rows, a.dim, (__bf16*)a.dweight);
    else
        hipLaunchKernelGGL(k_rotate_dw<float>, grid, dim3(1024), 0, a.stream, ws, rows, a.dim, (float*)a.dweight);
    timing_end(tk, a.stream);
    return hipGetLastError();
}

}  // namespace disco
