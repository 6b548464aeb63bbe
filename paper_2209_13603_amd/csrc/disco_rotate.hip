// disco_rotate.hip -- the norm of every head with the rotation to its token's
// position in the same pass, and its gradients.
//
// A row is one head of one token, D <= 128 entries.  With r = (mean x^2 +
// eps)^-1/2 and n = r x:
//   y = T (w n),  T the rotation of R / 2 pairs by the angles of the token;
//   g = T^-1 dy,  dw = sum of g n over the rows that share w,
//   dx = r (t - n mean(t n)) with t = w g.
// All of it is a few operations an entry: the bound is the memory's rate, so x
// (and dy) are read once and y (dx) written once, r is recomputed in the
// gradient instead of stored, and the tables and the weight are read once per
// token and lane for a run of heads.  A lane holds V pairs of one row (two
// loads of V entries, V the widest that sizes, strides and addresses allow), so
// that rotation stays within the lane in both layouts, and entries beyond R
// come in the same 2 V to a lane; the lanes of a row, a power of two of them,
// share the sums of squares by shuffles.  Statistics and sums are fp32; y, dx
// and dw are rounded once.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "disco_heads.h"
#include "disco_internal.h"

namespace disco {

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // heads whose loads are in flight together

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

struct Shape {
    int items, rot_items, lanes, slots, hpb, gx, gy;
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

// grid: (token blocks, groups of hpb heads).
template <typename T, int V, bool INTER>
__global__ __launch_bounds__(kThreads) void k_rotate(RotateArgs a, Shape sh) {
    const int item = threadIdx.x % sh.lanes, slot = threadIdx.x / sh.lanes;
    const int64_t t = (int64_t)blockIdx.x * sh.slots + slot, n_tok = (int64_t)a.batch * a.tokens;
    if (t >= n_tok) return;  // whole rows: the shuffles below stay within one
    const int64_t b = (uint32_t)t / (uint32_t)a.tokens, tok = t - b * a.tokens;
    const int h0 = blockIdx.y * sh.hpb, h1 = min(h0 + sh.hpb, a.heads);
    const Item it = item_of<V, INTER>(item, sh, a.rotary, a.dim);
    const T* x = (const T*)a.x.p + b * a.x.sb + tok * a.x.st;
    T* y = (T*)a.y.p + b * a.y.sb + tok * a.y.st;
    float c[V], s[V], w[2 * V];
    const float poison = load_angles<V>(a, b, tok, item, it.rot, c, s) ? 1.0f : __builtin_nanf("");
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) w[i] = 1.0f;
    auto load_weight = [&](int h) {
        const T* wp = (const T*)a.weight + (int64_t)h * a.weight_sh;
        if (it.has_a) load<T, V>(wp + it.a, w);
        if (it.has_b) load<T, V>(wp + it.b, w + V);
    };
    if (a.weight && a.weight_sh == 0) load_weight(0);
    const float inv_d = 1.0f / (float)a.dim;
    for (int h = h0; h < h1; h += kUnroll) {
        float e[kUnroll][2 * V];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) e[u][i] = 0.0f;
            const T* xp = x + (int64_t)min(h + u, h1 - 1) * a.x.sh;
            if (it.has_a) load<T, V>(xp + it.a, e[u]);
            if (it.has_b) load<T, V>(xp + it.b, e[u] + V);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (h + u >= h1) break;
            if (a.weight && a.weight_sh != 0) load_weight(h + u);
            float r = poison;
            if (a.norm) {
                float ss = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) ss = fmaf(e[u][i], e[u][i], ss);
                r *= rsqrtf(fmaf(lane_sum(ss, sh.lanes), inv_d, a.eps));
            }
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) e[u][i] = e[u][i] * r * w[i];
            if (it.rot) turn<V, INTER>(e[u], c, s, 1.0f);
            T* yp = y + (int64_t)(h + u) * a.y.sh;
            if (it.has_a) store<T, V>(yp + it.a, e[u]);
            if (it.has_b) store<T, V>(yp + it.b, e[u] + V);
        }
    }
}

// Gradients.  Each workgroup walks the token blocks with the grid's stride and
// leaves its sum of g n in partial[(blockIdx.y, blockIdx.x)][D].
template <typename T, int V, bool INTER>
__global__ __launch_bounds__(kThreads) void k_rotate_grad(RotateArgs a, Shape sh, float* __restrict__ partial) {
    __shared__ float red[kThreads * 2 * V];
    const int item = threadIdx.x % sh.lanes, slot = threadIdx.x / sh.lanes;
    const int64_t n_tok = (int64_t)a.batch * a.tokens;
    const int h0 = blockIdx.y * sh.hpb, h1 = min(h0 + sh.hpb, a.heads);
    const Item it = item_of<V, INTER>(item, sh, a.rotary, a.dim);
    const float inv_d = 1.0f / (float)a.dim;
    float w[2 * V], dw[2 * V];
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) w[i] = 1.0f, dw[i] = 0.0f;
    auto load_weight = [&](int h) {
        const T* wp = (const T*)a.weight + (int64_t)h * a.weight_sh;
        if (it.has_a) load<T, V>(wp + it.a, w);
        if (it.has_b) load<T, V>(wp + it.b, w + V);
    };
    if (a.weight && a.weight_sh == 0) load_weight(0);
    for (int64_t t = (int64_t)blockIdx.x * sh.slots + slot; t < n_tok; t += (int64_t)sh.gx * sh.slots) {
        const int64_t b = (uint32_t)t / (uint32_t)a.tokens, tok = t - b * a.tokens;
        const T* x = a.norm ? (const T*)a.x.p + b * a.x.sb + tok * a.x.st : nullptr;
        const T* dy = (const T*)a.dy.p + b * a.dy.sb + tok * a.dy.st;
        T* dx = a.dx.p ? (T*)a.dx.p + b * a.dx.sb + tok * a.dx.st : nullptr;
        float c[V], s[V];
        const float poison = load_angles<V>(a, b, tok, item, it.rot, c, s) ? 1.0f : __builtin_nanf("");
        constexpr int kU = kUnroll / 2;
        for (int h = h0; h < h1; h += kU) {
            float e[kU][2 * V], g[kU][2 * V];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
#pragma unroll
                for (int i = 0; i < 2 * V; ++i) e[u][i] = g[u][i] = 0.0f;
                const int hu = min(h + u, h1 - 1);
                const T* gp = dy + (int64_t)hu * a.dy.sh;
                if (it.has_a) load<T, V>(gp + it.a, g[u]);
                if (it.has_b) load<T, V>(gp + it.b, g[u] + V);
                if (a.norm) {
                    const T* xp = x + (int64_t)hu * a.x.sh;
                    if (it.has_a) load<T, V>(xp + it.a, e[u]);
                    if (it.has_b) load<T, V>(xp + it.b, e[u] + V);
                }
            }
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                if (h + u >= h1) break;
                if (a.weight && a.weight_sh != 0) load_weight(h + u);
                if (it.rot) turn<V, INTER>(g[u], c, s, -1.0f);
                if (a.norm) {
                    float ss = 0.0f, tx = 0.0f;
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) {
                        ss = fmaf(e[u][i], e[u][i], ss);
                        tx = fmaf(w[i] * g[u][i], e[u][i], tx);
                    }
                    const float r = poison * rsqrtf(fmaf(lane_sum(ss, sh.lanes), inv_d, a.eps));
                    const float m = r * r * lane_sum(tx, sh.lanes) * inv_d;  // mean(t n) r
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) {
                        dw[i] = fmaf(g[u][i] * r, e[u][i], dw[i]);
                        g[u][i] = r * fmaf(-m, e[u][i], w[i] * g[u][i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 2 * V; ++i) g[u][i] *= poison;
                }
                if (dx) {
                    T* dp = dx + (int64_t)(h + u) * a.dx.sh;
                    if (it.has_a) store<T, V>(dp + it.a, g[u]);
                    if (it.has_b) store<T, V>(dp + it.b, g[u] + V);
                }
            }
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

Shape shape_of(const RotateArgs& a, int v, bool per_head, int max_blocks) {
    Shape s;
    s.rot_items = a.rotary / 2 / v;
    s.items = s.rot_items + (a.dim - a.rotary + 2 * v - 1) / (2 * v);
    s.lanes = 1;
    while (s.lanes < s.items) s.lanes *= 2;
    s.slots = kThreads / s.lanes;
    const int64_t tokens = (int64_t)a.batch * a.tokens, gx = std::max<int64_t>(1, (tokens + s.slots - 1) / s.slots);
    // All heads of a token by one lane where that leaves the chip full (the
    // tables and weight are then read once a token), fewer below.
    s.hpb = per_head ? 1 : std::max(a.heads, 1);
    while (s.hpb > 1 && gx * ((a.heads + s.hpb - 1) / s.hpb) < 1024) s.hpb = (s.hpb + 1) / 2;
    s.gy = std::max(1, (a.heads + s.hpb - 1) / s.hpb);
    s.gx = (int)std::min<int64_t>(gx, max_blocks > 0 ? std::max(1, max_blocks / s.gy) : gx);
    return s;
}

// Workgroups of the gradient when it sums dw: each leaves one partial row.
constexpr int kGradBlocks = 2048;

Shape grad_shape(const RotateArgs& a, int v) {
    return shape_of(a, v, a.weight && a.weight_sh != 0 && a.dweight, a.dweight ? kGradBlocks : 0);
}

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
        hipLaunchKernelGGL((k_rotate<decltype(t), decltype(vv)::value, decltype(inter)::value>),
                           dim3((unsigned)s.gx, (unsigned)s.gy), dim3(kThreads), 0, a.stream, a, s);
        return hipGetLastError();
    });
    timing_end(tk, a.stream);
    return e;
}

size_t rotate_grad_ws_bytes(const RotateArgs& a) { return (size_t)(kGradBlocks + 4096) * a.dim * sizeof(float); }

hipError_t launch_rotate_grad(const RotateArgs& a, float* ws) {
    const int v = width(a);
    const Shape s = grad_shape(a, v);
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
