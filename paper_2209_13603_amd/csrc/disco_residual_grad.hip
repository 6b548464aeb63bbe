// disco_residual_grad.hip -- gradients of the residual sum with its norms, gate and
// dropout (the formulas stand in disco_residual.hip).
//
// One pass over x, f, dh and dy: h and both norms are recomputed, three sums a row
// (of f^2; of h^2 with t n2; of t n1) are taken within a wave or a workgroup, and
// the products that make the weights' gradients add up in LDS over a
// workgroup's run of rows.  With dropout and all three sums it reaches 4.2 TB/s (32768 x 1024
// bf16, 95 us): with two chunks a thread eight waves a CU are all that a row and the next one's loads leave
// room for.  One chunk a thread (up to 512 channels) holds sixteen; such rows over 128 lanes, with barriers for their
// sums, were not measured.  fp32 rows of more than 4096 channels, a workgroup of 1024 threads with 128 registers each, spill 16 to
// 97 of them (2000 x 8192 113 us by events, 3.5 TB/s).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "disco_internal.h"
#include "disco_residual.h"

namespace disco {

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));

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
};

// The next row's loads go out before this one's arithmetic, a run's weights stay in
// registers.
template <typename T, int NV, bool EIGHTS, bool DROP, int THREADS>
__global__ __launch_bounds__(THREADS) void k_residual_grad(ResidualArgs a, NormShape s, Partials ps) {
    constexpr int N = NV * kChunk;
    __shared__ float red[2][1024 / kNormWave][2];
    // The sums of the run's rows, a thread's own: in registers they would leave no room
    // for the next row.
    __shared__ f4 acc[kSums][N / 4][THREADS];
    const int lane = threadIdx.x & (s.lanes - 1), C = a.channels, c = lane * kChunk;
    const uint32_t slot = threadIdx.x / s.lanes;
    const int step = s.lanes * kChunk;  // entries between a thread's chunks
    const float inv = 1.0f / (float)C;
    RowSums rs{s.lanes, red};
    bool again;
    const uint64_t offset = DROP ? drop_offset(a.drop) : 0;
    auto clear = [&](int k) {
#pragma unroll
        for (int q = 0; q < N / 4; ++q) acc[k][q][threadIdx.x] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    };
#pragma unroll
    for (int k = 0; k < kSums; ++k) clear(k);
    // acc[k] += u v
    auto add = [&](int k, const float(&u)[N], auto&& v) {
        if (!ps.p[k].at) return;
#pragma unroll
        for (int q = 0; q < N / 4; ++q) {
            f4 e = acc[k][q][threadIdx.x];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = fmaf(u[4 * q + i], v(4 * q + i), e[i]);
            acc[k][q][threadIdx.x] = e;
        }
    };
    // Leaves the workgroup's sum k in a partial row, the slots' in slot order.
    auto flush = [&](int k, uint32_t at) {
        float* out = ps.p[k].at + (int64_t)at * C;
        __syncthreads();
        for (int d = threadIdx.x; d < C; d += s.threads) {
            const int chunk = d / kChunk, e = chunk / s.lanes * kChunk + d % kChunk;
            float v = 0.0f;
            for (int sl = 0; sl < s.slots; ++sl) v += acc[k][e / 4][sl * s.lanes + chunk % s.lanes][e % 4];
            out[d] = v;
        }
        __syncthreads();
        clear(k);
    };
    struct Row {
        Raw<T> x[NV], f[NV], dh[NV], dy[NV];
    };
    const uint64_t begin = (uint64_t)blockIdx.x * s.per_group, end = min(begin + s.per_group, (uint64_t)s.rows);
    for (uint64_t seg = begin; seg < end;) {
        // the run's rows of one item: positions first .. stop - 1
        const uint32_t item = s.by_length.quotient((uint32_t)seg), first = (uint32_t)(seg - (uint64_t)item * s.length);
        const uint32_t stop = (uint32_t)min((uint64_t)s.length, first + (end - seg));
        Cursor<const T> to_x(a.x, s, item, first + slot, c), to_f(a.f, s, item, first + slot, c);
        Cursor<const T> to_dh(a.dh, s, item, first + slot, c), to_dy(a.dy, s, item, first + slot, c);
        Cursor<T> to_dx(a.dx, s, item, first + slot, c), to_df(a.df, s, item, first + slot, c);
        auto load = [&](uint32_t at) {
            const int n = at < stop ? C - c : 0;
            Row r;
            const T *x = to_x.next(), *f = to_f.next(), *dh = to_dh.next(), *dy = to_dy.next();
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                r.f[j] = load_raw<T, EIGHTS>(f + j * step, n - j * step);
                r.x[j] = load_raw<T, EIGHTS>(x + j * step, has(s, kHasX) ? n - j * step : 0);
                r.dh[j] = load_raw<T, EIGHTS>(dh + j * step, has(s, kHasDh) ? n - j * step : 0);
                r.dy[j] = load_raw<T, EIGHTS>(dy + j * step, has(s, kHasDy) ? n - j * step : 0);
            }
            return r;
        };
        Raw<T> w[NV], g[NV], w2[NV];
        auto load_weights = [&] {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                w[j] = load_weight<T, EIGHTS>(a.post_w, a.post_sb, item, c + j * step, C - c - j * step);
                g[j] = load_weight<T, EIGHTS>(a.gate, a.gate_sb, item, c + j * step, C - c - j * step);
                w2[j] = load_weight<T, EIGHTS>(a.next_w, a.next_sb, item, c + j * step, C - c - j * step);
            }
        };
        auto raw = [&](Raw<T>(&r)[NV]) {
#pragma unroll
            for (int j = 0; j < NV; ++j) r[j].anew();
        };
        load_weights();
        Row next = load(first + slot);
        for (uint32_t base = first; base < stop; base += s.slots) {
            const uint32_t at = base + slot;
            const bool live = at < stop;
            const int n = live ? C - c : 0;
            Row now = next;
            raw(w), raw(g), raw(w2);
            if (base + s.slots < stop) next = load(at + s.slots);
            auto at_entry = [](const Raw<T>(&r)[NV], int i) { return r[i / kChunk].at(i % kChunk); };
            float n1[N], d[N], h[N], D[N];
#pragma unroll
            for (int i = 0; i < N; ++i) n1[i] = at_entry(now.f, i);
            float r1 = 1.0f, up1 = 1.0f;
            if (has(s, kHasPost)) {
                r1 = norm_factor(n1, a, rs.one(squares(n1)), rs, &up1, &again);
                r1 = live ? r1 : 0.0f;  // (without an eps a row of zeros has no norm)
#pragma unroll
                for (int i = 0; i < N; ++i) n1[i] *= r1;
                r1 *= up1;
            }
            // what an entry of the block is multiplied by; 0 takes out whatever it holds
            float kept[DROP ? N : 1];
            if constexpr (DROP) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const Words bits = drop_words(a.drop, offset, item * s.row_item + at * s.row_at, lane + j * s.lanes);
#pragma unroll
                    for (int i = 0; i < kChunk; ++i)
                        kept[DROP ? j * kChunk + i : 0] = stays(bits, i, a.drop.out) ? a.drop.factor : 0.0f;
                }
            }
            auto dropped = [&](float v, int i) {
                if constexpr (!DROP) return v;
                const float k = kept[DROP ? i : 0];
                return k != 0.0f ? k * v : 0.0f;
            };
#pragma unroll
            for (int i = 0; i < N; ++i) {
                d[i] = dropped(n1[i] * at_entry(w, i), i);
                h[i] = fmaf(a.scale, at_entry(now.x, i), d[i] * at_entry(g, i));
            }
            raw(w), raw(g);
            if (has(s, kHasDy)) {
                // mean(t n2) with the sum of squares, from h before it is normed
                float up2, ss = squares(h), m = 0.0f;
                auto products = [&] {
                    m = 0.0f;
#pragma unroll
                    for (int i = 0; i < N; ++i) m = fmaf(at_entry(now.dy, i) * at_entry(w2, i), h[i], m);
                };
                products();
                rs.two(ss, m);
                float r = norm_factor(h, a, ss, rs, &up2, &again);
                r = live ? r : 0.0f;
                if (again) {
                    products();
                    m = rs.one(m);
                }
                m *= r * inv;
                const float r2 = r * up2;
                raw(now.dy), raw(w2);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    h[i] *= r;  // n2
                    D[i] = fmaf(r2, fmaf(-m, h[i], at_entry(now.dy, i) * at_entry(w2, i)), at_entry(now.dh, i));
                }
                add(kNext, h, [&](int i) { return at_entry(now.dy, i); });
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) D[i] = at_entry(now.dh, i);
            }
            add(kGate, D, [&](int i) { return d[i]; });
#pragma unroll
            for (int i = 0; i < N; ++i) {
                h[i] = a.scale * D[i];
                D[i] = dropped(D[i] * at_entry(g, i), i);  // du
            }
            T *dx = to_dx.next(), *df = to_df.next();
            auto store = [&](T* to, const float(&v)[N]) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    float e[kChunk];
#pragma unroll
                    for (int i = 0; i < kChunk; ++i) e[i] = v[j * kChunk + i];
                    store_raw<T, EIGHTS>(to + j * step, n - j * step, e);
                }
            };
            if (has(s, kHasDx)) store(dx, h);
            if (has(s, kHasPost)) {
                float m = 0.0f;
                add(kPost, D, [&](int i) { return n1[i]; });
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    D[i] *= at_entry(w, i);
                    m = fmaf(D[i], n1[i], m);
                }
                m = rs.one(m) * inv;
#pragma unroll
                for (int i = 0; i < N; ++i) D[i] = r1 * fmaf(-m, n1[i], D[i]);
            }
            if (has(s, kHasDf)) store(df, D);
        }
#pragma unroll
        for (int k = 0; k < kSums; ++k)
            if (ps.p[k].at && ps.p[k].per_item) flush(k, blockIdx.x + item);
        seg += stop - first;
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
constexpr int kJoinColumns = 32, kJoinSlices = 32;

// Adds the partial rows of a weight's gradient in a fixed order.  grid: (columns /
// 32, items, sums); 32 columns x 32 slices of the rows.
template <typename T>
__global__ __launch_bounds__(1024) void k_residual_join(Joins js, NormShape s, int C) {
    __shared__ float red[kJoinSlices][kJoinColumns + 1];
    const SumJoin j = js.j[blockIdx.z];
    if (!j.to || (blockIdx.y > 0 && !j.per_item)) return;
    const int col = threadIdx.x % kJoinColumns, slice = threadIdx.x / kJoinColumns, c = blockIdx.x * kJoinColumns + col;
    for (uint32_t item = blockIdx.y; item < (j.per_item ? s.items : 1); item += gridDim.y) {
        uint32_t lo = 0, hi = s.groups;
        if (j.per_item) {  // rows workgroup + item of the runs that reach into the item
            const uint64_t r0 = (uint64_t)item * s.length;
            lo = (uint32_t)(r0 / s.per_group) + item;
            hi = s.rows ? (uint32_t)((r0 + s.length - 1) / s.per_group) + item + 1 : lo;
        }
        float v = 0.0f;
        if (c < C) {
#pragma unroll 8
            for (uint32_t r = lo + slice; r < hi; r += kJoinSlices) v += j.from[(int64_t)r * C + c];
        }
        __syncthreads();
        red[slice][col] = v;
        for (int m = kJoinSlices / 2; m > 0; m >>= 1) {
            __syncthreads();
            if (slice < m) red[slice][col] += red[slice + m][col];
        }
        if (slice == 0 && c < C) ((T*)j.to)[(int64_t)item * C + c] = (T)red[0][col];
    }
}

// Workgroups: as many as the CUs hold at a time by their registers (a part of a
// second round leaves most CUs idle).
NormShape grad_shape(ResidualArgs* a) {
    NormShape s = norm_shape(a, a->bf16 ? 2 : 1);
    const int waves = s.threads / kNormWave, held = s.threads > 512 ? 16 : a->bf16 ? s.nv == 1 ? 16 : 8 : 12;
    norm_runs(&s, 256 * (uint32_t)std::max(1, held / waves));
    return s;
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
size_t partial_rows(const ResidualArgs& a, const NormShape& s, const Sum& u) { return (size_t)s.groups + (u.sb ? a.batch : 0); }

}  // namespace

size_t residual_grad_ws_bytes(const ResidualArgs& args) {
    ResidualArgs a = args;
    const NormShape s = grad_shape(&a);
    Sum u[kSums];
    sums_of(a, u);
    size_t rows = 0;
    for (const Sum& k : u)
        if (k.weight) rows += partial_rows(a, s, k);
    return rows * a.channels * sizeof(float);
}

hipError_t launch_residual_grad(const ResidualArgs& args, float* ws) {
    ResidualArgs a = args;
    const NormShape s = grad_shape(&a);
    Sum u[kSums];
    sums_of(a, u);
    Partials ps{};
    Joins js{};
    bool any = false, items = false;
    for (int k = 0; k < kSums; ++k) {
        if (!u[k].to) continue;
        ps.p[k] = Partial{ws, u[k].sb != 0};
        js.j[k] = SumJoin{ws, u[k].to, u[k].sb != 0};
        ws += partial_rows(a, s, u[k]) * a.channels;
        items = items || u[k].sb != 0;
        any = true;
    }
    int tk = timing_begin("residual_norm_grad", a.stream);
    const hipError_t e = norm_dispatch(a, [&](auto t, auto w, auto drop) {
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(s.groups), dim3((unsigned)s.threads), 0, a.stream, a, s, ps);
            return hipGetLastError();
        };
        constexpr bool W = decltype(w)::value;
        constexpr bool DROP = decltype(drop)::value;
        if constexpr (sizeof(t) == 2) {
            if (s.nv == 1) return go(k_residual_grad<__bf16, 1, W, DROP, 256>);
            if (s.threads <= 128) return go(k_residual_grad<__bf16, 2, W, DROP, 128>);
            return s.threads <= 256 ? go(k_residual_grad<__bf16, 2, W, DROP, 256>) : go(k_residual_grad<__bf16, 2, W, DROP, 512>);
        } else {
            if (s.threads <= 128) return go(k_residual_grad<float, 1, W, DROP, 128>);
            if (s.threads <= 256) return go(k_residual_grad<float, 1, W, DROP, 256>);
            return s.threads <= 512 ? go(k_residual_grad<float, 1, W, DROP, 512>) : go(k_residual_grad<float, 1, W, DROP, 1024>);
        }
    });
    timing_end(tk, a.stream);
    if (e != hipSuccess || !any) return e;
    tk = timing_begin("residual_norm_join", a.stream);
    const dim3 grid((unsigned)((a.channels + kJoinColumns - 1) / kJoinColumns), items ? std::max(1u, std::min(s.items, 65535u)) : 1,
                    kSums);
    if (a.bf16) hipLaunchKernelGGL(k_residual_join<__bf16>, grid, dim3(1024), 0, a.stream, js, s, a.channels);
    else hipLaunchKernelGGL(k_residual_join<float>, grid, dim3(1024), 0, a.stream, js, s, a.channels);
    timing_end(tk, a.stream);
    return hipGetLastError();
}

}  // namespace disco
