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
// y is taken from h before its rounding to bf16.  Rows of up to 1024 entries (512 in the
// gradients of fp32) lie in one wave, whose lanes share the sums by shuffles and without a
// barrier; longer ones in a workgroup, with one barrier a sum.  A thread holds chunks of eight
// entries, the share of one block of the dropout's generator.  All sums are fp32.
//
// The gradients of the weights are summed in a fixed order: each workgroup walks
// a run of rows and leaves one partial row a sum (one an item for weights of
// [batch, channels]), which k_residual_join adds.
//
// Measured (kernel traces), bf16: 32768 rows of 1024, dropped, both norms and a gate 45.5 us forward (268 MB, 5.9 TB/s)
// and 95 us gradients (403 MB, 4.2 TB/s); 4050 rows of 8192 42 and 93 us; 32768 rows of 512
// forward 23 us (134 MB, in part from the caches).  Rows of weights by item go item by item: of few tokens an item most
// of a workgroup's slots are idle (bf16 kernels by events, one token each of 8192 items of 64 channels 42 us forward, 137 + 80
// gradients and join, with shared weights 7, 11 + 6; of 256 items of 1024 11, 29 + 42 and 6, 15 + 6).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "disco_internal.h"
#include "disco_residual.h"

namespace disco {

namespace {

template <typename T, int NV, bool EIGHTS, bool DROP>
__global__ __launch_bounds__(512) void k_residual(ResidualArgs a, NormShape s) {
    __shared__ float red[2][1024 / kNormWave][2];
    const int lane = threadIdx.x & (s.lanes - 1), c = lane * kChunk, C = a.channels;
    const uint32_t slot = threadIdx.x / s.lanes;
    RowSums rs{s.lanes, red};
    bool again;
    const uint64_t offset = DROP ? drop_offset(a.drop) : 0;
    const int step = s.lanes * kChunk;  // entries between a thread's chunks
    struct Row {
        Raw<T> x[NV], f[NV];
    };
    const uint64_t begin = (uint64_t)blockIdx.x * s.per_group, end = min(begin + s.per_group, (uint64_t)s.rows);
    for (uint64_t seg = begin; seg < end;) {
        // the run's rows of one item: positions at .. stop - 1
        const uint32_t item = s.by_length.quotient((uint32_t)seg), first = (uint32_t)(seg - (uint64_t)item * s.length);
        const uint32_t stop = (uint32_t)min((uint64_t)s.length, first + (end - seg));
        Cursor<const T> to_x(a.x, s, item, first + slot, c), to_f(a.f, s, item, first + slot, c);
        Cursor<T> to_h(a.h, s, item, first + slot, c), to_y(a.y, s, item, first + slot, c);
        auto load = [&](uint32_t at) {
            Row r;
            const int n = at < stop ? C - c : 0;
            const T *f = to_f.next(), *x = to_x.next();
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                r.f[j] = load_raw<T, EIGHTS>(f + j * step, n - j * step);
                if (has(s, kHasX)) r.x[j] = load_raw<T, EIGHTS>(x + j * step, n - j * step);
                else r.x[j].fill(0.0f);
            }
            return r;
        };
        Raw<T> w[NV], g[NV], w2[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            w[j] = load_weight<T, EIGHTS>(a.post_w, a.post_sb, item, c + j * step, C - c - j * step);
            g[j] = load_weight<T, EIGHTS>(a.gate, a.gate_sb, item, c + j * step, C - c - j * step);
            w2[j] = load_weight<T, EIGHTS>(a.next_w, a.next_sb, item, c + j * step, C - c - j * step);
        }
        Row next = load(first + slot);
        for (uint32_t base = first; base < stop; base += s.slots) {
            const uint32_t at = base + slot;
            const int n = at < stop ? C - c : 0;
            const Row now = next;
#pragma unroll
            for (int j = 0; j < NV; ++j) w[j].anew(), g[j].anew(), w2[j].anew();
            if (base + s.slots < stop) next = load(at + s.slots);
            float e[NV * kChunk];
#pragma unroll
            for (int i = 0; i < NV * kChunk; ++i) e[i] = now.f[i / kChunk].at(i % kChunk);
            float r = 1.0f, up;
            if (has(s, kHasPost)) r = norm_factor(e, a, rs.one(squares(e)), rs, &up, &again);
            r *= a.drop.factor;  // (1 where nothing is dropped)
            T *h = to_h.next(), *y = to_y.next();
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float* u = e + j * kChunk;
                float v[kChunk];
                Words bits;
                if constexpr (DROP) bits = drop_words(a.drop, offset, item * s.row_item + at * s.row_at, lane + s.lanes * j);
#pragma unroll
                for (int i = 0; i < kChunk; ++i) {
                    float d = u[i] * r * w[j].at(i);
                    if constexpr (DROP) d = stays(bits, i, a.drop.out) ? d : 0.0f;
                    v[i] = u[i] = fmaf(a.scale, now.x[j].at(i), d * g[j].at(i));
                }
                if (has(s, kHasH)) store_raw<T, EIGHTS>(h + j * step, n - j * step, v);
            }
            if (!has(s, kHasY)) continue;
            r = norm_factor(e, a, rs.one(squares(e)), rs, &up, &again);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float v[kChunk];
#pragma unroll
                for (int i = 0; i < kChunk; ++i) v[i] = e[j * kChunk + i] * r * w2[j].at(i);
                store_raw<T, EIGHTS>(y + j * step, n - j * step, v);
            }
        }
        seg += stop - first;
    }
}

constexpr int kForwardChunks = 2;
// Workgroups of a launch: as many as the CUs hold at a time by bf16's registers (of one chunk a thread they would hold
// one to three waves a SIMD more).  fp32 of two chunks holds three waves a SIMD, 768 workgroups of these 1024, and the rest go in a
// second round: 32768 rows of 1024 106 us by events (537 MB, 5.1 TB/s).
uint32_t forward_groups(const NormShape& s) {
    return 256 * (uint32_t)std::max(1, 4 * (s.nv == 1 ? 5 : 4) / (s.threads / kNormWave));
}

}  // namespace

hipError_t launch_residual(const ResidualArgs& args) {
    ResidualArgs a = args;
    NormShape s = norm_shape(&a, kForwardChunks);
    norm_runs(&s, forward_groups(s));
    const int tk = timing_begin("residual_norm", a.stream);
    const hipError_t e = norm_dispatch(a, [&](auto t, auto w, auto drop) {
        auto go = [&](auto n) {
            hipLaunchKernelGGL((k_residual<decltype(t), decltype(n)::value, decltype(w)::value, decltype(drop)::value>),
                               dim3(s.groups), dim3((unsigned)s.threads), 0, a.stream, a, s);
            return hipGetLastError();
        };
        return s.nv == 1 ? go(std::integral_constant<int, 1>{}) : go(std::integral_constant<int, 2>{});
    });
    timing_end(tk, a.stream);
    return e;
}

}  // namespace disco
