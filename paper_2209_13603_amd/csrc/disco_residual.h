// disco_residual.h -- parts shared by the residual sum with its norms and its gradients.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>
#include <utility>

#include "disco_blocks.h"

namespace disco {

constexpr int kNormThreads = 256;
constexpr int kNormWave = 64;

// How a call is cut.  lanes: threads of a row (a power of two; beyond a wave the
// whole workgroup); nv: chunks of a thread; slots: rows of a workgroup at a time.
// Rows go by item and position, as the tensors' strides have them: batch items and
// tokens, or tokens and batch items where series are short, or all rows as one
// item's.  Each workgroup takes a run of per_group of them.
struct NormShape {
    int lanes, nv, threads, slots;
    uint32_t rows, items, length, groups, per_group;
    uint32_t row_item, row_at;  // the generator's row: item * row_item + position * row_at
    uint32_t has;  // bits of the tensors that are there
    Divisor by_length;
};

enum { kHasX = 1, kHasH = 2, kHasY = 4, kHasDh = 8, kHasDy = 16, kHasDx = 32, kHasDf = 64, kHasPost = 128 };
// (Compared where it is asked: kept over a loop the conditions take twice the
// scalar registers that there are.)
__device__ __forceinline__ bool has(const NormShape& s, uint32_t bit) {
    uint32_t v = s.has;
    asm("" : "+s"(v));
    return (v & bit) != 0;
}

// Sums over a row's threads.  Beyond a wave through `red`, two buffers in turn.
struct RowSums {
    int lanes;
    float (*red)[1024 / kNormWave][2];
    int turn = 0;
    __device__ __forceinline__ void two(float& u, float& v) {
        u = lanes_sum(u, lanes);
        v = lanes_sum(v, lanes);
        if (lanes <= kNormWave) return;
        turn ^= 1;
        if ((threadIdx.x & (kNormWave - 1)) == 0) {
            red[turn][threadIdx.x / kNormWave][0] = u;
            red[turn][threadIdx.x / kNormWave][1] = v;
        }
        __syncthreads();
        u = v = 0.0f;
        for (int i = 0; i < lanes / kNormWave; ++i) {
            u += red[turn][i][0];
            v += red[turn][i][1];
        }
    }
    __device__ __forceinline__ float one(float v) {
        v = lanes_sum(v, lanes);
        if (lanes <= kNormWave) return v;
        turn ^= 1;
        if ((threadIdx.x & (kNormWave - 1)) == 0) red[turn][threadIdx.x / kNormWave][0] = v;
        __syncthreads();
        v = 0.0f;
        for (int i = 0; i < lanes / kNormWave; ++i) v += red[turn][i][0];
        return v;
    }
};

template <int N>
__device__ __forceinline__ float squares(const float (&e)[N]) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = fmaf(e[i], e[i], s);
    return s;
}

// What a row's values, of sum of squares ss, are multiplied by to be normed.  Values
// whose squares leave fp32 are multiplied by `up` first; then `again` is true and
// sums of the old values do not hold.
template <int N>
__device__ __forceinline__ float norm_factor(float (&e)[N], const ResidualArgs& a, float ss, RowSums& sums, float* up,
                                             bool* again) {
    const float inv = 1.0f / (float)a.channels;
    float eps = a.eps;
    const float f = row_scale(ss, inv, eps);
    *up = f;
    *again = __any(f != 1.0f);  // (the same in all waves of a row)
    if (*again) {
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] *= f;
        ss = sums.one(squares(e));
        eps = f > 1.0f ? a.eps_up : a.eps * f * f;
    }
    return rsqrtf(fmaf(ss, inv, eps));
}

// A thread's first entry of one tensor's rows, on its way from row to row.
template <typename T>
struct Cursor {
    T* p;
    int64_t step;
    __device__ __forceinline__ Cursor(const Rows& t, const NormShape& s, uint32_t item, uint32_t at, int c)
        : p((T*)t.p + item * t.sb + at * t.st + c), step((int64_t)s.slots * t.st) {}
    __device__ __forceinline__ T* next() {
        T* q = p;
        p += step;
        return q;
    }
};
// A chunk of a weight, or of ones.
template <typename T, bool EIGHTS>
__device__ __forceinline__ Raw<T> load_weight(const void* w, int64_t sb, uint32_t item, int c, int left) {
    Raw<T> r;
    r.fill(1.0f);
    return w ? load_raw<T, EIGHTS>((const T*)w + item * sb + c, left) : r;
}

// The items and positions of a call's rows, in a; most: chunks that a thread holds at
// most (in a wave as few idle lanes as can be).
inline NormShape norm_shape(ResidualArgs* a, int most) {
    NormShape s{};
    const int chunks = (a->channels + kChunk - 1) / kChunk;
    if (chunks <= kNormWave * most) {
        int best = 0;
        for (int nv = 1; nv <= most; ++nv) {
            int lanes = 1;
            while (lanes * nv < chunks) lanes *= 2;
            if (lanes > kNormWave || (best && lanes * nv >= best)) continue;
            best = lanes * nv;
            s.lanes = lanes;
            s.nv = nv;
        }
        s.threads = kNormThreads;
    } else {
        s.lanes = 2 * kNormWave;
        while (s.lanes * most < chunks) s.lanes *= 2;
        s.nv = (chunks + s.lanes - 1) / s.lanes;
        s.threads = s.lanes;
    }
    s.slots = s.threads / s.lanes;
    const uint32_t B = a->batch, S = (uint32_t)a->tokens;
    s.rows = B * S;
    s.items = B;
    s.length = S;
    s.row_item = S;
    s.row_at = 1;
    if (!a->post_sb && !a->gate_sb && !a->next_sb) {
        Rows* all[] = {&a->x, &a->f, &a->h, &a->y, &a->dh, &a->dy, &a->dx, &a->df};
        bool dense = true;
        for (const Rows* t : all) dense = dense && (!t->p || t->sb == (int64_t)S * t->st);
        if (dense || B == 1) {
            s.items = 1;
            s.length = s.rows;
        } else if (B > S) {
            std::swap(s.items, s.length);
            std::swap(s.row_item, s.row_at);
            for (Rows* t : all) std::swap(t->sb, t->st);
        }
    }
    s.by_length = divisor(std::max(s.length, 1u));
    const std::pair<const Rows*, uint32_t> there[] = {{&a->x, kHasX},   {&a->h, kHasH},   {&a->y, kHasY},  {&a->dh, kHasDh},
                                                      {&a->dy, kHasDy}, {&a->dx, kHasDx}, {&a->df, kHasDf}};
    for (const auto& t : there) s.has |= t.first->p ? t.second : 0;
    s.has |= a->post ? kHasPost : 0;
    return s;
}
// Cuts the rows into at most `most` runs of whole slots.
inline void norm_runs(NormShape* s, uint32_t most) {
    const uint32_t slots = (uint32_t)s->slots, runs = std::max(1u, std::min((s->rows + slots - 1) / slots, most));
    s->per_group = std::max(1u, ((s->rows + runs - 1) / runs + slots - 1) / slots) * slots;
    s->groups = std::max(1u, (s->rows + s->per_group - 1) / s->per_group);
}

// Calls f with the storage type, whether rows are of whole chunks and whether entries are dropped.
template <typename F>
hipError_t norm_dispatch(const ResidualArgs& a, F&& f) {
    auto dropped = [&](auto t, auto w) { return a.dropped ? f(t, w, std::true_type{}) : f(t, w, std::false_type{}); };
    auto width = [&](auto t) {
        return a.channels % kChunk == 0 ? dropped(t, std::true_type{}) : dropped(t, std::false_type{});
    };
    return a.bf16 ? width(__bf16{}) : width(float{});
}

}  // namespace disco
