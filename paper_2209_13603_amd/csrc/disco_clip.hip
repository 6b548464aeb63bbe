// disco_clip.hip -- the global 2-norm of many gradients and clipping by it.
//
//   norm = sqrt(sum g^2),  out = g min(1, max_norm / (norm + eps))
//
// Two launches: the first leaves one 64-bit sum of squares per workgroup, the
// second's workgroups each add all of those in the same order (so that no
// third launch and no atomic is needed, and every run gives the same bits) and
// scale their part.  Small sets take one launch of one workgroup.  Squares
// are added in 64 bits: an fp64 multiply-add a value is still far below the
// memory's time, and no fp32 gradient over- or underflows; the factor is taken
// in 64 bits too, since the norm of finite gradients may pass fp32.  Bound by the
// memory: two reads and a write of every value, the second read from the
// caches where the set fits them.  60 tensors of fp32 and bf16, 1.26 GB: 184 us
// (6.8 TB/s) and 503 us (5.0 TB/s).
//
// The tensors' addresses and sizes travel in the kernel arguments, up to
// kMaxTensors of them a launch: nothing is uploaded, kept or looked up.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "disco_heads.h"
#include "disco_internal.h"

namespace disco {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxTensors = 120;
// Values of one workgroup's piece: 16 KB of fp32 a step keeps four 16-byte
// loads a thread in flight.
constexpr int kPiece = 16 * kThreads;
constexpr int kMaxBlocks = 2048;  // partial sums of one launch: eight workgroups a CU
// Sets up to this many values go to one workgroup of kSmallThreads.
constexpr int64_t kSmallValues = 16384;
constexpr int kSmallThreads = 1024;

struct ClipSet {
    const void* g[kMaxTensors];
    void* out[kMaxTensors];
    int64_t n[kMaxTensors];
    int32_t first[kMaxTensors];  // first piece of each tensor
    uint8_t bf16[kMaxTensors];
    int32_t count, pieces;
};
static_assert(sizeof(ClipSet) <= 3900, "the arguments of a launch");

template <typename T>
struct Wide;
template <>
struct Wide<float> {
    typedef float type __attribute__((ext_vector_type(4)));
    static constexpr int n = 4;
};
template <>
struct Wide<__bf16> {
    typedef __bf16 type __attribute__((ext_vector_type(8)));
    static constexpr int n = 8;
};

// Calls f(value index, vector of W::n values) on [lo, hi) of p: 16-byte loads
// where the address allows, single values before and after (f1).
template <typename T, int THREADS, bool PAST, typename F, typename F1>
__device__ __forceinline__ void walk(const T* p, const T* q, int64_t lo, int64_t hi, F&& f, F1&& f1) {
    typedef typename Wide<T>::type V;
    constexpr int n = Wide<T>::n;
    const int tid = threadIdx.x;
    // p and q (the output, or p itself) step together: vectors need both on the
    // same 16-byte phase.
    const int64_t off = ((16 - (int64_t)((uintptr_t)(p + lo) & 15)) & 15) / (int64_t)sizeof(T);
    const bool wide = (((uintptr_t)p ^ (uintptr_t)q) & 15) == 0;
    const int64_t head = wide ? (off < hi - lo ? lo + off : hi) : hi;
    for (int64_t i = lo + tid; i < head; i += THREADS) f1(i);
    const int64_t vecs = (hi - head) / n;
    constexpr int U = 4;
    for (int64_t i = tid; i < vecs; i += U * THREADS) {
        V v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * THREADS < vecs) {
                const V* at = (const V*)(p + head + (i + u * THREADS) * n);
                if constexpr (PAST) v[u] = __builtin_nontemporal_load(at);
                else v[u] = *at;
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * THREADS < vecs) f(head + (i + u * THREADS) * n, v[u]);
    }
    for (int64_t i = head + vecs * n + tid; i < hi; i += THREADS) f1(i);
}

template <typename T, int THREADS, bool PAST>
__device__ __forceinline__ double squares(const T* p, int64_t lo, int64_t hi) {
    double s = 0.0;
    walk<T, THREADS, PAST>(
        p, p, lo, hi,
        [&](int64_t, auto v) {
#pragma unroll
            for (int j = 0; j < Wide<T>::n; ++j) {
                const double d = (double)(float)v[j];
                s = fma(d, d, s);
            }
        },
        [&](int64_t i) {
            const double d = (double)(float)p[i];
            s = fma(d, d, s);
        });
    return s;
}

// The factor in two: what is below the normal values of fp32 keeps its bits.
struct Factor {
    float first, second;
    __device__ __forceinline__ bool one() const { return first == 1.0f && second == 1.0f; }
};

template <typename T, int THREADS>
__device__ __forceinline__ void scale(const T* p, T* q, int64_t lo, int64_t hi, Factor c) {
    walk<T, THREADS, false>(
        p, q, lo, hi,
        [&](int64_t i, auto v) {
            typedef decltype(v) V;
            V r;
#pragma unroll
            for (int j = 0; j < Wide<T>::n; ++j) r[j] = (T)((float)v[j] * c.first * c.second);
            *(V*)(q + i) = r;
        },
        [&](int64_t i) { q[i] = (T)((float)p[i] * c.first * c.second); });
}

// Sum over the workgroup, the same value in every thread.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double red[THREADS / 64];
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    for (int i = 0; i < THREADS / 64; ++i) s += red[i];
    return s;
}

__device__ __forceinline__ Factor factor(double total, double max_norm, double eps, float* norm) {
    const double n = sqrt(total);
    if (norm && threadIdx.x == 0) *norm = (float)n;
    const double q = max_norm / (n + eps), c = q > 1.0 ? 1.0 : q;  // NaN stays
    const float first = c < 0x1p-126 ? 0x1p-126f : 1.0f;
    return Factor{first, (float)(c / first)};
}

// Calls f(tensor, lo, hi) on this workgroup's pieces: every gridDim.x-th, so
// that the workgroups sweep the memory side by side (each on a stretch of its
// own: 256 and 493 us for 1.26 GB, 249 and 483 us so).
template <typename F>
__device__ __forceinline__ void pieces_of(const ClipSet& s, F&& f) {
    int t = 0;
    for (int64_t p = blockIdx.x; p < s.pieces; p += gridDim.x) {
        while (t + 1 < s.count && s.first[t + 1] <= p) ++t;
        const int64_t lo = (p - s.first[t]) * kPiece;
        f(t, lo, min(lo + kPiece, s.n[t]));
    }
}

// PAST: the loads leave no trace in the caches.
template <bool PAST>
__global__ __launch_bounds__(kThreads) void k_clip_squares(ClipSet s, double* __restrict__ partial) {
    double v = 0.0;
    pieces_of(s, [&](int t, int64_t lo, int64_t hi) {
        v += s.bf16[t] ? squares<__bf16, kThreads, PAST>((const __bf16*)s.g[t], lo, hi)
                       : squares<float, kThreads, PAST>((const float*)s.g[t], lo, hi);
    });
    v = block_sum<kThreads>(v);
    if (threadIdx.x == 0) partial[blockIdx.x] = v;
}

// norm is written by the launch that is given it.
__global__ __launch_bounds__(kThreads) void k_clip_scale(ClipSet s, const double* __restrict__ partial, int n_partial,
                                                         double max_norm, double eps, float* __restrict__ norm) {
    double v = 0.0;
    for (int i = threadIdx.x; i < n_partial; i += kThreads) v += partial[i];
    const Factor c = factor(block_sum<kThreads>(v), max_norm, eps, blockIdx.x == 0 ? norm : nullptr);
    pieces_of(s, [&](int t, int64_t lo, int64_t hi) {
        if (!s.out[t] || (c.one() && s.out[t] == s.g[t])) return;
        if (s.bf16[t]) scale<__bf16, kThreads>((const __bf16*)s.g[t], (__bf16*)s.out[t], lo, hi, c);
        else scale<float, kThreads>((const float*)s.g[t], (float*)s.out[t], lo, hi, c);
    });
}

__global__ __launch_bounds__(kSmallThreads) void k_clip_small(ClipSet s, double max_norm, double eps,
                                                              float* __restrict__ norm) {
    double v = 0.0;
    for (int t = 0; t < s.count; ++t)
        v += s.bf16[t] ? squares<__bf16, kSmallThreads, false>((const __bf16*)s.g[t], 0, s.n[t])
                       : squares<float, kSmallThreads, false>((const float*)s.g[t], 0, s.n[t]);
    const Factor c = factor(block_sum<kSmallThreads>(v), max_norm, eps, norm);
    for (int t = 0; t < s.count; ++t) {
        if (!s.out[t] || (c.one() && s.out[t] == s.g[t])) continue;
        if (s.bf16[t]) scale<__bf16, kSmallThreads>((const __bf16*)s.g[t], (__bf16*)s.out[t], 0, s.n[t], c);
        else scale<float, kSmallThreads>((const float*)s.g[t], (float*)s.out[t], 0, s.n[t], c);
    }
}

// A launch's worth of tensors from `at` on, skipping empty ones; returns where the next begins.
int fill(const ClipTensor* t, int n, int at, ClipSet* s) {
    s->count = 0;
    int64_t pieces = 0;
    for (; at < n && s->count < kMaxTensors; ++at) {
        if (t[at].n == 0) continue;
        const int64_t more = (t[at].n + kPiece - 1) / kPiece;
        if (pieces + more > 0x7fffffff && s->count > 0) break;
        const int i = s->count++;
        s->g[i] = t[at].g;
        s->out[i] = t[at].out;
        s->n[i] = t[at].n;
        s->bf16[i] = t[at].bf16;
        s->first[i] = (int32_t)pieces;
        pieces += more;
    }
    s->pieces = (int32_t)std::min<int64_t>(pieces, 0x7fffffff);
    return at;
}

int blocks_of(const ClipSet& s) { return std::max(1, std::min(s.pieces, kMaxBlocks)); }

bool small_set(const ClipTensor* t, int n, int64_t* total) {
    int count = 0;
    *total = 0;
    for (int i = 0; i < n; ++i) *total += t[i].n, count += t[i].n > 0;
    return *total <= kSmallValues && count <= kMaxTensors;
}

}  // namespace

size_t clip_ws_bytes(const ClipTensor* t, int n) {
    int64_t total;
    if (small_set(t, n, &total)) return 0;
    size_t blocks = 0;
    ClipSet s;
    for (int at = 0; at < n;) {
        at = fill(t, n, at, &s);
        if (s.count) blocks += (size_t)blocks_of(s);
    }
    return blocks * sizeof(double);
}

hipError_t launch_clip(const ClipTensor* t, int n, double max_norm, double eps, float* norm, void* ws,
                       hipStream_t stream) {
    ClipSet s;
    int64_t total;
    if (small_set(t, n, &total)) {
        fill(t, n, 0, &s);
        const int tk = timing_begin("clip_small", stream);
        hipLaunchKernelGGL(k_clip_small, dim3(1), dim3(kSmallThreads), 0, stream, s, max_norm, eps, norm);
        timing_end(tk, stream);
        return hipGetLastError();
    }
    double* partial = (double*)ws;
    int done = 0;
    // A set beyond the 256 MB cache is read past it: 1.26 GB in 190 us instead
    // of 249.  A smaller one stays there for the second pass.
    int64_t bytes = 0;
    for (int i = 0; i < n; ++i) bytes += t[i].n * (t[i].bf16 ? 2 : 4);
    const bool past = bytes > (int64_t)256 << 20;
    bool write = false;
    for (int at = 0; at < n;) {
        at = fill(t, n, at, &s);
        if (!s.count) break;
        const int tk = timing_begin("clip_squares", stream);
        const dim3 grid((unsigned)blocks_of(s));
        if (past) hipLaunchKernelGGL(k_clip_squares<true>, grid, dim3(kThreads), 0, stream, s, partial + done);
        else hipLaunchKernelGGL(k_clip_squares<false>, grid, dim3(kThreads), 0, stream, s, partial + done);
        timing_end(tk, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        done += blocks_of(s);
        for (int i = 0; i < s.count; ++i) write = write || s.out[i];
    }
    for (int at = 0; at < n;) {
        const bool first = at == 0;
        at = fill(t, n, at, &s);
        if (!s.count && !first) break;
        const int tk = timing_begin("clip_scale", stream);
        hipLaunchKernelGGL(k_clip_scale, dim3((unsigned)(write ? blocks_of(s) : 1)), dim3(kThreads), 0, stream, s,
                           partial, done, max_norm, eps, first ? norm : nullptr);
        timing_end(tk, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (!write) break;
    }
    return hipSuccess;
}

}  // namespace disco
