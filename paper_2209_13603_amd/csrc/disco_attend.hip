// disco_attend.hip -- cross attention, forward.
//
// Scores are held in units of log 2: t_ij = scale2 q_i.k_j + bias2_j, and
// p_ij = 2^(t_ij - m_i) / l_i with the running row maximum m and sum l, fp32.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "disco_attend.h"
#include "disco_internal.h"

namespace disco {

namespace {

constexpr int kTile = 256;

template <typename T>
__device__ __forceinline__ float dot(const T* a, const T* b, int D) {
    float s = 0.0f;
    for (int d = 0; d < D; ++d) s = fmaf((float)a[d], (float)b[d], s);
    return s;
}

__device__ __forceinline__ float block_max(float v, float* red) {
    for (int m = 32; m > 0; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

// One workgroup a query row; grid: (queries, batch * heads).
template <typename T>
__global__ __launch_bounds__(kTile) void k_attend(AttendArgs a) {
    __shared__ float p[kTile], red[4], acc[kTile];
    const int64_t i = blockIdx.x;
    const int b = blockIdx.y / a.heads, h = blockIdx.y % a.heads, hk = h / (a.heads / a.kv_heads);
    const T* q = (const T*)a.q.p + b * a.q.sb + i * a.q.st + h * a.q.sh;
    const T* k = (const T*)a.k.p + b * a.k.sb + hk * a.k.sh;
    const T* v = (const T*)a.v.p + b * a.v.sb + hk * a.v.sh;
    const int64_t n = key_count(a, b);
    const int dp = a.dim <= 32 ? 32 : a.dim <= 64 ? 64 : 128, d = threadIdx.x % dp, slice = threadIdx.x / dp;
    float m = -INFINITY, l = 0.0f, o = 0.0f;
    for (int64_t j0 = 0; j0 < n; j0 += kTile) {
        const int64_t j = j0 + threadIdx.x;
        float t = -INFINITY;
        if (j < n) {
            const float bias2 = key_bias2(a, b, j);
            if (bias2 != -INFINITY) t = fmaf(dot(q, k + j * a.k.st, a.dim), a.scale2, bias2);
        }
        const float m1 = fmaxf(m, block_max(t, red)), ms = m1 == -INFINITY ? 0.0f : m1;
        const float e = exp2f(t - ms), f = exp2f(m - ms);
        p[threadIdx.x] = e;
        l = l * f + e;
        o *= f;
        m = m1;
        __syncthreads();
        if (d < a.dim)
            for (int u = slice; u < kTile && j0 + u < n; u += kTile / dp)
                if (p[u] != 0.0f) o = fmaf(p[u], (float)v[(j0 + u) * a.v.st + d], o);
    }
    acc[threadIdx.x] = o;
    __syncthreads();
    for (int w = 32; w > 0; w >>= 1) l += __shfl_xor(l, w);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = l;
    __syncthreads();
    l = red[0] + red[1] + red[2] + red[3];
    if (threadIdx.x < a.dim) {
        float s = 0.0f;
        for (int u = threadIdx.x; u < kTile; u += dp) s += acc[u];
        T* out = (T*)a.out.p + b * a.out.sb + i * a.out.st + h * a.out.sh;
        out[threadIdx.x] = (T)(l == 0.0f ? 0.0f : s / l);
    }
    if (a.stats && threadIdx.x == 0) {
        float* st = a.stats + ((int64_t)blockIdx.y * a.queries + i) * 2;
        st[0] = m;
        st[1] = l;
    }
}

}  // namespace

size_t attend_ws_bytes(const AttendArgs&) { return 0; }

hipError_t launch_attend(const AttendArgs& a, void*) {
    const dim3 grid((unsigned)a.queries, (unsigned)(a.batch * a.heads));
    const int tk = timing_begin("attend", a.stream);
    if (a.bf16) hipLaunchKernelGGL(k_attend<__bf16>, grid, dim3(kTile), 0, a.stream, a);
    else hipLaunchKernelGGL(k_attend<float>, grid, dim3(kTile), 0, a.stream, a);
    timing_end(tk, a.stream);
    return hipGetLastError();
}

}  // namespace disco
