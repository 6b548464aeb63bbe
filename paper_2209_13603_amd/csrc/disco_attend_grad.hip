// disco_attend_grad.hip -- gradients of cross attention.
//
//   delta_i = dout_i . out_i,   ds_ij = p_ij (dout_i . v_j - delta_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij dout_i
// with p rebuilt from the row maximum and sum that the forward call left.
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

// p_ij from the row's statistics; 0 where the row has no key.
__device__ __forceinline__ float weight(float t, float m, float l) {
    return l == 0.0f ? 0.0f : exp2f(t - m) / l;
}

// One workgroup a query row; grid: (queries, batch * heads).
template <typename T>
__global__ __launch_bounds__(kTile) void k_attend_dq(AttendArgs a) {
    __shared__ float s[kTile], acc[kTile];
    const int64_t i = blockIdx.x;
    const int b = blockIdx.y / a.heads, h = blockIdx.y % a.heads, hk = h / (a.heads / a.kv_heads);
    const T* q = (const T*)a.q.p + b * a.q.sb + i * a.q.st + h * a.q.sh;
    const T* o = (const T*)a.out.p + b * a.out.sb + i * a.out.st + h * a.out.sh;
    const T* g = (const T*)a.dout.p + b * a.dout.sb + i * a.dout.st + h * a.dout.sh;
    const T* k = (const T*)a.k.p + b * a.k.sb + hk * a.k.sh;
    const T* v = (const T*)a.v.p + b * a.v.sb + hk * a.v.sh;
    const float* st = a.stats + ((int64_t)blockIdx.y * a.queries + i) * 2;
    const float m = st[0], l = st[1], delta = dot(g, o, a.dim);
    const int64_t n = key_count(a, b);
    const int dp = a.dim <= 32 ? 32 : a.dim <= 64 ? 64 : 128, d = threadIdx.x % dp, slice = threadIdx.x / dp;
    float sum = 0.0f;
    for (int64_t j0 = 0; j0 < n; j0 += kTile) {
        const int64_t j = j0 + threadIdx.x;
        float ds = 0.0f;
        if (j < n) {
            const float bias2 = key_bias2(a, b, j);
            if (bias2 != -INFINITY)
                ds = weight(fmaf(dot(q, k + j * a.k.st, a.dim), a.scale2, bias2), m, l) *
                     (dot(g, v + j * a.v.st, a.dim) - delta);
        }
        __syncthreads();
        s[threadIdx.x] = ds;
        __syncthreads();
        if (d < a.dim)
            for (int u = slice; u < kTile && j0 + u < n; u += kTile / dp)
                if (s[u] != 0.0f) sum = fmaf(s[u], (float)k[(j0 + u) * a.k.st + d], sum);
    }
    acc[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x < a.dim) {
        float r = 0.0f;
        for (int u = threadIdx.x; u < kTile; u += dp) r += acc[u];
        ((T*)a.dq.p + b * a.dq.sb + i * a.dq.st + h * a.dq.sh)[threadIdx.x] = (T)(r * a.scale);
    }
}

// One workgroup a key; grid: (keys, batch * kv_heads).
template <typename T>
__global__ __launch_bounds__(kTile) void k_attend_dkv(AttendArgs a) {
    __shared__ float s[kTile], w[kTile], acc[2][kTile];
    const int64_t j = blockIdx.x;
    const int b = blockIdx.y / a.kv_heads, hk = blockIdx.y % a.kv_heads, group = a.heads / a.kv_heads;
    const T* k = (const T*)a.k.p + b * a.k.sb + j * a.k.st + hk * a.k.sh;
    const T* v = (const T*)a.v.p + b * a.v.sb + j * a.v.st + hk * a.v.sh;
    const float bias2 = key_bias2(a, b, j);
    const bool live = j < key_count(a, b) && bias2 != -INFINITY;
    const int dp = a.dim <= 32 ? 32 : a.dim <= 64 ? 64 : 128, d = threadIdx.x % dp, slice = threadIdx.x / dp;
    float dk = 0.0f, dv = 0.0f;
    for (int h = hk * group; live && h < (hk + 1) * group; ++h) {
        const T* q = (const T*)a.q.p + b * a.q.sb + h * a.q.sh;
        const T* o = (const T*)a.out.p + b * a.out.sb + h * a.out.sh;
        const T* g = (const T*)a.dout.p + b * a.dout.sb + h * a.dout.sh;
        const float* st = a.stats + (int64_t)(b * a.heads + h) * a.queries * 2;
        for (int64_t i0 = 0; i0 < a.queries; i0 += kTile) {
            const int64_t i = i0 + threadIdx.x;
            float p = 0.0f, ds = 0.0f;
            if (i < a.queries) {
                p = weight(fmaf(dot(q + i * a.q.st, k, a.dim), a.scale2, bias2), st[2 * i], st[2 * i + 1]);
                ds = p * (dot(g + i * a.dout.st, v, a.dim) - dot(g + i * a.dout.st, o + i * a.out.st, a.dim));
            }
            __syncthreads();
            s[threadIdx.x] = ds;
            w[threadIdx.x] = p;
            __syncthreads();
            if (d < a.dim)
                for (int u = slice; u < kTile && i0 + u < a.queries; u += kTile / dp) {
                    dk = fmaf(s[u], (float)q[(i0 + u) * a.q.st + d], dk);
                    dv = fmaf(w[u], (float)g[(i0 + u) * a.dout.st + d], dv);
                }
        }
    }
    acc[0][threadIdx.x] = dk;
    acc[1][threadIdx.x] = dv;
    __syncthreads();
    if (threadIdx.x < a.dim) {
        float rk = 0.0f, rv = 0.0f;
        for (int u = threadIdx.x; u < kTile; u += dp) rk += acc[0][u], rv += acc[1][u];
        ((T*)a.dk.p + b * a.dk.sb + j * a.dk.st + hk * a.dk.sh)[threadIdx.x] = (T)(rk * a.scale);
        ((T*)a.dv.p + b * a.dv.sb + j * a.dv.st + hk * a.dv.sh)[threadIdx.x] = (T)rv;
    }
}

template <typename T>
hipError_t launch(const AttendArgs& a) {
    int tk = timing_begin("attend_dq", a.stream);
    if (a.queries > 0)
        hipLaunchKernelGGL(k_attend_dq<T>, dim3((unsigned)a.queries, (unsigned)(a.batch * a.heads)), dim3(kTile), 0,
                           a.stream, a);
    timing_end(tk, a.stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.keys == 0) return e;
    tk = timing_begin("attend_dkv", a.stream);
    hipLaunchKernelGGL(k_attend_dkv<T>, dim3((unsigned)a.keys, (unsigned)(a.batch * a.kv_heads)), dim3(kTile), 0,
                       a.stream, a);
    timing_end(tk, a.stream);
    return hipGetLastError();
}

}  // namespace

size_t attend_grad_ws_bytes(const AttendArgs&) { return 0; }

hipError_t launch_attend_grad(const AttendArgs& a, void*) { return a.bf16 ? launch<__bf16>(a) : launch<float>(a); }

}  // namespace disco
