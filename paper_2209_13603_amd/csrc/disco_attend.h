// disco_attend.h -- device helpers shared by the cross-attention kernels.
#pragma once
#include <hip/hip_runtime.h>

#include "disco_heads.h"

namespace disco {

constexpr float kLog2e = 1.4426950408889634f;

// Keys of batch item b that its length leaves.
__device__ __forceinline__ int64_t key_count(const AttendArgs& a, int b) {
    if (!a.lengths) return a.keys;
    const int64_t n = a.lengths[b];
    return n < 0 ? 0 : n > a.keys ? a.keys : n;
}

// The bias of a key in units of log 2: -inf takes the key out, finite values
// stay finite (a mask of the type's lowest value must not become -inf).
__device__ __forceinline__ float bias2_of(float bias) {
    const float t = bias * kLog2e;
    return bias < -0x1p+127f && bias != -INFINITY ? -0x1p+127f * kLog2e : t;
}
__device__ __forceinline__ float key_bias2(const AttendArgs& a, int b, int64_t j) {
    return a.bias ? bias2_of(a.bias[b * a.bias_sb + j]) : 0.0f;
}

}  // namespace disco
