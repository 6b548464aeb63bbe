// disco_heads.h -- arguments and launchers of the token kernels (head norm and
// rotation, cross attention) and of gradient clipping.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "disco.h"
#include "disco_launch.h"

namespace disco {

// A token tensor [batch][tokens][heads][dim] as the kernels see it.
struct Heads {
    void* p = nullptr;
    int64_t sb = 0, st = 0, sh = 0;  // strides in elements
};

constexpr int kMaxHeadDim = 128;

inline dim3 grid_dim(uint32_t groups) {
    const Grid g = grid_of(groups);
    return dim3(g.x, g.y);
}
// The workgroup's place in a grid of grid_dim.
__device__ __forceinline__ uint32_t group_index() { return blockIdx.y * gridDim.x + blockIdx.x; }

// ---- head norm and rotation (disco_rotate.hip) ------------------------------
struct RotateArgs {
    Heads x, y, dy, dx;
    const void* weight = nullptr;  // x's type
    void* dweight = nullptr;
    int64_t weight_sh = 0;  // elements between heads: dim, or 0 for one weight
    const float* cosines = nullptr;
    const float* sines = nullptr;
    int64_t rows = 0;
    const int32_t* positions = nullptr;
    int64_t pos_sb = 0, pos0 = 0;
    int32_t batch = 0, heads = 0, dim = 0, rotary = 0;
    int64_t tokens = 0;
    float eps = 0.0f, eps_up = 0.0f;  // eps_up: 2^192 eps
    bool norm = false, interleaved = false, bf16 = false;
    hipStream_t stream = nullptr;
};
hipError_t launch_rotate(const RotateArgs& a);
size_t rotate_grad_ws_bytes(const RotateArgs& a);
hipError_t launch_rotate_grad(const RotateArgs& a, float* ws);

// ---- cross attention (disco_attend.hip, disco_attend_grad.hip) ---------------
struct AttendArgs {
    Heads q, k, v, out, dout, dq, dk, dv;
    Heads low;  // bf16: what rounding took from out, kept for the gradients
    const float* bias = nullptr;
    int64_t bias_sb = 0;
    const int32_t* lengths = nullptr;
    float* stats = nullptr;  // [batch][heads][queries][2]
    int32_t batch = 0, heads = 0, kv_heads = 0, dim = 0;
    int64_t queries = 0, keys = 0;
    float scale2 = 0.0f;  // scale / log 2: the scores in units of log 2
    float scale = 0.0f;
    float bias_limit = 0.0f;  // finite biases stay within it, in units of the scale
    bool bf16 = false;
    hipStream_t stream = nullptr;
};
size_t attend_ws_bytes(const AttendArgs& a);
hipError_t launch_attend(const AttendArgs& a, void* ws);
size_t attend_grad_ws_bytes(const AttendArgs& a);
hipError_t launch_attend_grad(const AttendArgs& a, void* ws);

// ---- gradient clipping (disco_clip.hip) --------------------------------------
struct ClipTensor {
    const void* g;
    void* out;  // nullptr: the norm alone
    int64_t n;
    bool bf16;
};
size_t clip_ws_bytes(const ClipTensor* t, int n);
hipError_t launch_clip(const ClipTensor* t, int n, double max_norm, double eps, float* norm, void* ws,
                       hipStream_t stream);

}  // namespace disco
