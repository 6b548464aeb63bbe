// disco_blocks.h -- arguments and launchers of the residual sum with its norms,
// of dropout and of the gated recurrence, and the device parts that they share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "disco_heads.h"

namespace disco {

// A channel tensor [batch][tokens][channels] as the kernels see it.
struct Rows {
    void* p = nullptr;
    int64_t sb = 0, st = 0;  // strides in elements
};

constexpr int kMaxNormChannels = 8192;  // of a row that is normed
constexpr int kChunk = 8;                // entries of a row that a thread holds together

// ---- dropout (disco_dropout.hip) ---------------------------------------------
struct DropArgs {
    uint32_t out = 0;  // an entry whose 16 bits lie below falls out; 65536: all
    float factor = 1.0f;
    uint32_t key0 = 0, key1 = 0;
    uint64_t offset = 0;
    const uint64_t* counter = nullptr;  // added to the offset
};
struct DropoutArgs {
    Rows x, y;
    DropArgs drop;
    uint32_t batch = 0;
    int64_t tokens = 0, channels = 0;
    bool bf16 = false;
    hipStream_t stream = nullptr;
};
hipError_t launch_dropout(const DropoutArgs& a);

// ---- residual sum with its norms (disco_residual.hip) -------------------------
struct ResidualArgs {
    Rows x, f, h, y, dh, dy, dx, df;
    // x's type; elements between batch items, 0 where all share one
    const void *post_w = nullptr, *gate = nullptr, *next_w = nullptr;
    int64_t post_sb = 0, gate_sb = 0, next_sb = 0;
    void *dpost = nullptr, *dgate = nullptr, *dnext = nullptr;
    DropArgs drop;
    bool dropped = false, post = false, bf16 = false;
    uint32_t batch = 0;
    int64_t tokens = 0;
    int32_t channels = 0;
    float scale = 1.0f, eps = 0.0f, eps_up = 0.0f;  // eps_up: 2^192 eps
    hipStream_t stream = nullptr;
};
hipError_t launch_residual(const ResidualArgs& a);
size_t residual_grad_ws_bytes(const ResidualArgs& a);
hipError_t launch_residual_grad(const ResidualArgs& a, float* ws);

// ---- gated recurrence (disco_recur.hip, disco_recur_grad.hip) -----------------
constexpr int kRun = 16;  // steps between two states that a forward call keeps for its gradients
enum { kGainMean = 0, kGainPower = 1, kGainOne = 2 };
struct RecurArgs {
    Rows x, g, z, y;  // z: the output gate, or none
    Rows dy, dx, dg, dz;
    const int32_t* lengths = nullptr;
    const float* state = nullptr;  // [batch][channels], or zeros
    float* last = nullptr;         // [batch][channels]
    float* carries = nullptr;      // [batch][runs][channels]: the state before each run
    const float* dlast = nullptr;  // [batch][channels]
    float* dstate = nullptr;       // [batch][channels]
    uint32_t batch = 0;
    int64_t steps = 0, channels = 0;
    int gain = 0;
    bool bf16 = false;
    hipStream_t stream = nullptr;
};
size_t recur_ws_bytes(const RecurArgs& a);  // of either direction
hipError_t launch_recur(const RecurArgs& a, float* ws);
hipError_t launch_recur_grad(const RecurArgs& a, float* ws);

// ---- device parts --------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as
// 1, 2, 3; 2011): four words from a counter of four and a key of two.
struct Words {
    uint32_t w[4];
};
__device__ __forceinline__ Words philox(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p = (uint64_t)a * 0xD2511F53u, q = (uint64_t)c * 0xCD9E8D57u;
        a = (uint32_t)(q >> 32) ^ b ^ k0;
        b = (uint32_t)q;
        c = (uint32_t)(p >> 32) ^ d ^ k1;
        d = (uint32_t)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words{{a, b, c, d}};
}
__device__ __forceinline__ uint64_t drop_offset(const DropArgs& d) { return d.offset + (d.counter ? *d.counter : 0); }
// The 16 bits of the entries 8 chunk .. 8 chunk + 7 of a row: one block of the
// generator serves a chunk of either type.
__device__ __forceinline__ Words drop_words(const DropArgs& d, uint64_t offset, uint32_t row, uint32_t chunk) {
    return philox(chunk, row, (uint32_t)offset, (uint32_t)(offset >> 32), d.key0, d.key1);
}
// Whether entry i of the chunk stays.
__device__ __forceinline__ bool stays(const Words& r, int i, uint32_t out) {
    return (i % 2 ? r.w[i / 2] >> 16 : r.w[i / 2] & 0xffffu) >= out;
}

// Eight entries of a row as they lie in memory: bf16 two in a register (as single
// values, once branches meet, they take one each).
template <typename T>
struct Raw;
template <>
struct Raw<__bf16> {
    uint32_t w[kChunk / 2];
    __device__ __forceinline__ float at(int i) const {
        return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void fill(float v) {
#pragma unroll
        for (int i = 0; i < kChunk / 2; ++i) w[i] = (__float_as_uint(v) >> 16) * 0x10001u;
    }
    // A new value to the compiler: without it what a loop does not change is
    // converted before it, into twice the registers.
    __device__ __forceinline__ void anew() {
#pragma unroll
        for (int i = 0; i < kChunk / 2; ++i) asm("" : "+v"(w[i]));
    }
    // Entries i .. i + W - 1
    template <int W>
    __device__ __forceinline__ void load(int i, const __bf16* p) {
        if constexpr (W == 1) {
            const uint32_t v = *(const uint16_t*)p;
            w[i / 2] = i % 2 ? (w[i / 2] & 0xffffu) | v << 16 : (w[i / 2] & 0xffff0000u) | v;
        } else {
            typedef uint32_t U __attribute__((ext_vector_type(W / 2)));
            const U v = *(const U*)p;
#pragma unroll
            for (int j = 0; j < W / 2; ++j) w[i / 2 + j] = v[j];
        }
    }
};
template <>
struct Raw<float> {
    float w[kChunk];
    __device__ __forceinline__ float at(int i) const { return w[i]; }
    __device__ __forceinline__ void fill(float v) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) w[i] = v;
    }
    __device__ __forceinline__ void anew() {}
    template <int W>
    __device__ __forceinline__ void load(int i, const float* p) {
        typedef float U __attribute__((ext_vector_type(W)));
        const U v = *(const U*)p;
#pragma unroll
        for (int j = 0; j < W; ++j) w[i + j] = v[j];
    }
};
// The first eight entries at p, of which `left` are there (perhaps none), W at a time: left and
// the address are multiples of W entries.  Zeros beyond.
template <typename T, int W>
__device__ __forceinline__ Raw<T> load_raw(const T* p, int left) {
    Raw<T> r;
    r.fill(0.0f);
#pragma unroll
    for (int i = 0; i < kChunk; i += W)
        if (i < left) r.template load<W>(i, p + i);
    return r;
}
template <typename T, int W>
__device__ __forceinline__ void store_raw(T* p, int left, const float (&e)[kChunk]) {
    typedef float F __attribute__((ext_vector_type(W)));
    typedef T V __attribute__((ext_vector_type(W)));
#pragma unroll
    for (int i = 0; i < kChunk; i += W) {
        F f;
#pragma unroll
        for (int j = 0; j < W; ++j) f[j] = e[i + j];
        if (i < left) *(V*)(p + i) = __builtin_convertvector(f, V);
    }
}

// Sum over the 2^k neighbouring lanes of a row, in each of them: exchanges within
// quads, eights, sixteens and the wave's halves on the vector unit (through LDS, as
// shuffles go, a row's three sums took longer than its loads).
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
    asm("" : "+s"(lanes));  // (compared here: kept over a loop the conditions spill)
    if (lanes >= 2) v = dpp_add<0xB1>(v);    // lane ^ 1
    if (lanes >= 4) v = dpp_add<0x4E>(v);    // lane ^ 2
    if (lanes >= 8) v = dpp_add<0x141>(v);   // mirrored within eight
    if (lanes >= 16) v = dpp_add<0x140>(v);  // mirrored within sixteen
    if (lanes >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (lanes >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

// Host: whether rows of a tensor are read or written w entries at a time.
inline bool rows_fit(const Rows& t, int w, size_t elem) {
    return !t.p || ((uintptr_t)t.p % (w * elem) == 0 && t.sb % w == 0 && t.st % w == 0);
}

}  // namespace disco
