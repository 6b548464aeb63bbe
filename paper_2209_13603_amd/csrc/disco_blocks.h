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

// Pieces of rows at any address of their entries' alignment: the memory takes these
// loads and stores whole (entry by entry, rows of 167 in bf16 took three times as long).
typedef uint32_t Any4 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t Any2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t Any1 __attribute__((aligned(2)));
typedef float Any4f __attribute__((ext_vector_type(4), aligned(4)));
typedef float Any2f __attribute__((ext_vector_type(2), aligned(4)));

// One of two values (of the values, not of their places).
template <typename X>
__device__ __forceinline__ X pick(bool first, X a, X b) {
    return first ? a : b;
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
    __device__ __forceinline__ void load(const __bf16* p) {
        const Any4 v = *(const Any4*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = v[i];
    }
    // The first `left` < 8 entries: pieces of four, two and one.
    __device__ __forceinline__ void load(const __bf16* p, int left) {
        uint32_t four[2] = {0u, 0u}, two = 0u, one = 0u;
        if (left & 4) {
            const Any2 v = *(const Any2*)p;
            four[0] = v[0], four[1] = v[1];
        }
        if (left & 2) two = *(const Any1*)(p + (left & 4));
        if (left & 1) one = *(const uint16_t*)(p + (left & 6));
        const bool q = left & 4, h = left & 2;
        const uint32_t a = pick(h, two, one), b = pick(h, one, 0u);
        w[0] = pick(q, four[0], a);
        w[1] = pick(q, four[1], b);
        w[2] = pick(q, a, 0u);
        w[3] = pick(q, b, 0u);
    }
    __device__ __forceinline__ void pack(const float (&e)[kChunk]) {
#pragma unroll
        for (int i = 0; i < kChunk / 2; ++i) {
            typedef float F __attribute__((ext_vector_type(2)));
            typedef __bf16 B __attribute__((ext_vector_type(2)));
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((F{e[2 * i], e[2 * i + 1]}), B));
        }
    }
    __device__ __forceinline__ void store(__bf16* p) const { *(Any4*)p = Any4{w[0], w[1], w[2], w[3]}; }
    __device__ __forceinline__ void store(__bf16* p, int left) const {
        if (left & 4) *(Any2*)p = Any2{w[0], w[1]};
        const uint32_t a = pick<uint32_t>(left & 4, w[2], w[0]), b = pick<uint32_t>(left & 4, w[3], w[1]);
        if (left & 2) *(Any1*)(p + (left & 4)) = a;
        if (left & 1) *(uint16_t*)(p + (left & 6)) = (uint16_t)pick<uint32_t>(left & 2, b, a);
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
    __device__ __forceinline__ void load(const float* p) {
        const Any4f u = *(const Any4f*)p, v = *(const Any4f*)(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = u[i], w[4 + i] = v[i];
    }
    __device__ __forceinline__ void load(const float* p, int left) {
        float four[4] = {0.0f}, two[2] = {0.0f}, one = 0.0f;
        if (left & 4) {
            const Any4f v = *(const Any4f*)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) four[i] = v[i];
        }
        if (left & 2) two[0] = p[left & 4], two[1] = p[(left & 4) + 1];
        if (left & 1) one = p[left & 6];
        const bool q = left & 4, h = left & 2;
        const float r[4] = {pick(h, two[0], one), pick(h, two[1], 0.0f), pick(h, one, 0.0f), 0.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = pick(q, four[i], r[i]);
            w[4 + i] = pick(q, r[i], 0.0f);
        }
    }
    __device__ __forceinline__ void pack(const float (&e)[kChunk]) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) w[i] = e[i];
    }
    __device__ __forceinline__ void store(float* p) const {
        *(Any4f*)p = Any4f{w[0], w[1], w[2], w[3]};
        *(Any4f*)(p + 4) = Any4f{w[4], w[5], w[6], w[7]};
    }
    __device__ __forceinline__ void store(float* p, int left) const {
        if (left & 4) *(Any4f*)p = Any4f{w[0], w[1], w[2], w[3]};
        float r[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) r[i] = pick<float>(left & 4, w[4 + i], w[i]);
        if (left & 2) p[left & 4] = r[0], p[(left & 4) + 1] = r[1];
        if (left & 1) p[left & 6] = pick<float>(left & 2, r[2], r[0]);
    }
};
// The first eight entries at p, of which `left` are there (perhaps none): zeros beyond.  EIGHTS:
// rows are of whole chunks.
template <typename T, bool EIGHTS>
__device__ __forceinline__ Raw<T> load_raw(const T* p, int left) {
    Raw<T> r;
    r.fill(0.0f);
    if (left >= kChunk) r.load(p);
    else if (!EIGHTS && left > 0) r.load(p, left);
    return r;
}
template <typename T, bool EIGHTS>
__device__ __forceinline__ void store_raw(T* p, int left, const float (&e)[kChunk]) {
    Raw<T> r;
    r.pack(e);
    if (left >= kChunk) r.store(p);
    else if (!EIGHTS && left > 0) r.store(p, left);
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

}  // namespace disco
