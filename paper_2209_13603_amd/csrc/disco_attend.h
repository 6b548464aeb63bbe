// disco_attend.h -- device parts shared by the cross-attention kernels.
//
// All products run on matrix-core tiles of 32 x 32 whose column is a lane's own
// (lane % 32), so that the softmax of a row, which stands in the columns of the
// transposed scores, needs one exchange between two lanes and no broadcast.
//
//   scores  S[32 rows of an LDS tile][32 columns] += tile x fragments, the
//           fragments (one vector of `dim` entries a column) in registers;
//   values  O[32 entries d][32 columns] += tile^T x P, P in the layout that the
//           scores leave: lane n + 32 h holds in register i the column n of row
//           8 (i / 4) + 4 h + i % 4.  The sum over rows may run in any order, so
//           P goes back into the matrix cores as it lies and the tile is read in
//           that order.
//
// bf16 takes v_mfma_f32_32x32x16_bf16 and the transposing LDS read; fp32 takes
// v_mfma_f32_32x32x2_f32 (its operands are single values, so nothing needs to be
// transposed) and is exact to fp32 rounding.
//
// LDS tile: chunks of 16 bytes, 16 rows x 4 chunks to a segment of 1 KB, chunk c
// of row r at (r % 16) * 64 + ((c % 4) ^ (r / 4 % 4)) * 16.  Row reads (a lane a
// row, 16 bytes), transposed reads (4 rows x 16 entries) and the staging writes (4
// lanes a row) all spread over the banks, and every address is a lane's own
// offset plus a constant.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "disco_heads.h"

namespace disco {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f8 __attribute__((ext_vector_type(8)));
typedef float f16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char lds_t;

constexpr int kWave = 64;
constexpr int kAttendWaves = kAttendThreads / kWave;
// References m of a softmax row beyond this, in units of log 2, are far: see
// near_reference.
constexpr float kFarReference = 0x1p+12f;

// Keys of batch item b that its length leaves.
__device__ __forceinline__ int64_t key_count(const AttendArgs& a, int b) {
    if (!a.lengths) return a.keys;
    const int64_t n = a.lengths[b];
    return n < 0 ? 0 : n > a.keys ? a.keys : n;
}

// What a key's score starts from, in units of the scale (positive here): the
// product is added onto it in the matrix cores.  Finite biases stay within
// `limit`: a mask of the type's lowest value takes no key out, and must not
// become -inf on the way.
__device__ __forceinline__ float start_of(float bias, float inv_scale, float limit) {
    const float t = bias * inv_scale;
    return fabsf(bias) < INFINITY ? fminf(fmaxf(t, -limit), limit) : t;
}

// A score's exponent against its row's reference -neg: the product rounded to
// fp32, as the reference was, so that the largest score's exponent is 0
// whatever its size, and then the difference, which is exact where it matters.
__device__ __forceinline__ float exponent(float s, float scale2, float neg) {
#pragma clang fp contract(off)
    const float t = s * scale2;
    return t + neg;
}
// The forward pass, which has no instruction to spare, takes one multiply-add
// s scale2 - m instead where m is near: the product is then exact, and what
// rounding took from m (half a spacing, 2^-13 below the line) is in every
// weight of the row and leaves their quotients.  Of a far m, the -1e10 of a mask, it
// would be an exponent of hundreds: infinite weights or none.  Returns what to
// add to the products of a lane's column s; a far row's scores become their
// differences from the reference first.  (32768 queries of 8 heads to
// 8192 keys: rounded products for every row 690 us, so 671.)
template <int N>
__device__ __forceinline__ float near_reference(f16 (&s)[N], float scale2, float neg) {
    const bool far = fabsf(neg) > kFarReference && fabsf(neg) < INFINITY;
    if (__any(far)) {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[k][r] = far ? exponent(s[k][r], scale2, neg) / scale2 : s[k][r];
    }
    return far ? 0.0f : neg;
}

// Workgroups go round the XCDs one by one: gives each XCD runs of `run`
// consecutive work items, which share keys, values or queries in its L2.
__device__ __forceinline__ uint32_t xcd_item(uint32_t run) {
    const uint32_t at = group_index(), k = at / 8;
    return (k / run * 8 + at % 8) * run + k % run;
}
inline dim3 xcd_grid(uint32_t n, uint32_t run) { return grid_dim(((n + run - 1) / run + 7) / 8 * 8 * run); }
// One run an XCD where all items cost the same.  With lengths, which the host
// does not see, whole runs may have nothing to do: eight and more an XCD (3 x
// 4050 queries of 5 heads, fp32, 1013, 845 and no keys: the step 615 us with one run, 458 us so).
inline uint32_t xcd_run(const AttendArgs& a, uint32_t n) { return (n + (a.lengths ? 63 : 7)) / (a.lengths ? 64 : 8) + (n == 0); }

// First of the tiles of part `part` when `tiles` are dealt to `parts`.
__device__ __forceinline__ int first_tile(int tiles, int part, int parts) {
    const int q = tiles / parts, r = tiles % parts;
    return q * part + min(part, r);
}

template <int N>
__device__ __forceinline__ void clear(f16 (&o)[N]) {
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
}

// (Selects: a branch behind the loop has cost registers in it, fp32 heads of 36
// 100 -> 125 us.)
template <int N>
__device__ __forceinline__ void clear_if(bool yes, f16 (&o)[N]) {
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = yes ? 0.0f : o[d][r];
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

template <int N, typename F>
__device__ __forceinline__ void flip(F (&f)[N], uint32_t mask) {
    asm("" : "+v"(mask));  // not known to the compiler: the operation stays
#pragma unroll
    for (int s = 0; s < N; ++s) f[s] = __builtin_bit_cast(F, __builtin_bit_cast(u4, f[s]) ^ mask);
}

template <typename T>
struct Mat;
template <>
struct Mat<__bf16> {
    typedef bf8 Frag;
    static constexpr int CH = 8;  // entries of a chunk
    // The fragments with the sign of `by`.  (Done before a loop it also ends the
    // wait for their loads there; otherwise every round of the loop waits for
    // all loads under way.)
    template <int N>
    static __device__ __forceinline__ void sign(Frag (&f)[N], float by) {
        const uint32_t mask = (__float_as_uint(by) >> 31) * 0x80008000u;
        flip<N>(f, mask);
    }
    static __device__ __forceinline__ f16 scores(Frag a, Frag b, f16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    // P as the values' operand, and in the gradients P and dS: rounded to nearest,
    // which the bf16 instructions need (fp32 ones run at an eighth of the rate).
    // Each term carries a rounding of 2^-8 at most, as the result does: outputs are
    // 2.1e-3 to 2.5e-3 from the definition in 64 bits, where a single rounding
    // leaves 1.7e-3.  In two bf16 parts each they would leave that too, for 43 % more
    // time forward (32768 x 8192, heads of 64: 670 -> 960 us; heads of 128 300 ->
    // 393) and 24 % for dq (413 -> 512).  Sums, softmax statistics and the row sums of the
    // gradients stay in fp32, and fp32 calls round nothing on the way.
    struct Probs {
        bf8 v[2];
        __device__ __forceinline__ Probs() {}
        __device__ __forceinline__ Probs(const f16& p) {
#pragma unroll
            for (int q = 0; q < 4; ++q) set(q, f4{p[4 * q], p[4 * q + 1], p[4 * q + 2], p[4 * q + 3]});
        }
        __device__ __forceinline__ void set(int q, f4 p) {
            const bf4 b = __builtin_convertvector(p, bf4);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[q / 2][q % 2 * 4 + j] = b[j];
        }
    };
};
template <>
struct Mat<float> {
    typedef f4 Frag;
    static constexpr int CH = 4;
    template <int N>
    static __device__ __forceinline__ void sign(Frag (&f)[N], float by) {
        flip<N>(f, __float_as_uint(by) & 0x80000000u);
    }
    static __device__ __forceinline__ f16 scores(Frag a, Frag b, f16 c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
    struct Probs {
        f16 v;
        __device__ __forceinline__ Probs() {}
        __device__ __forceinline__ Probs(const f16& p) : v(p) {}
        __device__ __forceinline__ void set(int q, f4 p) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * q + j] = p[j];
        }
    };
};

template <typename T, int DP>
struct TileOf {
    static constexpr int CH = Mat<T>::CH, NC = DP / CH, SEGS = NC / 4, NS = NC / 2;
    static constexpr int kStep16 = SEGS * 1024;  // bytes of 16 rows
    static_assert(NC % 4 == 0, "whole segments");
    typedef typename Mat<T>::Frag Frag;
    struct Lane {
        uint32_t even, odd;  // row reads: chunks 2s + h of row lane % 32, s even and odd
        uint32_t t0, t1;     // transposed reads: the first and the second eight rows of 16
    };
    static __device__ __forceinline__ Lane lane_of(int lane) {
        const int h = lane / 32, i = lane % 16;
        Lane o;
        const uint32_t r = (uint32_t)((lane % 32) / 16) * kStep16;
        o.even = r + i * 64 + ((h ^ (i / 4)) * 16);
        o.odd = r + i * 64 + (((2 + h) ^ (i / 4)) * 16);
        if (std::is_same<T, __bf16>::value) {
            const int cm = 2 * ((lane / 16) % 2) + (i % 4) / 2, row = 4 * h + i / 4;
            o.t0 = row * 64 + ((cm ^ h) * 16) + (i % 2) * 8;
            o.t1 = (row + 8) * 64 + ((cm ^ (2 + h)) * 16) + (i % 2) * 8;
        } else {
            const int cm = (lane / 4) % 4;
            const uint32_t base = ((lane % 32) / 16) * 1024 + (lane % 4) * 4;
            o.t0 = base + 4 * h * 64 + ((cm ^ h) * 16);
            o.t1 = base + (8 + 4 * h) * 64 + ((cm ^ (2 + h)) * 16);
        }
        return o;
    }
    // Rows 32 k .. 32 k + 31 of the tile, fragment s of each lane's row.
    static __device__ __forceinline__ Frag row(const lds_t* tile, const Lane& l, int k, int s) {
        typedef __attribute__((address_space(3))) const Frag F;
        return *(F*)(tile + (s % 2 ? l.odd : l.even) + (s / 2) * 1024 + k * 2 * kStep16);
    }
    // Fragments wholly beyond D are left out in fp32, where one costs four products.
    static __device__ __forceinline__ bool used(int s, int D) {
        return std::is_same<T, __bf16>::value || 2 * CH * s < DP - 32 || 2 * CH * s < D;
    }
    static __device__ __forceinline__ f16 scores(const lds_t* tile, const Lane& l, int k, const Frag (&f)[NS], int D, f16 c) {
#pragma unroll
        for (int s = 0; s < NS; ++s)
            if (used(s, D)) c = Mat<T>::scores(row(tile, l, k, s), f[s], c);
        return c;
    }
    // Fragments that each lane keeps in LDS for itself (NS KB a wave) where they
    // would not fit the registers.
    static __device__ __forceinline__ void keep(lds_t* at, int lane, const Frag (&f)[NS]) {
        typedef __attribute__((address_space(3))) Frag F;
#pragma unroll
        for (int s = 0; s < NS; ++s) *(F*)(at + s * 1024 + lane * 16) = f[s];
    }
    // The product of a tile's rows with the fragments on top of `start`.  bf16
    // starts the accumulators from it, at no cost.  fp32 adds it last: a bias of -10
    // is -98 in units of a scale of 0.1, and every product added onto that would
    // round to its last place (heads of 96: an error of 1.9e-6 in out, 8e-7 so).
    static __device__ __forceinline__ f16 scores_from(f16 start, const lds_t* tile, const Lane& l, int k, const Frag (&f)[NS],
                                                      int D) {
        if constexpr (std::is_same<T, __bf16>::value) return scores(tile, l, k, f, D, start);
        else return scores(tile, l, k, f, D) + start;
    }
    // The same with the fragments that keep() left at `at`.
    static __device__ __forceinline__ f16 scores_kept(f16 start, const lds_t* tile, const Lane& l, int k, const lds_t* at,
                                                      int lane, int D) {
        typedef __attribute__((address_space(3))) const Frag F;
        constexpr bool last = !std::is_same<T, __bf16>::value;
        f16 c = {0.0f};
        if constexpr (!last) c = start;
#pragma unroll
        for (int s = 0; s < NS; ++s)
            if (used(s, D)) c = Mat<T>::scores(row(tile, l, k, s), *(F*)(at + s * 1024 + lane * 16), c);
        if constexpr (last) c += start;
        return c;
    }
    static __device__ __forceinline__ f16 scores(const lds_t* tile, const Lane& l, int k, const Frag (&f)[NS], int D) {
        const f16 zero = {0.0f};
        return scores(tile, l, k, f, D, zero);
    }
    // fp32 heads whose last 32 entries are eight or fewer in use: 16 products of
    // 64 clocks for those would take more time than their multiply-adds on the
    // vector unit (heads of 36, the step of 3 x 4050 queries to 1013 states: 511 us, 482 so).  The
    // first registers of the last accumulator then hold the lane's own sums over
    // the rows that stand in its registers, which settle() joins and puts in place.
    static __device__ __forceinline__ bool tail(int D) { return std::is_same<T, float>::value && D <= DP - 24; }
    static __device__ __forceinline__ void settle(f16 (&o)[DP / 32], int D, int lane) {
        if (!tail(D)) return;
        f16& e = o[DP / 32 - 1];
#pragma unroll
        for (int r = 0; r < 8; ++r) e[r] += other_half(e[r]);
#pragma unroll
        for (int r = 0; r < 4; ++r) e[r] = lane < 32 ? e[r] : e[4 + r];
#pragma unroll
        for (int r = 4; r < 16; ++r) e[r] = 0.0f;
    }
    // o[D / 32] += (rows 32 k .. 32 k + 31 of the tile)^T x p
    static __device__ __forceinline__ void values(const lds_t* tile, const Lane& l, int k, const typename Mat<T>::Probs& p,
                                                  int D, int lane, f16 (&o)[DP / 32]) {
        if constexpr (std::is_same<T, __bf16>::value) {
            typedef __attribute__((address_space(3))) s4 V;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) {
                    const uint32_t at = d * 1024 + (2 * k + ks) * kStep16;
                    const s4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((V*)(tile + l.t0 + at));
                    const s4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((V*)(tile + l.t1 + at));
                    const bf8 a = __builtin_bit_cast(bf8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p.v[ks], o[d], 0, 0, 0);
                }
            }
        } else {
            typedef __attribute__((address_space(3))) const float V;
            // The 32 rows' own sum first, then onto o: a chain of roundings as
            // long as the tiles, not as the rows.
            const bool few = tail(D);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) {
                if (d == DP / 32 - 1 && few) {
                    const int h = lane / 32;
                    f4 t0 = {0.0f}, t1 = {0.0f};
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        // chunks 8 d and 8 d + 1 of row 8 (i / 4) + 4 h + i % 4
                        typedef __attribute__((address_space(3))) const f4 C;
                        const int r = 8 * ((i / 4) % 2) + 4 * h + i % 4, f = r / 4;
                        const lds_t* at = tile + 2 * d * 1024 + (2 * k + i / 8) * kStep16 + r * 64;
                        const f4 a = *(C*)(at + f * 16), b = *(C*)(at + (1 ^ f) * 16);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            t0[j] = fmaf(p.v[i], a[j], t0[j]);
                            t1[j] = fmaf(p.v[i], b[j], t1[j]);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[d][j] += t0[j], o[d][4 + j] += t1[j];
                    continue;
                }
                f16 t;
#pragma unroll
                for (int i = 0; i < 16; ++i) t[i] = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t at = 2 * d * 1024 + (2 * k + i / 8) * kStep16 + (i % 4) * 64;
                    const float v = *(V*)(tile + ((i / 4) % 2 ? l.t1 : l.t0) + at);
                    t = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p.v[i], t, 0, 0, 0);
                }
                o[d] += t;
            }
        }
    }
};

// 16 bytes of a row from entry c on, zeros beyond D.  W = 2: in one load, 1: in
// two, 0: entry by entry.
template <typename T, int W>
__device__ __forceinline__ u4 load_chunk(const T* row, int c, int D) {
    constexpr int CH = Mat<T>::CH;
    if (c >= D) return u4{0u, 0u, 0u, 0u};
    if constexpr (W == 2) return *(const u4*)(row + c);
    if constexpr (W == 1) {
        const u2 z = {0u, 0u}, lo = *(const u2*)(row + c), hi = c + CH / 2 < D ? *(const u2*)(row + c + CH / 2) : z;
        return u4{lo[0], lo[1], hi[0], hi[1]};
    }
    typename Mat<T>::Frag f;
#pragma unroll
    for (int j = 0; j < CH; ++j) f[j] = c + j < D ? row[c + j] : (T)0.0f;
    return __builtin_bit_cast(u4, f);
}

// Where the next tile of a matrix begins: rows of D entries, `stride` entries apart.
template <typename T>
struct Cursor {
    const T* p;
    int64_t stride;
    int left;  // rows from p on
    int D;
    __device__ __forceinline__ void advance(int rows) {
        p += rows * stride;
        left -= rows;
    }
};

// A tile of ROWS rows on its way from memory to LDS.  Each thread holds chunks
// of one row: a row's 64 bytes by four lanes, a segment by a wave.
template <typename T, int DP, int ROWS>
struct Stage {
    typedef TileOf<T, DP> Tile;
    static constexpr int kHalves = ROWS == 64 ? 1 : 2;  // waves to a row
    static constexpr int N = (Tile::SEGS + kHalves - 1) / kHalves;
    static constexpr int kBytes = ROWS / 16 * Tile::SEGS * 1024;
    static_assert(ROWS * kHalves == 64, "a thread for each quarter of a row's segments");
    u4 v[N];
    static __device__ __forceinline__ int row_of(int wave, int lane) { return wave / kHalves * 16 + lane / 4; }
    // Segment u of this thread's row.
    static __device__ __forceinline__ int seg(int wave, int u) { return kHalves * u + wave % kHalves; }
    static __device__ __forceinline__ bool has(int wave, int u) {
        return Tile::SEGS % kHalves == 0 || seg(wave, u) < Tile::SEGS;
    }
    // W = 2, 1: 16- or 8-byte loads through a buffer over the tile's rows, to
    // which the entries beyond D and the rows beyond the last are out of range
    // and come as zeros.  0: entry by entry, the rows beyond the last coming as
    // the last.
    template <int W>
    __device__ __forceinline__ void load(const Cursor<T>& m, int wave, int lane) {
        const int c = (seg(wave, 0) * 4 + lane % 4) * Mat<T>::CH;
        constexpr int step = kHalves * 4 * Mat<T>::CH;
        if constexpr (W > 0) {
            const int bytes = ((min(m.left, ROWS) - 1) * (int)m.stride + m.D) * (int)sizeof(T);
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(m.p), (short)0, bytes, 0x00020000);
            const int off = (row_of(wave, lane) * (int)m.stride + c) * (int)sizeof(T);
#pragma unroll
            for (int u = 0; u < N; ++u) {
                constexpr int half = Mat<T>::CH / 2, beyond = (int)0x80000000;
                const int at = off + u * step * (int)sizeof(T);
                const bool in = has(wave, u) && c + u * step < m.D;
                if constexpr (W == 2) {
                    v[u] = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(r, in ? at : beyond, 0, 0));
                } else {
                    const bool in1 = has(wave, u) && c + u * step + half < m.D;
                    const auto lo = __builtin_amdgcn_raw_buffer_load_b64(r, in ? at : beyond, 0, 0);
                    const auto hi = __builtin_amdgcn_raw_buffer_load_b64(r, in1 ? at + 8 : beyond, 0, 0);
                    v[u] = u4{lo[0], lo[1], hi[0], hi[1]};
                }
            }
        } else {
            const int r = min(row_of(wave, lane), m.left - 1);
#pragma unroll
            for (int u = 0; u < N; ++u)
                if (has(wave, u)) v[u] = load_chunk<T, 0>(m.p + r * m.stride, c + u * step, m.D);
        }
    }
    // keep: whether this thread's row counts; zeros otherwise, so that whatever
    // memory holds there meets no product.
    __device__ __forceinline__ void store(lds_t* tile, int wave, int lane, bool keep) {
        typedef __attribute__((address_space(3))) u4 V;
        if (!__all(keep)) {
#pragma unroll
            for (int u = 0; u < N; ++u) v[u] = keep ? v[u] : u4{0u, 0u, 0u, 0u};
        }
        lds_t* to = tile + wave / kHalves * Tile::kStep16 + wave % kHalves * 1024 + (lane / 4) * 64 +
                    (((lane % 4) ^ (lane / 16)) * 16);
#pragma unroll
        for (int u = 0; u < N; ++u)
            if (has(wave, u)) *(V*)(to + u * kHalves * 1024) = v[u];
    }
};

// A lane's column vector as fragments: entries 2 CH s + CH h + j.
template <typename T, int DP, int W>
__device__ __forceinline__ void load_frags(const T* row, int D, bool live, int lane,
                                           typename Mat<T>::Frag (&f)[TileOf<T, DP>::NS]) {
    constexpr int CH = Mat<T>::CH;
#pragma unroll
    for (int s = 0; s < TileOf<T, DP>::NS; ++s) {
        const u4 z = {0u, 0u, 0u, 0u};
        f[s] = __builtin_bit_cast(typename Mat<T>::Frag,
                                  live ? load_chunk<T, W>(row, 2 * CH * s + CH * (lane / 32), D) : z);
    }
}

// Exchanges a's upper 32 lanes with b's lower 32.
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}

// A lane's column of accumulators o (entry 32 d + 8 (i / 4) + 4 h + i % 4 in
// register i), times f, to the row's D entries.  W = 2, 1: in 16- or 8-byte stores.
// For the former, bf16 lanes first trade groups of four with the lane that holds the other half of
// their row, so that each has eight in a row (stores of 8 bytes: 66 us for the
// forward pass of 2 x 32768 queries, 8 heads of 64, to 77 keys; so 53 us).  All
// lanes call it; `live`: whether this one's row exists.
template <typename T, int DP, int W>
__device__ __forceinline__ void store_column(T* row, const f16 (&o)[DP / 32], float f, int D, int lane, bool live) {
    if constexpr (W == 2 && std::is_same<T, __bf16>::value) {
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int q = 0; q < 4; q += 2) {
                uint32_t w[2][2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const f4 v = {o[d][4 * (q + k)] * f, o[d][4 * (q + k) + 1] * f, o[d][4 * (q + k) + 2] * f,
                                  o[d][4 * (q + k) + 3] * f};
                    const uint2 u = __builtin_bit_cast(uint2, __builtin_convertvector(v, bf4));
                    w[k][0] = u.x;
                    w[k][1] = u.y;
                }
                swap_halves(w[0][0], w[1][0]);
                swap_halves(w[0][1], w[1][1]);
                const int c = 32 * d + 8 * (q + lane / 32);
                if (live && c < D) *(u4*)(row + c) = u4{w[0][0], w[0][1], w[1][0], w[1][1]};
            }
        return;
    }
    if (!live) return;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = 32 * d + 8 * q + 4 * (lane / 32);
            const f4 v = {o[d][4 * q] * f, o[d][4 * q + 1] * f, o[d][4 * q + 2] * f, o[d][4 * q + 3] * f};
            if constexpr (W == 1 && std::is_same<T, __bf16>::value) {
                if (c < D) *(bf4*)(row + c) = __builtin_convertvector(v, bf4);
            } else if constexpr (W == 2) {
                if (c < D) *(f4*)(row + c) = v;
            } else if constexpr (W == 1) {
                if (c < D) *(f2*)(row + c) = f2{v[0], v[1]};
                if (c + 2 < D) *(f2*)(row + c + 2) = f2{v[2], v[3]};
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c + j < D) row[c + j] = (T)v[j];
            }
        }
}

// Host: whether rows of D entries can be read or written `entries` at a time,
// and the rows of a tile through one buffer.
inline bool wide_rows(const Heads& t, int dim, int entries, size_t elem) {
    if (!t.p) return true;  // not there
    return dim % entries == 0 && (uintptr_t)t.p % (entries * elem) == 0 && t.sb % entries == 0 && t.st % entries == 0 &&
           t.sh % entries == 0 && t.st >= dim && t.st * (int64_t)elem < (int64_t)1 << 24;
}

// How a call's rows go: 2 in 16-byte pieces, 1 in 8-byte pieces, 0 entry by
// entry.  The step of 2 x 8192 queries to 2048 keys, 8 heads, bf16: heads of 40
// (2) 384 us, of 36 (1) 387 us and entry by entry 775 us, of 37 (0) 725 us.
inline int row_width(const AttendArgs& a) {
    const int ch = a.bf16 ? 8 : 4;
    int w = 2;
    for (const Heads* t : {&a.q, &a.k, &a.v, &a.out, &a.low, &a.dout, &a.dq, &a.dk, &a.dv})
        while (w > 0 && !wide_rows(*t, a.dim, w == 2 ? ch : ch / 2, a.bf16 ? 2 : 4)) --w;
    return w;
}
// The width of rows of D partial sums in fp32 for a call of width W.
template <typename T>
constexpr int part_width(int w) { return std::is_same<T, __bf16>::value && w > 0 ? 2 : w; }

}  // namespace disco
