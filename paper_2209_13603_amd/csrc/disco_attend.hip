// disco_attend.hip -- cross attention, forward.
//
// One pass over the keys with the running maximum m and sum l of each row's
// softmax, in units of log 2: t_ij = scale2 (q_i . k_j + bias_j / scale),
// p_ij = 2^(t_ij - m_i), o_i = sum_j p_ij v_j / l_i (m and t rounded alike where they
// are large: near_reference).  The heads that share keys
// and values are rows of one tile (row = query * group + head of the group), so
// that a single query of grouped heads reads them once.
//
// Bound.  Heads of 64, many rows: the matrix products and the softmax's vector
// instructions share the issue of a SIMD and fill it (counters of the 32768 x 8192
// case: products 37 % of the cycles, vector 62 %; moving the row sums onto the
// matrix cores only moved the time, 675 -> 710 us).  Heads of 128: 40 and 40 %, the rest waits
// at the tiles' barriers with two workgroups a CU.  Measured: 32768 queries, 8192
// keys, 8 heads of 64, 682 us (806 TFLOP/s); 2 x 8192 queries, 2048 keys, 16
// heads of 128, 301 us (914 TFLOP/s).  Few rows: reading the keys and values once; 4
// queries of 16 heads on 4 against 131072 keys of 128, 1.07 GB, 194 us a call
// (5.5 TB/s).  fp32 (4050 x 1013, 15 heads of 36): 99 us.
//
// Where the rows leave CUs without two workgroups, the keys go to parts (at
// least four tiles each) whose unnormed sums k_attend_join adds in their order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "disco_attend.h"
#include "disco_internal.h"

namespace disco {

namespace {

// How a call is cut: blocks of kRows rows of each (batch item, kv head), their
// keys in `splits` parts.  Parts leave unnormed sums, joined by k_attend_join.
constexpr int kRows = 32 * kAttendWaves;
struct Cut {
    uint32_t rows, row_blocks, items, run;
    int32_t splits;
    float* part;   // [splits][all rows][dim]
    float* stat;   // [splits][all rows][2]
    int width;     // see row_width
};

// Workgroups of a CU that the registers are sized for.
template <typename T, int DP>
constexpr int kWorkgroups = std::is_same<T, float>::value && DP > 96 ? 1 : 2;
template <typename T>
constexpr int kKeys = std::is_same<T, __bf16>::value ? 64 : 32;  // keys of a tile

// Each wave holds 32 rows; the workgroup's waves share the tiles of keys and
// values, double-buffered in LDS, the next tile's loads in flight in registers.
template <typename T, int DP, int W>
__global__ __launch_bounds__(kAttendThreads, (kWorkgroups<T, DP>)) void k_attend(AttendArgs a, Cut c) {
    typedef TileOf<T, DP> Tile;
    constexpr int KT = kKeys<T>, NK = KT / 32;
    typedef Stage<T, DP, KT> St;
    __shared__ __align__(16) char smem[2 * 2 * St::kBytes];
    __shared__ float starts[2][KT];
    lds_t* lds = (lds_t*)smem;

    const uint32_t id = xcd_item(c.run);
    if (id >= c.items) return;
    const int split = (int)(id % c.splits);
    const uint32_t rb = id / c.splits % c.row_blocks;
    const int bh = (int)(id / c.splits / c.row_blocks), b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, G = a.heads / a.kv_heads;
    const uint32_t row = rb * kRows + wave * 32 + lane % 32;
    const bool live = row < c.rows;
    const int64_t i = live ? row / (uint32_t)G : 0;
    const int h = hk * G + (int)(live ? row % (uint32_t)G : 0);
    const int64_t n = key_count(a, b);
    const int tiles = (int)((n + KT - 1) / KT);
    const int t0 = first_tile(tiles, split, c.splits), t1 = first_tile(tiles, split + 1, c.splits);

    typename Tile::Frag qf[Tile::NS];
    load_frags<T, DP, W>((const T*)a.q.p + b * a.q.sb + i * a.q.st + h * a.q.sh, a.dim, live, lane, qf);
    Mat<T>::template sign<Tile::NS>(qf, a.scale2);
    const float scale2 = fabsf(a.scale2), inv_scale = 1.0f / fabsf(a.scale);
    const typename Tile::Lane ln = Tile::lane_of(lane);

    f16 o[DP / 32];
    clear(o);
    float m = -INFINITY, l = 0.0f;

    St sk, sv;
    float bias = 0.0f;  // of the staged row
    int left = 0;       // rows of the staged tile that exist
    uint64_t any = 0;   // whose staged keys were left, once at least
    const int64_t key0 = (int64_t)t0 * KT;
    Cursor<T> keys{(const T*)a.k.p + b * a.k.sb + hk * a.k.sh + key0 * a.k.st, a.k.st, (int)(n - key0), a.dim};
    Cursor<T> vals{(const T*)a.v.p + b * a.v.sb + hk * a.v.sh + key0 * a.v.st, a.v.st, (int)(n - key0), a.dim};
    const float* biases = a.bias ? a.bias + b * a.bias_sb + key0 : nullptr;
    const int srow = St::row_of(wave, lane);
    auto load = [&] {
        sk.template load<W>(keys, wave, lane);
        sv.template load<W>(vals, wave, lane);
        left = keys.left;
        if (biases) {
            bias = biases[min(srow, left - 1)];
            biases += KT;
        }
        keys.advance(KT);
        vals.advance(KT);
    };
    auto store = [&](int buf) {
        const float start = srow < left ? start_of(bias, inv_scale, a.bias_limit) : -INFINITY;
        const bool keep = start != -INFINITY;
        any |= __ballot(keep);
        sk.store(lds + buf * 2 * St::kBytes, wave, lane, keep);
        sv.store(lds + (buf * 2 + 1) * St::kBytes, wave, lane, keep);
        if (lane % 4 == 0) starts[buf][srow] = start;  // (two waves to a row: the same value)
    };
    if (t0 < t1) {
        load();
        store(0);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1;
        const bool more = t + 1 < t1, plain = !a.bias && left >= KT;
        if (more) load();
        const lds_t* kt = lds + buf * 2 * St::kBytes;
        const lds_t* vt = kt + St::kBytes;
        f16 s[NK];
        if (plain) {
#pragma unroll
            for (int k = 0; k < NK; ++k) s[k] = Tile::scores(kt, ln, k, qf, a.dim);
        } else {
#pragma unroll
            for (int k = 0; k < NK; ++k) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f4 v = *(const f4*)&starts[buf][32 * k + 8 * q + 4 * (lane / 32)];
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[k][4 * q + r] = v[r];
                }
                s[k] = Tile::scores_from(s[k], kt, ln, k, qf, a.dim);
            }
        }
        float top = s[0][0];
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[k][r]);
        top = fmaxf(top, other_half(top)) * scale2;
        // The reference m follows the maximum only where it grew by more than
        // 2^8: p stays below 2^8 and the accumulators are rarely rescaled.
        if (__any(top > m + 8.0f)) {
            const float m1 = fmaxf(m, top), f = __builtin_amdgcn_exp2f(m - (m1 == -INFINITY ? 0.0f : m1));
            m = m1;
            l *= f;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] *= f;
        }
        const float neg = near_reference(s, scale2, m == -INFINITY ? 0.0f : -m);
        float sum = 0.0f;  // of the tile, then onto l: a shorter chain of roundings
#pragma unroll
        for (int k = 0; k < NK; ++k) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[k][r] = __builtin_amdgcn_exp2f(fmaf(s[k][r], scale2, neg));
                sum += s[k][r];
            }
            Tile::values(vt, ln, k, s[k], a.dim, lane, o);
        }
        l += sum;
        if (more) store(buf ^ 1);
        __syncthreads();
    }
    l += other_half(l);
    Tile::settle(o, a.dim, lane);
    // No key left here: zeros, whatever the queries hold (NaN times the zeros that
    // stand for the keys is NaN).
    const bool none = a.bias && !__syncthreads_or(any != 0);
    m = none ? -INFINITY : m;
    l = none ? 0.0f : l;
    clear_if(none, o);
    const int64_t stat = ((int64_t)b * a.heads + h) * a.queries + i;
    if (c.splits > 1) {
        const int64_t all = (int64_t)a.batch * a.kv_heads * c.rows;
        const int64_t at = split * all + (int64_t)bh * c.rows + row;
        store_column<float, DP, part_width<T>(W)>(c.part + at * a.dim, o, 1.0f, a.dim, lane, live);
        if (live && lane < 32) {
            c.stat[2 * at] = m;
            c.stat[2 * at + 1] = l;
        }
        return;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    store_column<T, DP, W>((T*)a.out.p + b * a.out.sb + i * a.out.st + h * a.out.sh, o, inv, a.dim, lane, live);
    if (a.stats && live && lane < 32) {
        a.stats[2 * stat] = m;
        a.stats[2 * stat + 1] = l;
    }
    if constexpr (std::is_same<T, __bf16>::value) {
        if (a.low.p) {  // what rounding took from out
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float v = o[d][r] * inv;
                    o[d][r] = v - (float)(__bf16)v;
                }
            store_column<T, DP, W>((T*)a.low.p + b * a.low.sb + i * a.low.st + h * a.low.sh, o, 1.0f, a.dim, lane, live);
        }
    }
}

// Joins the parts of each row.  A thread holds four entries of a row; where the
// rows are few, `slices` threads share its parts, and their sums are added in
// slice order (see Join).
template <typename T>
__global__ __launch_bounds__(kAttendThreads) void k_attend_join(AttendArgs a, Cut c, Join g) {
    __shared__ f4 part[kAttendThreads];
    __shared__ float sums[kAttendThreads];
    const int lane = g.lane(threadIdx.x), slice = g.slice(threadIdx.x);
    const int64_t all = (int64_t)a.batch * a.kv_heads * c.rows, first = (int64_t)blockIdx.x * g.rows, left = all - first;
    const int64_t at = first + g.row(threadIdx.x);
    const bool live = g.live(threadIdx.x, left), adds = g.adds(threadIdx.x, left);
    const int d = 4 * lane, n = min(4, a.dim - d);
    float m = -INFINITY, l = 0.0f;
    f4 o = {0.0f};
    if (live) {
#pragma unroll 8
        for (int s = 0; s < c.splits; ++s) m = fmaxf(m, c.stat[2 * (s * all + at)]);
        const float ms = m == -INFINITY ? 0.0f : m;
#pragma unroll 4
        for (int s = slice; s < c.splits; s += g.slices) {
            const float f = __builtin_amdgcn_exp2f(c.stat[2 * (s * all + at)] - ms);
            const float* p = c.part + (s * all + at) * a.dim + d;
            f4 v = {0.0f};
            if (a.dim % 4 == 0) v = *(const f4*)p;
            else
                for (int j = 0; j < n; ++j) v[j] = p[j];
            l = fmaf(f, c.stat[2 * (s * all + at) + 1], l);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = fmaf(f, v[j], o[j]);
        }
    }
    if (g.slices > 1) {
        part[threadIdx.x] = o;
        sums[threadIdx.x] = l;
        __syncthreads();
        if (adds)
            for (int s = 1; s < g.slices; ++s) {
                o += part[threadIdx.x + s * g.lanes];
                l += sums[threadIdx.x + s * g.lanes];
            }
    }
    if (!adds) return;
    o *= l == 0.0f ? 0.0f : 1.0f / l;
    const int G = a.heads / a.kv_heads;
    const uint32_t bh = (uint32_t)(at / c.rows), row = (uint32_t)(at - (int64_t)bh * c.rows);
    const int64_t b = bh / (uint32_t)a.kv_heads, i = row / (uint32_t)G;
    const int h = (int)(bh % (uint32_t)a.kv_heads) * G + (int)(row % (uint32_t)G);
    T* out = (T*)a.out.p + b * a.out.sb + i * a.out.st + h * a.out.sh + d;
    T* low = a.low.p ? (T*)a.low.p + b * a.low.sb + i * a.low.st + h * a.low.sh + d : nullptr;
    typedef T T4 __attribute__((ext_vector_type(4)));
    const T4 v = __builtin_convertvector(o, T4);
    if (part_width<T>(c.width) == 2) *(T4*)out = v;
    else
        for (int j = 0; j < n; ++j) out[j] = v[j];
    if (low)
        for (int j = 0; j < n; ++j) low[j] = (T)(o[j] - (float)v[j]);
    if (a.stats && lane == 0) {
        float* st = a.stats + 2 * ((b * a.heads + h) * a.queries + i);
        st[0] = m;
        st[1] = l;
    }
}

Cut cut_of(const AttendArgs& a) {
    Cut c{};
    c.rows = (uint32_t)(a.queries * (a.heads / a.kv_heads));
    c.row_blocks = (c.rows + kRows - 1) / kRows;
    const int64_t blocks = (int64_t)c.row_blocks * a.batch * a.kv_heads;
    const int KT = a.bf16 ? kKeys<__bf16> : kKeys<float>;
    const int64_t tiles = (a.keys + KT - 1) / KT;
    // Two workgroups a CU where there are keys enough for a part of four tiles each.
    const int64_t want = blocks > 0 ? (2 * 256 + blocks - 1) / blocks : 1;
    c.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>({want, tiles / 4, 256}));
    c.items = (uint32_t)(blocks * c.splits);
    c.run = xcd_run(a, c.items);
    return c;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t part_bytes(const AttendArgs& a, const Cut& c) {
    return round256((size_t)c.splits * a.batch * a.kv_heads * c.rows * a.dim * sizeof(float));
}

template <typename T, int DP>
void launch(const AttendArgs& a, const Cut& c) {
    const dim3 grid = xcd_grid(c.items, c.run), block(kAttendThreads);
    if (c.width == 2) hipLaunchKernelGGL((k_attend<T, DP, 2>), grid, block, 0, a.stream, a, c);
    else if (c.width == 1) hipLaunchKernelGGL((k_attend<T, DP, 1>), grid, block, 0, a.stream, a, c);
    else hipLaunchKernelGGL((k_attend<T, DP, 0>), grid, block, 0, a.stream, a, c);
}

template <typename T>
void launch_dim(const AttendArgs& a, const Cut& c) {
    if (a.dim <= 32) launch<T, 32>(a, c);
    else if (a.dim <= 64) launch<T, 64>(a, c);
    else if (a.dim <= 96) launch<T, 96>(a, c);
    else launch<T, 128>(a, c);
}

}  // namespace

size_t attend_ws_bytes(const AttendArgs& a) {
    const Cut c = cut_of(a);
    if (c.splits == 1) return 0;
    return part_bytes(a, c) + (size_t)c.splits * a.batch * a.kv_heads * c.rows * 2 * sizeof(float);
}

hipError_t launch_attend(const AttendArgs& a, void* ws) {
    Cut c = cut_of(a);
    c.width = row_width(a);
    if (c.splits > 1) {
        c.part = (float*)ws;
        c.stat = (float*)((char*)ws + part_bytes(a, c));
    }
    int tk = timing_begin("attend", a.stream);
    if (a.bf16) launch_dim<__bf16>(a, c);
    else launch_dim<float>(a, c);
    timing_end(tk, a.stream);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess || c.splits == 1) return err;
    const int64_t all = (int64_t)a.batch * a.kv_heads * c.rows;
    tk = timing_begin("attend_join", a.stream);
    const Join g = join_of(a.dim, c.splits, all);
    const dim3 grid((unsigned)((all + g.rows - 1) / g.rows));
    if (a.bf16) hipLaunchKernelGGL(k_attend_join<__bf16>, grid, dim3(kAttendThreads), 0, a.stream, a, c, g);
    else hipLaunchKernelGGL(k_attend_join<float>, grid, dim3(kAttendThreads), 0, a.stream, a, c, g);
    timing_end(tk, a.stream);
    return hipGetLastError();
}

}  // namespace disco
