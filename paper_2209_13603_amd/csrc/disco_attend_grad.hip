// disco_attend_grad.hip -- gradients of cross attention.
//
//   delta_i = dout_i . out_i,   ds_ij = p_ij (dout_i . v_j - delta_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij dout_i
// with p rebuilt from the row reference and sum that the forward call left.
//
// Two kernels, one with the rows and one with the keys in its columns, each of
// which keeps its own sums in registers: seven products instead of the five
// of a single pass, but no atomics, so that every run gives the same bits.  The
// first also leaves delta and the row's constants for the second.  delta comes
// from out and from what rounding took from it (`low`): with the rounded out alone
// dq and dk had errors of up to 2.4e-3, before any other rounding, where their
// own is 1.7e-3.
//
// Bound.  2 x 8192 queries, 2048 keys, 16 heads on 4, of 128, bf16: dq 416 us (three
// products, 991 TFLOP/s; products 45 % and vector instructions 40 % of the
// cycles, which they share), dk and dv 558 us (four, 985 TFLOP/s; 42 and 29 %: the sums of
// dk and dv take half the registers, so the key fragments stay in LDS, 950 us in one
// workgroup a CU, 545 in two, and a tile's parts run one after the other between
// fences).  2 x 32768 queries, 77 keys, 8 heads of 64: 93 and 50 us, the rows' memory
// (0.34 GB for dq) in short workgroups.  fp32 (4050 x 1013, 15 heads of 36): 132
// and 178 us, products 39 and 33 %: workgroups of unequal lengths.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "disco_attend.h"
#include "disco_internal.h"

namespace disco {

namespace {

constexpr int kCols = 32 * kAttendWaves;  // rows (dq) or keys (dk, dv) of a workgroup
constexpr int kKeys = 32, kQueries = 32;  // keys, queries of a tile

struct GradCut {
    uint32_t rows, row_blocks, key_blocks, items_q, items_k, run_q, run_k;
    int32_t splits_q, splits_k;
    f4* row_c;    // [batch][heads][queries]: -reference, 1 / sum, delta, written with dq for dk and dv
    float* part;  // [splits][...][dim]
    int width;    // see row_width
};

// Workgroups of a CU that the registers are sized for.
template <typename T, int DP>
constexpr int kWorkgroups = std::is_same<T, float>::value && DP > 64 ? 1 : 2;
// The key fragments of the dk, dv kernel stay in LDS where the registers
// (fragments of k and v, sums of dk and dv) would not hold them.
template <typename T, int DP>
constexpr bool kKeysInLds = DP > (std::is_same<T, float>::value ? 32 : 96);

// dq: each wave holds 32 rows; keys and values come in tiles as in the forward pass.
template <typename T, int DP, int W>
__global__ __launch_bounds__(kAttendThreads, (kWorkgroups<T, DP>)) void k_attend_dq(AttendArgs a, GradCut c) {
    typedef TileOf<T, DP> Tile;
    constexpr int KT = kKeys;
    typedef Stage<T, DP, KT> St;
    __shared__ __align__(16) char smem[2 * 2 * St::kBytes];
    __shared__ float starts[2][KT];
    lds_t* lds = (lds_t*)smem;

    const uint32_t id = xcd_item(c.run_q);
    if (id >= c.items_q) return;
    const int split = (int)(id % c.splits_q);
    const uint32_t rb = id / c.splits_q % c.row_blocks;
    const int bh = (int)(id / c.splits_q / c.row_blocks), b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, G = a.heads / a.kv_heads;
    const uint32_t row = rb * kCols + wave * 32 + lane % 32;
    const bool live = row < c.rows;
    const int64_t i = live ? row / (uint32_t)G : 0;
    const int h = hk * G + (int)(live ? row % (uint32_t)G : 0);
    const int64_t n = key_count(a, b);
    const int tiles = (int)((n + KT - 1) / KT);
    const int t0 = first_tile(tiles, split, c.splits_q), t1 = first_tile(tiles, split + 1, c.splits_q);

    typename Tile::Frag qf[Tile::NS], gf[Tile::NS];
    load_frags<T, DP, W>((const T*)a.dout.p + b * a.dout.sb + i * a.dout.st + h * a.dout.sh, a.dim, live, lane, gf);
    // delta from this lane's half of the entries and the other's
    float delta = 0.0f;
    auto add = [&](const Heads& t) {
        load_frags<T, DP, W>((const T*)t.p + b * t.sb + i * t.st + h * t.sh, a.dim, live, lane, qf);
#pragma unroll
        for (int s = 0; s < Tile::NS; ++s)
#pragma unroll
            for (int j = 0; j < Tile::CH; ++j) delta = fmaf((float)gf[s][j], (float)qf[s][j], delta);
    };
    add(a.out);
    if (a.low.p) add(a.low);
    delta += other_half(delta);
    load_frags<T, DP, W>((const T*)a.q.p + b * a.q.sb + i * a.q.st + h * a.q.sh, a.dim, live, lane, qf);
    Mat<T>::template sign<Tile::NS>(qf, a.scale2);
    Mat<T>::template sign<Tile::NS>(gf, 1.0f);
    const int64_t at = ((int64_t)b * a.heads + h) * a.queries + i;
    const float m = a.stats[2 * at], l = a.stats[2 * at + 1];
    const float neg = l == 0.0f ? -INFINITY : -m, inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (split == 0 && live && lane < 32) c.row_c[at] = f4{neg, inv, delta, 0.0f};
    const float scale2 = fabsf(a.scale2), inv_scale = 1.0f / fabsf(a.scale);
    const typename Tile::Lane ln = Tile::lane_of(lane);

    f16 dq[DP / 32];
    clear(dq);

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
        f16 s;
        if (plain) {
            s = Tile::scores(kt, ln, 0, qf, a.dim);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f4 v = *(const f4*)&starts[buf][8 * q + 4 * (lane / 32)];
#pragma unroll
                for (int r = 0; r < 4; ++r) s[4 * q + r] = v[r];
            }
            s = Tile::scores_from(s, kt, ln, 0, qf, a.dim);
        }
        const f16 dp = Tile::scores(vt, ln, 0, gf, a.dim);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(exponent(s[r], scale2, neg)) * (dp[r] - delta);
        Tile::values(kt, ln, 0, s, a.dim, lane, dq);
        if (more) store(buf ^ 1);
        __syncthreads();
    }
    Tile::settle(dq, a.dim, lane);
    clear_if(a.bias && !__syncthreads_or(any != 0), dq);  // as in the forward pass
    const float f = inv * a.scale;
    if (c.splits_q > 1) {
        const int64_t all = (int64_t)a.batch * a.kv_heads * c.rows;
        store_column<float, DP, part_width<T>(W)>(c.part + (split * all + (int64_t)bh * c.rows + row) * a.dim, dq, f, a.dim, lane, live);
    } else {
        store_column<T, DP, W>((T*)a.dq.p + b * a.dq.sb + i * a.dq.st + h * a.dq.sh, dq, f, a.dim, lane, live);
    }
}

// dk, dv: each wave holds 32 keys; queries and output gradients of every head
// of the group come in tiles.
template <typename T, int DP, int W>
__global__ __launch_bounds__(kAttendThreads, (kWorkgroups<T, DP>)) void k_attend_dkv(AttendArgs a, GradCut c) {
    typedef TileOf<T, DP> Tile;
    constexpr int QT = kQueries;
    typedef Stage<T, DP, QT> St;
    __shared__ __align__(16) char smem[2 * 2 * St::kBytes];
    constexpr bool kept = kKeysInLds<T, DP>;
    __shared__ __align__(16) char kmem[kept ? kAttendWaves * Tile::NS * 1024 : 16];
    __shared__ __align__(16) float row_c[2][4][QT];  // GradCut::row_c of the tile's rows
    lds_t* lds = (lds_t*)smem;

    const uint32_t id = xcd_item(c.run_k);
    if (id >= c.items_k) return;
    const int split = (int)(id % c.splits_k);
    const uint32_t kb = id / c.splits_k % c.key_blocks;
    const int bh = (int)(id / c.splits_k / c.key_blocks), b = bh / a.kv_heads, hk = bh % a.kv_heads;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave, G = a.heads / a.kv_heads;
    const int64_t j = (int64_t)kb * kCols + wave * 32 + lane % 32, n = key_count(a, b);
    const float scale2 = fabsf(a.scale2);
    const float start = j >= n ? -INFINITY : a.bias ? start_of(a.bias[b * a.bias_sb + j], 1.0f / fabsf(a.scale), a.bias_limit) : 0.0f;
    const bool live = start != -INFINITY;
    const int64_t jr = live ? j : 0;

    typename Tile::Frag kf[Tile::NS], vf[Tile::NS];
    load_frags<T, DP, W>((const T*)a.k.p + b * a.k.sb + jr * a.k.st + hk * a.k.sh, a.dim, live, lane, kf);
    load_frags<T, DP, W>((const T*)a.v.p + b * a.v.sb + jr * a.v.st + hk * a.v.sh, a.dim, live, lane, vf);
    Mat<T>::template sign<Tile::NS>(kf, a.scale2);
    Mat<T>::template sign<Tile::NS>(vf, 1.0f);
    lds_t* const mine = (lds_t*)kmem + wave * Tile::NS * 1024;
    if constexpr (kept) Tile::keep(mine, lane, kf);
    const typename Tile::Lane ln = Tile::lane_of(lane);
    f16 dk[DP / 32], dv[DP / 32];
    clear(dk);
    clear(dv);

    // The tiles of the group's heads one after the other.
    const int tiles = (int)((a.queries + QT - 1) / QT), steps = (int64_t)kb * kCols < n ? tiles * G : 0;
    const int t0 = first_tile(steps, split, c.splits_k), t1 = first_tile(steps, split + 1, c.splits_k);
    St sq, sg;
    float rc = 0.0f;  // entry threadIdx.x of the staged tile's row constants
    int left = 0;  // rows of the staged tile that exist, QT at most (four entries each are counted in 32 bits)
    const int g0 = tiles > 0 ? t0 / tiles : 0;
    int at = tiles > 0 ? t0 % tiles : 0;  // tile of the next load among its head's
    int64_t head = hk * G + g0;
    Cursor<T> qs{(const T*)a.q.p + b * a.q.sb + head * a.q.sh + (int64_t)at * QT * a.q.st, a.q.st, (int)a.queries - at * QT, a.dim};
    Cursor<T> gs{(const T*)a.dout.p + b * a.dout.sb + head * a.dout.sh + (int64_t)at * QT * a.dout.st, a.dout.st, qs.left, a.dim};
    const f4* consts = c.row_c + ((int64_t)b * a.heads + head) * a.queries + (int64_t)at * QT;
    auto load = [&] {
        sq.template load<W>(qs, wave, lane);
        sg.template load<W>(gs, wave, lane);
        left = min(qs.left, QT);
        rc = ((const float*)consts)[min((int)threadIdx.x, 4 * left - 1)];
        if (++at < tiles) {
            qs.advance(QT);
            gs.advance(QT);
            consts += QT;
        } else {  // the next head of the group
            at = 0;
            ++head;
            qs.p = (const T*)a.q.p + b * a.q.sb + head * a.q.sh;
            gs.p = (const T*)a.dout.p + b * a.dout.sb + head * a.dout.sh;
            qs.left = gs.left = (int)a.queries;
            consts = c.row_c + ((int64_t)b * a.heads + head) * a.queries;
        }
    };
    auto store = [&](int buf) {
        const bool keep = St::row_of(wave, lane) < left;
        sq.store(lds + buf * 2 * St::kBytes, wave, lane, keep);
        sg.store(lds + (buf * 2 + 1) * St::kBytes, wave, lane, keep);
        if (threadIdx.x < 4 * QT) {
            const int k = threadIdx.x % 4;
            row_c[buf][k][threadIdx.x / 4] = (int)threadIdx.x < 4 * left ? rc : k == 0 ? -INFINITY : 0.0f;
        }
    };
    if (t0 < t1) {
        load();
        store(0);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1;
        const bool more = t + 1 < t1;
        if (more) load();
        const lds_t* qt = lds + buf * 2 * St::kBytes;
        const lds_t* gt = qt + St::kBytes;
        f16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = start;
        if constexpr (kept) s = Tile::scores_kept(s, qt, ln, 0, mine, lane, a.dim);
        else s = Tile::scores_from(s, qt, ln, 0, kf, a.dim);
        if constexpr (kept) __builtin_amdgcn_sched_barrier(0);
        const f16 dp = Tile::scores(gt, ln, 0, vf, a.dim);
        if constexpr (kept) __builtin_amdgcn_sched_barrier(0);
        typename Mat<T>::Probs p, ds;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int at4 = 8 * q + 4 * (lane / 32);
            const f4 neg = *(const f4*)&row_c[buf][0][at4], inv = *(const f4*)&row_c[buf][1][at4];
            const f4 delta = *(const f4*)&row_c[buf][2][at4];
            f4 e, f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                e[r] = __builtin_amdgcn_exp2f(exponent(s[4 * q + r], scale2, neg[r])) * inv[r];
                f[r] = e[r] * (dp[4 * q + r] - delta[r]);
            }
            p.set(q, e);
            ds.set(q, f);
        }
        if constexpr (kept) __builtin_amdgcn_sched_barrier(0);
        Tile::values(gt, ln, 0, p, a.dim, lane, dv);
        if constexpr (kept) __builtin_amdgcn_sched_barrier(0);
        Tile::values(qt, ln, 0, ds, a.dim, lane, dk);
        if (more) store(buf ^ 1);
        __syncthreads();
    }
    Tile::settle(dk, a.dim, lane);
    Tile::settle(dv, a.dim, lane);
    clear_if(!live, dk);  // nothing of a key that is taken out
    clear_if(!live, dv);
    const bool there = j < a.keys;
    if (c.splits_k > 1) {
        const int64_t all = (int64_t)a.batch * a.kv_heads * a.keys, at = split * 2 * all + (int64_t)bh * a.keys + j;
        store_column<float, DP, part_width<T>(W)>(c.part + at * a.dim, dk, a.scale, a.dim, lane, there);
        store_column<float, DP, part_width<T>(W)>(c.part + (at + all) * a.dim, dv, 1.0f, a.dim, lane, there);
    } else {
        store_column<T, DP, W>((T*)a.dk.p + b * a.dk.sb + j * a.dk.st + hk * a.dk.sh, dk, a.scale, a.dim, lane, there);
        store_column<T, DP, W>((T*)a.dv.p + b * a.dv.sb + j * a.dv.st + hk * a.dv.sh, dv, 1.0f, a.dim, lane, there);
    }
}

// Adds the parts of each row in their order: entry e of part s of row r of
// matrix blockIdx.y stands at part[(s * matrices + blockIdx.y) * all * dim + r * dim + e].
// Rows are (batch, kv head, row), a row being (token, head of the group).
template <typename T>
__global__ __launch_bounds__(256) void k_attend_sum(const float* __restrict__ part, int splits, int64_t rows,
                                                    int kv_heads, int G, int dim, int64_t all, Heads o0, Heads o1) {
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= all * dim) return;
    const float* p = part + (int64_t)blockIdx.y * all * dim + e;
    const int64_t step = (int64_t)gridDim.y * all * dim;
    float v = 0.0f;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) v += p[s * step];
    const int64_t r = e / dim, bh = r / rows, row = r % rows;
    const Heads& o = blockIdx.y ? o1 : o0;
    T* out = (T*)o.p + bh / kv_heads * o.sb + row / G * o.st + (bh % kv_heads * G + row % G) * o.sh;
    out[e % dim] = (T)v;
}

int32_t parts(int64_t blocks, int64_t steps, int64_t least) {
    const int64_t want = blocks > 0 ? (2 * 256 + blocks - 1) / blocks : 1;
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>({want, steps / least, 256}));
}

GradCut cut_of(const AttendArgs& a) {
    GradCut c{};
    const int G = a.heads / a.kv_heads;
    c.rows = (uint32_t)(a.queries * G);
    c.row_blocks = (c.rows + kCols - 1) / kCols;
    c.key_blocks = (uint32_t)((a.keys + kCols - 1) / kCols);
    const int64_t bq = (int64_t)c.row_blocks * a.batch * a.kv_heads, bk = (int64_t)c.key_blocks * a.batch * a.kv_heads;
    // Parts of at least eight tiles, as many as give every CU two workgroups.
    c.splits_q = parts(bq, (a.keys + kKeys - 1) / kKeys, 8);
    c.splits_k = parts(bk, (a.queries + kQueries - 1) / kQueries * G, 8);
    c.items_q = (uint32_t)(bq * c.splits_q);
    c.items_k = (uint32_t)(bk * c.splits_k);
    c.run_q = xcd_run(a, c.items_q);
    c.run_k = xcd_run(a, c.items_k);
    return c;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t row_bytes(const AttendArgs& a) { return round256((size_t)a.batch * a.heads * a.queries * sizeof(f4)); }

template <typename T, int DP>
void launch_dq(const AttendArgs& a, const GradCut& c) {
    const dim3 grid = xcd_grid(c.items_q, c.run_q), block(kAttendThreads);
    if (c.width == 2) hipLaunchKernelGGL((k_attend_dq<T, DP, 2>), grid, block, 0, a.stream, a, c);
    else if (c.width == 1) hipLaunchKernelGGL((k_attend_dq<T, DP, 1>), grid, block, 0, a.stream, a, c);
    else hipLaunchKernelGGL((k_attend_dq<T, DP, 0>), grid, block, 0, a.stream, a, c);
}
template <typename T, int DP>
void launch_dkv(const AttendArgs& a, const GradCut& c) {
    const dim3 grid = xcd_grid(c.items_k, c.run_k), block(kAttendThreads);
    if (c.width == 2) hipLaunchKernelGGL((k_attend_dkv<T, DP, 2>), grid, block, 0, a.stream, a, c);
    else if (c.width == 1) hipLaunchKernelGGL((k_attend_dkv<T, DP, 1>), grid, block, 0, a.stream, a, c);
    else hipLaunchKernelGGL((k_attend_dkv<T, DP, 0>), grid, block, 0, a.stream, a, c);
}

template <typename T>
hipError_t run(const AttendArgs& a, const GradCut& c) {
    const int G = a.heads / a.kv_heads;
    hipError_t e = hipSuccess;
    auto sum = [&](int splits, int64_t rows, int g, int matrices, const Heads& o0, const Heads& o1) {
        const int64_t all = (int64_t)a.batch * a.kv_heads * rows;
        const int tk = timing_begin("attend_sum", a.stream);
        hipLaunchKernelGGL(k_attend_sum<T>, dim3((unsigned)((all * a.dim + 255) / 256), (unsigned)matrices), dim3(256), 0,
                           a.stream, c.part, splits, rows, a.kv_heads, g, a.dim, all, o0, o1);
        timing_end(tk, a.stream);
        return hipGetLastError();
    };
    if (c.items_q > 0) {
        const int tk = timing_begin("attend_dq", a.stream);
        if (a.dim <= 32) launch_dq<T, 32>(a, c);
        else if (a.dim <= 64) launch_dq<T, 64>(a, c);
        else if (a.dim <= 96) launch_dq<T, 96>(a, c);
        else launch_dq<T, 128>(a, c);
        timing_end(tk, a.stream);
        e = hipGetLastError();
        if (e == hipSuccess && c.splits_q > 1) e = sum(c.splits_q, c.rows, G, 1, a.dq, a.dq);
    }
    if (e == hipSuccess && c.items_k > 0) {
        const int tk = timing_begin("attend_dkv", a.stream);
        if (a.dim <= 32) launch_dkv<T, 32>(a, c);
        else if (a.dim <= 64) launch_dkv<T, 64>(a, c);
        else if (a.dim <= 96) launch_dkv<T, 96>(a, c);
        else launch_dkv<T, 128>(a, c);
        timing_end(tk, a.stream);
        e = hipGetLastError();
        if (e == hipSuccess && c.splits_k > 1) e = sum(c.splits_k, a.keys, 1, 2, a.dk, a.dv);
    }
    return e;
}

}  // namespace

size_t attend_grad_ws_bytes(const AttendArgs& a) {
    const GradCut c = cut_of(a);
    const size_t row = (size_t)a.batch * a.kv_heads * a.dim * sizeof(float);
    const size_t q = c.splits_q > 1 ? c.splits_q * row * c.rows : 0, k = c.splits_k > 1 ? c.splits_k * 2 * row * a.keys : 0;
    return row_bytes(a) + std::max(q, k);
}

hipError_t launch_attend_grad(const AttendArgs& a, void* ws) {
    GradCut c = cut_of(a);
    c.width = row_width(a);
    c.row_c = (f4*)ws;
    c.part = (float*)((char*)ws + row_bytes(a));
    return a.bf16 ? run<__bf16>(a, c) : run<float>(a, c);
}

}  // namespace disco
