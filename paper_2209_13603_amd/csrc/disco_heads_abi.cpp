// disco_heads_abi.cpp -- C entries of the token operators (head norm and
// rotation, cross attention) and of gradient clipping, declared in disco.h:
// argument validation, workspaces, dispatch to the launchers of disco_heads.h.
// Validation is synchronous and comes before anything is enqueued.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <string>
#include <utility>
#include <vector>

#include "disco_token_abi.h"

using namespace disco;
using namespace disco::token;

namespace {

// ---- head norm and rotation ---------------------------------------------------
void check_rotate(const disco_heads_t* x, int32_t norm, const disco_tensor_t* w, double eps,
                  const disco_rotation_t* r, RotateArgs* a) {
    if (norm != 0 && norm != 1) refuse(DISCO_ERR_INVALID_ARGUMENT, "norm must be 0 or 1");
    if (!norm && w) refuse(DISCO_ERR_INVALID_ARGUMENT, "a weight needs the norm");
    if (norm && !(eps >= 0.0 && eps <= FLT_MAX)) refuse(DISCO_ERR_INVALID_ARGUMENT, "eps must be >= 0 and finite in fp32");
    if (w) {
        if (w->dtype != x->dtype) refuse(DISCO_ERR_DTYPE, "weight and x have different dtypes");
        const bool shared = w->ndim == 1 && w->shape[0] == x->dim;
        if (!shared && !(w->ndim == 2 && w->shape[0] == x->heads && w->shape[1] == x->dim))
            refuse(DISCO_ERR_SHAPE, "weight must be [dim] or [heads, dim]");
        if (!w->data && !(w->ndim == 2 && x->heads == 0)) refuse(DISCO_ERR_INVALID_ARGUMENT, "weight.data is NULL");
        a->weight = w->data;
        a->weight_sh = shared ? 0 : x->dim;
    }
    if (x->batch * x->tokens * x->heads >= kMaxRows)
        refuse(DISCO_ERR_SHAPE, "2^31 rows (batch * tokens * heads) or more");
    a->batch = (int32_t)x->batch;
    a->heads = x->heads;
    a->dim = x->dim;
    a->tokens = x->tokens;
    a->eps = (float)eps;
    a->eps_up = eps > 0.0 ? std::max((float)(eps * 0x1p+192), FLT_MIN) : 0.0f;
    a->norm = norm != 0;
    a->bf16 = x->dtype == DISCO_BFLOAT16;
    if (!r || r->rotary_dim == 0) return;
    if (r->rotary_dim < 0 || r->rotary_dim > x->dim || r->rotary_dim % 2)
        refuse(DISCO_ERR_SHAPE, "rotary_dim must be even and at most dim");
    if (r->layout != DISCO_ROTARY_HALF && r->layout != DISCO_ROTARY_INTERLEAVED)
        refuse(DISCO_ERR_INVALID_ARGUMENT, "unknown rotary layout");
    if (r->rows < 0 || r->first_position < 0 || r->position_stride_batch < 0)
        refuse(DISCO_ERR_INVALID_ARGUMENT, "negative rows, first_position or position stride");
    if (r->rows > 0 && (!r->cosines || !r->sines)) refuse(DISCO_ERR_INVALID_ARGUMENT, "rotation tables are NULL");
    if (!r->positions && !empty(*x) && (r->first_position > r->rows || x->tokens > r->rows - r->first_position))
        refuse(DISCO_ERR_SHAPE, "the rotation tables end before the last token");
    if (r->position_stride_batch > kMaxOffset / std::max<int64_t>(x->batch, 1))
        refuse(DISCO_ERR_INVALID_ARGUMENT, "position stride out of range");
    a->rotary = r->rotary_dim;
    a->interleaved = r->layout == DISCO_ROTARY_INTERLEAVED;
    a->cosines = r->cosines;
    a->sines = r->sines;
    a->rows = r->rows;
    a->positions = r->positions;
    a->pos_sb = r->position_stride_batch;
    a->pos0 = r->first_position;
}

// The small arguments as places.
Place weight_place(const RotateArgs& a, const char* name, const void* p) {
    return place(name, p, (a.weight_sh ? a.heads : 1) * a.dim * (int64_t)(a.bf16 ? 2 : 4));
}
Place table_place(const RotateArgs& a, const char* name, const float* p) { return place(name, p, std::min(a.rows, kMaxOffset) * (a.rotary / 2) * (int64_t)sizeof(float)); }
Place position_place(const RotateArgs& a) {
    return place("positions", a.positions, ((a.batch - 1) * a.pos_sb + a.tokens) * (int64_t)sizeof(int32_t));
}

void take_rotation(Device* d, const RotateArgs& a) {
    d->take(a.weight, "weight");
    if (a.rotary > 0) {
        d->take(a.cosines, "cosines");
        d->take(a.sines, "sines");
        d->take(a.positions, "positions");
    }
}

// ---- cross attention ------------------------------------------------------------
void check_attend(const disco_heads_t* q, const disco_heads_t* k, const disco_heads_t* v,
                  const disco_attention_t* o, AttendArgs* a) {
    check_heads(q, "q");
    check_heads(k, "k");
    if (v) {
        check_heads(v, "v");
        check_same(k, "k", v, "v");
    }
    if (q->dtype != k->dtype) refuse(DISCO_ERR_DTYPE, "q and k have different dtypes");
    if (q->batch != k->batch || q->dim != k->dim) refuse(DISCO_ERR_SHAPE, "q and k differ in batch or dim");
    if (k->heads < 1 || q->heads < 1 || q->heads % k->heads)
        refuse(DISCO_ERR_SHAPE, "the heads of q must be a multiple of those of k and v");
    // (the kernels count the rows of one kv head, tiles and workgroups in 32 bits)
    if (q->batch * q->heads > 65535 * 8 || q->tokens * q->heads >= kMaxRows || k->tokens * k->heads >= kMaxRows * 128 ||
        q->batch * q->tokens * q->heads >= kMaxRows * 16 || k->batch * k->tokens * k->heads >= kMaxRows * 16)
        refuse(DISCO_ERR_SHAPE, "batch * tokens * heads out of range");
    const double scale = o && o->scale != 0.0 ? o->scale : 1.0 / std::sqrt((double)q->dim);
    // (the kernels take it, its product with 1 / log 2 and its reciprocal in fp32)
    if (!(std::fabs(scale) >= FLT_MIN) || !(std::fabs(scale) * 1.4426950408889634074 <= FLT_MAX))
        refuse(DISCO_ERR_INVALID_ARGUMENT, "scale must be a normal number of fp32, at most 2^127");
    a->batch = (int32_t)q->batch;
    a->heads = q->heads;
    a->kv_heads = k->heads;
    a->dim = q->dim;
    a->queries = q->tokens;
    a->keys = k->tokens;
    a->scale = (float)scale;
    a->scale2 = (float)(scale * 1.4426950408889634074);
    // (with a product added and in units of log 2 too such a bias is finite)
    a->bias_limit = (float)std::min(0x1p+126, 0x1p+126 / std::fabs(scale * 1.4426950408889634074));
    a->bf16 = q->dtype == DISCO_BFLOAT16;
    a->q = heads_of(q);
    a->k = heads_of(k);
    if (v) a->v = heads_of(v);
    if (!o) return;
    if (o->bias_stride_batch < 0 || o->bias_stride_batch > kMaxOffset / std::max<int64_t>(q->batch, 1))
        refuse(DISCO_ERR_INVALID_ARGUMENT, "bias stride out of range");
    a->bias = o->key_bias;
    a->bias_sb = o->bias_stride_batch;
    a->lengths = o->key_lengths;
}

Place bias_place(const AttendArgs& a) {
    return place("key_bias", a.bias, a.keys > 0 ? ((a.batch - 1) * a.bias_sb + a.keys) * (int64_t)sizeof(float) : 0);
}
Place lengths_place(const AttendArgs& a) { return place("key_lengths", a.lengths, a.batch * (int64_t)sizeof(int32_t)); }
Place stats_place(const AttendArgs& a) {
    return place("stats", a.stats, (int64_t)a.batch * a.heads * a.queries * 2 * (int64_t)sizeof(float));
}

void take_attend(Device* d, const AttendArgs& a, const disco_heads_t* q, const disco_heads_t* k) {
    if (!empty(*q)) d->take(a.q.p, "q");
    if (!empty(*k)) {
        d->take(a.k.p, "k");
        d->take(a.v.p, "v");
        d->take(a.bias, "key_bias");
    }
    if (q->batch > 0) d->take(a.lengths, "key_lengths");
}

// ---- gradient clipping ------------------------------------------------------------
int64_t check_gradient(const disco_tensor_t& t, const char* list, int32_t i) {
    auto no = [&](disco_status_t status, const char* why) { refuse(status, std::string(list) + "[" + std::to_string(i) + "]" + why); };
    if (t.dtype != DISCO_FLOAT32 && t.dtype != DISCO_BFLOAT16) no(DISCO_ERR_DTYPE, " has an unknown dtype");
    if (t.ndim < 0 || t.ndim > 4) no(DISCO_ERR_SHAPE, " needs 0 to 4 axes");
    int64_t n = 1;
    for (int k = 0; k < t.ndim; ++k) {
        if (t.shape[k] < 0) no(DISCO_ERR_SHAPE, " has a negative size");
        if (t.shape[k] > 0 && n > kMaxOffset / t.shape[k]) no(DISCO_ERR_SHAPE, " is too large");
        n *= t.shape[k];
    }
    if (n > 0 && !t.data) no(DISCO_ERR_INVALID_ARGUMENT, ".data is NULL");
    if ((uintptr_t)t.data % bytes_of(t.dtype) != 0) no(DISCO_ERR_INVALID_ARGUMENT, ".data is not aligned to its type");
    return n;
}

std::vector<ClipTensor> check_gradients(int32_t count, const disco_tensor_t* grads, const disco_tensor_t* clipped) {
    if (count < 0) refuse(DISCO_ERR_INVALID_ARGUMENT, "count is negative");
    if (count > 0 && !grads) refuse(DISCO_ERR_INVALID_ARGUMENT, "grads is NULL");
    std::vector<ClipTensor> v((size_t)count);
    for (int32_t i = 0; i < count; ++i) {
        const disco_tensor_t& g = grads[i];
        v[i] = ClipTensor{g.data, nullptr, check_gradient(g, "grads", i), g.dtype == DISCO_BFLOAT16};
        if (!clipped) continue;
        const disco_tensor_t& c = clipped[i];
        (void)check_gradient(c, "clipped", i);
        if (c.dtype != g.dtype)
            refuse(DISCO_ERR_DTYPE, "clipped[" + std::to_string(i) + "] has another dtype than its gradient");
        bool same = c.ndim == g.ndim;
        for (int a = 0; same && a < g.ndim; ++a) same = c.shape[a] == g.shape[a];
        if (!same) refuse(DISCO_ERR_SHAPE, "clipped[" + std::to_string(i) + "] has another shape than its gradient");
        v[i].out = c.data;
    }
    return v;
}

// Every written range must lie apart from all other ranges (a gradient
// clipped in place is one range).
void check_ranges(const std::vector<ClipTensor>& t) {
    struct Range { uintptr_t lo, hi; int32_t tensor; bool out; };
    std::vector<Range> r;
    r.reserve(2 * t.size());
    bool any = false;
    for (size_t i = 0; i < t.size(); ++i) {
        const uintptr_t n = (uintptr_t)t[i].n * (t[i].bf16 ? 2 : 4);
        if (n == 0) continue;
        const uintptr_t g = (uintptr_t)t[i].g, o = (uintptr_t)t[i].out;
        if (o != g) r.push_back({g, g + n, (int32_t)i, false});
        if (o) r.push_back({o, o + n, (int32_t)i, true});
        any = any || o;
    }
    if (!any) return;
    std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
    uintptr_t hi = 0, hi_out = 0;  // ends of all ranges and of the written ones so far
    for (const Range& x : r) {
        if (x.lo < hi_out || (x.out && x.lo < hi))
            refuse(DISCO_ERR_INVALID_ARGUMENT, "clipped[" + std::to_string(x.tensor) + "] or its gradient overlaps another tensor");
        hi = std::max(hi, x.hi);
        if (x.out) hi_out = std::max(hi_out, x.hi);
    }
}

}  // namespace

extern "C" {

disco_status_t disco_norm_rotate(const disco_heads_t* x, int32_t norm, const disco_tensor_t* weight, double eps,
                                 const disco_rotation_t* rotation, disco_heads_t* y, hipStream_t stream) {
    return guard([&] {
        TraceRange range("disco_norm_rotate");
        check_heads(x, "x");
        check_output(y, "y");
        check_same(x, "x", y, "y");
        RotateArgs a;
        check_rotate(x, norm, weight, eps, rotation, &a);
        if (empty(*x)) return;
        check_apart({place("y", y)}, {place("x", same_place(*x, *y) ? nullptr : x), weight_place(a, "weight", a.weight),
                                      table_place(a, "cosines", a.cosines), table_place(a, "sines", a.sines), position_place(a)});
        a.x = heads_of(x);
        a.y = heads_of(y);
        a.stream = stream;
        Device d;
        d.take(x->data, "x");
        d.take(y->data, "y");
        take_rotation(&d, a);
        d.enter();
        check_hip(launch_rotate(a), "kernel launch");
    });
}

disco_status_t disco_norm_rotate_workspace(const disco_heads_t* x, const disco_tensor_t* weight, size_t* bytes) {
    return guard([&] {
        if (!bytes) refuse(DISCO_ERR_INVALID_ARGUMENT, "bytes is NULL");
        *bytes = 0;
        check_heads(x, "x");
        if (!weight) return;
        RotateArgs a;
        check_rotate(x, 1, weight, 0.0, nullptr, &a);
        *bytes = rotate_grad_ws_bytes(a);
    });
}

disco_status_t disco_norm_rotate_backward(const disco_heads_t* x, int32_t norm, const disco_tensor_t* weight,
                                          double eps, const disco_rotation_t* rotation, const disco_heads_t* dy,
                                          disco_heads_t* dx, disco_tensor_t* dweight, void* workspace,
                                          size_t workspace_bytes, hipStream_t stream) {
    return guard([&] {
        TraceRange range("disco_norm_rotate_backward");
        check_heads(dy, "dy");
        if (x) {
            check_heads(x, "x");
            check_same(x, "x", dy, "dy");
        } else if (norm) {
            refuse(DISCO_ERR_INVALID_ARGUMENT, "x is NULL");
        }
        if (dx) {
            check_output(dx, "dx");
            check_same(dx, "dx", dy, "dy");
        }
        RotateArgs a;
        check_rotate(dy, norm, weight, eps, rotation, &a);
        if (dweight) {
            if (!weight) refuse(DISCO_ERR_INVALID_ARGUMENT, "dweight needs a weight");
            bool same = dweight->ndim == weight->ndim;
            for (int i = 0; same && i < weight->ndim; ++i) same = dweight->shape[i] == weight->shape[i];
            if (!same) refuse(DISCO_ERR_SHAPE, "dweight and weight have different shapes");
            if (dweight->dtype != weight->dtype) refuse(DISCO_ERR_DTYPE, "dweight and weight have different dtypes");
            if (weight->ndim == 2 && dy->heads == 0) dweight = nullptr;  // no entries
        }
        if (dweight) {
            if (!dweight->data) refuse(DISCO_ERR_INVALID_ARGUMENT, "dweight.data is NULL");
            a.dweight = dweight->data;
        }
        if (!a.dweight && (!dx || empty(*dy))) return;
        const size_t need = a.dweight ? rotate_grad_ws_bytes(a) : 0;
        const Place dw = weight_place(a, "dweight", a.dweight), in_x = place("x", x), in_dy = place("dy", dy),
                    wt = weight_place(a, "weight", a.weight), c = table_place(a, "cosines", a.cosines),
                    sn = table_place(a, "sines", a.sines), pos = position_place(a), ws_in = place("the workspace", workspace, (int64_t)need);
        check_apart({dw, ws_in}, {in_x, in_dy, wt, c, sn, pos});
        if (dx) check_apart({place("dx", dx)}, {in_x, same_place(*dx, *dy) ? Place{} : in_dy, wt, c, sn, pos, dw, ws_in});
        a.dy = heads_of(dy);
        if (x) a.x = heads_of(x);
        if (dx) a.dx = heads_of(dx);
        a.stream = stream;
        Device d;
        if (!empty(*dy)) {
            d.take(dy->data, "dy");
            if (norm) d.take(x->data, "x");
            if (dx) d.take(dx->data, "dx");
        }
        d.take(a.dweight, "dweight");
        take_rotation(&d, a);
        if (need && workspace) d.take(workspace, "workspace");
        d.enter();
        Workspace ws(workspace, workspace_bytes, need, stream);
        check_hip(launch_rotate_grad(a, (float*)ws.p), "kernel launch");
    });
}

disco_status_t disco_cross_attention_workspace(const disco_heads_t* q, const disco_heads_t* k, int32_t backward,
                                               size_t* bytes) {
    return guard([&] {
        if (!bytes) refuse(DISCO_ERR_INVALID_ARGUMENT, "bytes is NULL");
        *bytes = 0;
        AttendArgs a;
        check_attend(q, k, nullptr, nullptr, &a);
        *bytes = backward ? attend_grad_ws_bytes(a) : attend_ws_bytes(a);
    });
}

disco_status_t disco_cross_attention(const disco_heads_t* q, const disco_heads_t* k, const disco_heads_t* v,
                                     const disco_attention_t* options, disco_heads_t* out, float* stats,
                                     disco_heads_t* low, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return guard([&] {
        TraceRange range("disco_cross_attention");
        if (!v) refuse(DISCO_ERR_INVALID_ARGUMENT, "v is NULL");
        AttendArgs a;
        check_attend(q, k, v, options, &a);
        check_output(out, "out");
        check_same(q, "q", out, "out");
        if (low) {
            if (!a.bf16) refuse(DISCO_ERR_DTYPE, "low is for bf16");
            check_output(low, "low");
            check_same(q, "q", low, "low");
            a.low = heads_of(low);
        }
        if (empty(*q)) return;
        a.out = heads_of(out);
        a.stats = stats;
        a.stream = stream;
        const size_t need = attend_ws_bytes(a);
        check_apart({place("out", out), place("low", low), stats_place(a), place("the workspace", workspace, (int64_t)need)},
                    {place("q", q), place("k", k), place("v", v), bias_place(a), lengths_place(a)});
        Device d;
        take_attend(&d, a, q, k);
        d.take(out->data, "out");
        d.take(a.low.p, "low");
        d.take(stats, "stats");
        if (need && workspace) d.take(workspace, "workspace");
        d.enter();
        Workspace ws(workspace, workspace_bytes, need, stream);
        check_hip(launch_attend(a, ws.p), "kernel launch");
    });
}

disco_status_t disco_cross_attention_backward(const disco_heads_t* q, const disco_heads_t* k,
                                              const disco_heads_t* v, const disco_attention_t* options,
                                              const disco_heads_t* out, const float* stats,
                                              const disco_heads_t* low, const disco_heads_t* dout, disco_heads_t* dq, disco_heads_t* dk,
                                              disco_heads_t* dv, void* workspace, size_t workspace_bytes,
                                              hipStream_t stream) {
    return guard([&] {
        TraceRange range("disco_cross_attention_backward");
        if (!v) refuse(DISCO_ERR_INVALID_ARGUMENT, "v is NULL");
        AttendArgs a;
        check_attend(q, k, v, options, &a);
        check_heads(out, "out");
        check_heads(dout, "dout");
        check_same(q, "q", out, "out");
        check_same(q, "q", dout, "dout");
        if (low) {
            if (!a.bf16) refuse(DISCO_ERR_DTYPE, "low is for bf16");
            check_heads(low, "low");
            check_same(q, "q", low, "low");
            a.low = heads_of(low);
        }
        const std::pair<disco_heads_t*, const char*> outs[] = {{dq, "dq"}, {dk, "dk"}, {dv, "dv"}};
        for (int i = 0; i < 3; ++i) {
            check_output(outs[i].first, outs[i].second);
            check_same(outs[i].first, outs[i].second, i == 0 ? q : k, i == 0 ? "q" : "k");
        }
        if (empty(*q) && empty(*k)) return;
        if (!empty(*q) && !stats) refuse(DISCO_ERR_INVALID_ARGUMENT, "stats is NULL");
        a.out = heads_of(out);
        a.dout = heads_of(dout);
        a.dq = heads_of(dq);
        a.dk = heads_of(dk);
        a.dv = heads_of(dv);
        a.stats = const_cast<float*>(stats);
        a.stream = stream;
        const size_t need = attend_grad_ws_bytes(a);
        check_apart({place("dq", dq), place("dk", dk), place("dv", dv), place("the workspace", workspace, (int64_t)need)},
                    {place("q", q), place("k", k), place("v", v), place("out", out), place("low", low), place("dout", dout),
                     stats_place(a), bias_place(a), lengths_place(a)});
        Device d;
        take_attend(&d, a, q, k);
        if (!empty(*q)) {
            d.take(out->data, "out");
            d.take(a.low.p, "low");
            d.take(dout->data, "dout");
            d.take(dq->data, "dq");
            d.take(stats, "stats");
        }
        if (!empty(*k)) {
            d.take(dk->data, "dk");
            d.take(dv->data, "dv");
        }
        if (need && workspace) d.take(workspace, "workspace");
        d.enter();
        Workspace ws(workspace, workspace_bytes, need, stream);
        check_hip(launch_attend_grad(a, ws.p), "kernel launch");
    });
}

disco_status_t disco_gradient_clip_workspace(int32_t count, const disco_tensor_t* grads, size_t* bytes) {
    return guard([&] {
        if (!bytes) refuse(DISCO_ERR_INVALID_ARGUMENT, "bytes is NULL");
        *bytes = 0;
        const auto t = check_gradients(count, grads, nullptr);
        *bytes = clip_ws_bytes(t.data(), (int)t.size());
    });
}

disco_status_t disco_gradient_clip(int32_t count, const disco_tensor_t* grads, disco_tensor_t* clipped,
                                   double max_norm, double eps, float* norm, void* workspace,
                                   size_t workspace_bytes, hipStream_t stream) {
    return guard([&] {
        TraceRange range("disco_gradient_clip");
        const auto t = check_gradients(count, grads, clipped);
        if (!norm) refuse(DISCO_ERR_INVALID_ARGUMENT, "norm is NULL");
        if (clipped && !(max_norm >= 0.0)) refuse(DISCO_ERR_INVALID_ARGUMENT, "max_norm must be >= 0");
        if (!(eps >= 0.0) || !std::isfinite(eps)) refuse(DISCO_ERR_INVALID_ARGUMENT, "eps must be >= 0 and finite");
        check_ranges(t);
        const size_t need = clip_ws_bytes(t.data(), (int)t.size());
        const Place n0 = place("norm", norm, sizeof(float)), w0 = place("the workspace", workspace, (int64_t)need);
        check_apart({n0, w0}, {});
        for (const ClipTensor& x : t) {
            const int64_t len = x.n * (x.bf16 ? 2 : 4);
            check_apart({n0, w0}, {place("a gradient", x.g, len), place("a clipped gradient", x.out, len)});
        }
        Device d;
        d.take(norm, "norm");
        for (const ClipTensor& x : t) {
            if (x.n == 0) continue;
            d.take(x.g, "a gradient");
            if (x.out && x.out != x.g) d.take(x.out, "a clipped gradient");
        }
        if (need && workspace) d.take(workspace, "workspace");
        d.enter();
        Workspace ws(workspace, workspace_bytes, need, stream);
        check_hip(launch_clip(t.data(), (int)t.size(), max_norm, eps, norm, ws.p, stream), "kernel launch");
    });
}

}  // extern "C"
