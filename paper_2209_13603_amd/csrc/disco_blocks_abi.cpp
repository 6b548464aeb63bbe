// disco_blocks_abi.cpp -- C entries of the residual sum with its norms, of dropout
// and of the gated recurrence, declared in disco.h: argument validation, workspaces,
// dispatch to the launchers of disco_blocks.h.  Validation is synchronous and
// comes before anything is enqueued.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <string>
#include <utility>

#include "disco_blocks.h"
#include "disco_token_abi.h"

using namespace disco;
using namespace disco::token;

namespace {

bool empty(const disco_rows_t& t) { return t.batch == 0 || t.tokens == 0; }

void check_rows(const disco_rows_t* t, const char* name, int64_t most) {
    const std::string n(name);
    if (!t) refuse(DISCO_ERR_INVALID_ARGUMENT, n + " is NULL");
    if (t->dtype != DISCO_FLOAT32 && t->dtype != DISCO_BFLOAT16) refuse(DISCO_ERR_DTYPE, n + " has an unknown dtype");
    if (t->reserved != 0) refuse(DISCO_ERR_INVALID_ARGUMENT, n + ".reserved is not 0");
    if (t->channels < 1 || t->channels > most)
        refuse(DISCO_ERR_SHAPE, n + " needs 1 to " + std::to_string(most) + " channels");
    if (t->batch < 0 || t->tokens < 0) refuse(DISCO_ERR_SHAPE, n + " has a negative size");
    if (t->stride_batch < 0 || t->stride_token < 0) refuse(DISCO_ERR_INVALID_ARGUMENT, n + " has a negative stride");
    if (t->batch >= kMaxRows || t->tokens >= kMaxRows || t->tokens * t->batch >= kMaxRows)
        refuse(DISCO_ERR_SHAPE, n + " has 2^31 tokens or more");
    if (empty(*t)) return;
    if (t->stride_batch > kMaxOffset / t->batch || t->stride_token > kMaxOffset / t->tokens ||
        (t->batch - 1) * t->stride_batch + (t->tokens - 1) * t->stride_token + t->channels > kMaxOffset)
        refuse(DISCO_ERR_INVALID_ARGUMENT, n + " spans more than 2^46 elements");
    if (!t->data) refuse(DISCO_ERR_INVALID_ARGUMENT, n + ".data is NULL");
    if ((uintptr_t)t->data % bytes_of(t->dtype) != 0)
        refuse(DISCO_ERR_INVALID_ARGUMENT, n + ".data is not aligned to its type");
}

// A tensor of `like`'s sizes and type; an output's rows must not overlap each other.
void check_like(const disco_rows_t* t, const char* name, const disco_rows_t* like, const char* other, bool written) {
    check_rows(t, name, like->channels);
    if (t->dtype != like->dtype) refuse(DISCO_ERR_DTYPE, std::string(name) + " and " + other + " have different dtypes");
    if (t->batch != like->batch || t->tokens != like->tokens || t->channels != like->channels)
        refuse(DISCO_ERR_SHAPE, std::string(name) + " and " + other + " have different sizes");
    if (!written || empty(*t)) return;
    std::pair<int64_t, int64_t> ax[2] = {{t->stride_batch, t->batch}, {t->stride_token, t->tokens}};
    std::sort(ax, ax + 2);
    int64_t span = t->channels;
    for (const auto& a : ax) {
        if (a.second <= 1) continue;
        if (a.first < span) refuse(DISCO_ERR_INVALID_ARGUMENT, std::string(name) + " is written and its rows overlap");
        span += a.first * (a.second - 1);
    }
}

Place place(const char* name, const disco_rows_t* t) {
    if (!t) return Place{name, 0, 0, {0, 0, 0}, {1, 1, 1}};
    const int64_t e = (int64_t)bytes_of(t->dtype);
    return Place{name, (uintptr_t)t->data, t->channels * e, {t->stride_batch * e, t->stride_token * e, 0}, {t->batch, t->tokens, 1}};
}
using disco::token::place;

// Of tensors of one size: whether each entry of one lies where the other's does.
bool same_place(const disco_rows_t& a, const disco_rows_t& b) {
    return a.data == b.data && (a.batch <= 1 || a.stride_batch == b.stride_batch) &&
           (a.tokens <= 1 || a.stride_token == b.stride_token);
}
// An input's place beside an output that may lie exactly on it.
Place beside(const char* name, const disco_rows_t* in, const disco_rows_t* out) {
    return in && out && same_place(*in, *out) ? place(name, (const disco_rows_t*)nullptr) : place(name, in);
}

Rows rows_of(const disco_rows_t* t) { return t ? Rows{t->data, t->stride_batch, t->stride_token} : Rows{}; }
void take(Device* d, const disco_rows_t* t, const char* name) {
    if (t && !empty(*t)) d->take(t->data, name);
}

DropArgs drop_of(const disco_dropout_t& o) {
    if (!(o.p >= 0.0 && o.p <= 1.0)) refuse(DISCO_ERR_INVALID_ARGUMENT, "p must be 0 to 1");
    if ((uintptr_t)o.counter % 8 != 0) refuse(DISCO_ERR_INVALID_ARGUMENT, "counter is not aligned to 8 bytes");
    DropArgs d;
    d.out = (uint32_t)std::nearbyint(o.p * 65536.0);
    d.factor = d.out == 65536 ? 0.0f : (float)(65536.0 / (65536.0 - d.out));
    d.key0 = (uint32_t)o.seed;
    d.key1 = (uint32_t)(o.seed >> 32);
    d.offset = o.offset;
    d.counter = o.counter;
    return d;
}
Place counter_place(const DropArgs& d) { return place("counter", d.counter, sizeof(uint64_t)); }

// ---- residual sum with its norms ----------------------------------------------
void check_weight(const disco_tensor_t* w, const char* name, const disco_rows_t* f, const void** p, int64_t* sb) {
    if (!w) return;
    const std::string n(name);
    if (w->dtype != f->dtype) refuse(DISCO_ERR_DTYPE, n + " and f have different dtypes");
    const bool shared = w->ndim == 1 && w->shape[0] == f->channels;
    if (!shared && !(w->ndim == 2 && w->shape[0] == f->batch && w->shape[1] == f->channels))
        refuse(DISCO_ERR_SHAPE, n + " must be [channels] or [batch, channels]");
    if (!w->data && (shared || f->batch > 0)) refuse(DISCO_ERR_INVALID_ARGUMENT, n + ".data is NULL");
    if ((uintptr_t)w->data % bytes_of(w->dtype) != 0) refuse(DISCO_ERR_INVALID_ARGUMENT, n + ".data is not aligned to its type");
    *p = w->data;
    *sb = shared ? 0 : f->channels;
}

void check_residual(const disco_rows_t* x, const disco_rows_t* f, const disco_residual_t* o, ResidualArgs* a) {
    check_rows(f, "f", kMaxNormChannels);
    if (x) check_like(x, "x", f, "f", false);
    a->x = rows_of(x);
    a->f = rows_of(f);
    a->bf16 = f->dtype == DISCO_BFLOAT16;
    a->batch = (uint32_t)f->batch;
    a->tokens = f->tokens;
    a->channels = (int32_t)f->channels;
    double eps = 1e-6;
    if (o) {
        eps = o->eps;
        if (o->reserved != 0) refuse(DISCO_ERR_INVALID_ARGUMENT, "reserved is not 0");
        if (o->post_norm != 0 && o->post_norm != 1) refuse(DISCO_ERR_INVALID_ARGUMENT, "post_norm must be 0 or 1");
        if (o->post_weight && !o->post_norm) refuse(DISCO_ERR_INVALID_ARGUMENT, "a post_weight needs the post norm");
        if (!(std::fabs(o->scale) <= FLT_MAX)) refuse(DISCO_ERR_INVALID_ARGUMENT, "scale must be finite in fp32");
        if (!(eps >= 0.0 && eps <= FLT_MAX)) refuse(DISCO_ERR_INVALID_ARGUMENT, "eps must be >= 0 and finite in fp32");
        a->post = o->post_norm != 0;
        a->scale = (float)o->scale;
        check_weight(o->post_weight, "post_weight", f, &a->post_w, &a->post_sb);
        check_weight(o->gate, "gate", f, &a->gate, &a->gate_sb);
        check_weight(o->next_weight, "next_weight", f, &a->next_w, &a->next_sb);
        if (o->dropout) {
            a->drop = drop_of(*o->dropout);
            a->dropped = a->drop.out > 0;
        }
    }
    a->eps = (float)eps;
    a->eps_up = eps > 0.0 ? std::max((float)(eps * 0x1p+192), FLT_MIN) : 0.0f;
}

Place weight_place(const ResidualArgs& a, const char* name, const void* p, int64_t sb) {
    return place(name, p, (sb ? (int64_t)a.batch : 1) * a.channels * (int64_t)(a.bf16 ? 2 : 4));
}
void take_weights(Device* d, const ResidualArgs& a) {
    d->take(a.post_w, "post_weight");
    d->take(a.gate, "gate");
    d->take(a.next_w, "next_weight");
    if (a.dropped) d->take(a.drop.counter, "counter");
}

// The gradient of a weight: its shape and type.
void* check_sum(disco_tensor_t* d, const char* name, const disco_tensor_t* w, const char* weight, int64_t batch) {
    if (!d) return nullptr;
    const std::string n(name);
    if (!w) refuse(DISCO_ERR_INVALID_ARGUMENT, n + " needs a " + weight);
    bool same = d->ndim == w->ndim;
    for (int i = 0; same && i < w->ndim; ++i) same = d->shape[i] == w->shape[i];
    if (!same) refuse(DISCO_ERR_SHAPE, n + " and " + weight + " have different shapes");
    if (d->dtype != w->dtype) refuse(DISCO_ERR_DTYPE, n + " and " + weight + " have different dtypes");
    if (w->ndim == 2 && batch == 0) return nullptr;  // no entries
    if (!d->data) refuse(DISCO_ERR_INVALID_ARGUMENT, n + ".data is NULL");
    if ((uintptr_t)d->data % bytes_of(d->dtype) != 0) refuse(DISCO_ERR_INVALID_ARGUMENT, n + ".data is not aligned to its type");
    return d->data;
}

// ---- gated recurrence ------------------------------------------------------------
constexpr int64_t kMaxChannels = (int64_t)1 << 24;

void check_recur(const disco_rows_t* x, const disco_rows_t* g, const disco_rows_t* z, const disco_recurrence_t* o, RecurArgs* a) {
    check_rows(x, "x", kMaxChannels);
    if (g) check_like(g, "gate", x, "x", false);
    if (z) check_like(z, "out_gate", x, "x", false);
    if (x->batch * x->channels >= kMaxRows) refuse(DISCO_ERR_SHAPE, "2^31 states (batch * channels) or more");
    a->x = rows_of(x);
    a->g = rows_of(g);
    a->z = rows_of(z);
    a->bf16 = x->dtype == DISCO_BFLOAT16;
    a->batch = (uint32_t)x->batch;
    a->steps = x->tokens;
    a->channels = x->channels;
    if (!o) return;
    if (o->gain != DISCO_GAIN_MEAN && o->gain != DISCO_GAIN_POWER && o->gain != DISCO_GAIN_ONE)
        refuse(DISCO_ERR_INVALID_ARGUMENT, "unknown gain");
    if (o->reserved != 0) refuse(DISCO_ERR_INVALID_ARGUMENT, "reserved is not 0");
    a->gain = o->gain;
    a->lengths = o->lengths;
}
Place states(const RecurArgs& a, const char* name, const float* p) {
    return place(name, p, (int64_t)a.batch * a.channels * (int64_t)sizeof(float));
}
Place carries_place(const RecurArgs& a) {
    return place("carries", a.carries, (int64_t)a.batch * ((a.steps + kRun - 1) / kRun) * a.channels * (int64_t)sizeof(float));
}
Place lengths_place(const RecurArgs& a) { return place("lengths", a.lengths, (int64_t)a.batch * (int64_t)sizeof(int32_t)); }

}  // namespace

extern "C" {

disco_status_t disco_dropout(const disco_rows_t* x, const disco_dropout_t* dropout, disco_rows_t* y, hipStream_t stream) {
    return guard([&] {
        TraceRange range("disco_dropout");
        check_rows(x, "x", (int64_t)1 << 34);
        check_like(y, "y", x, "x", true);
        if (!dropout) refuse(DISCO_ERR_INVALID_ARGUMENT, "dropout is NULL");
        DropoutArgs a;
        a.drop = drop_of(*dropout);
        if ((x->channels + kChunk - 1) / kChunk * std::max<int64_t>(x->batch * x->tokens, 1) >= kMaxRows)
            refuse(DISCO_ERR_SHAPE, "2^31 chunks of eight entries or more");
        if (empty(*x)) return;
        check_apart({place("y", y)}, {beside("x", x, y), counter_place(a.drop)});
        a.x = rows_of(x);
        a.y = rows_of(y);
        a.batch = (uint32_t)x->batch;
        a.tokens = x->tokens;
        a.channels = x->channels;
        a.bf16 = x->dtype == DISCO_BFLOAT16;
        a.stream = stream;
        Device d;
        take(&d, x, "x");
        take(&d, y, "y");
        d.take(a.drop.counter, "counter");
        d.enter();
        check_hip(launch_dropout(a), "kernel launch");
    });
}

disco_status_t disco_residual_norm(const disco_rows_t* x, const disco_rows_t* f, const disco_residual_t* options,
                                   disco_rows_t* h, disco_rows_t* y, hipStream_t stream) {
    return guard([&] {
        TraceRange range("disco_residual_norm");
        ResidualArgs a;
        check_residual(x, f, options, &a);
        if (!h && !y) refuse(DISCO_ERR_INVALID_ARGUMENT, "neither h nor y is asked for");
        if (h) check_like(h, "h", f, "f", true);
        if (y) check_like(y, "y", f, "f", true);
        if (empty(*f)) return;
        const Place pw = weight_place(a, "post_weight", a.post_w, a.post_sb), gate = weight_place(a, "gate", a.gate, a.gate_sb),
                    nw = weight_place(a, "next_weight", a.next_w, a.next_sb), c = counter_place(a.drop);
        check_apart({place("h", h), place("y", y)}, {pw, gate, nw, c});
        for (const auto& o : {std::pair<const disco_rows_t*, const char*>{h, "h"}, {y, "y"}})
            check_apart({place(o.second, o.first)}, {beside("x", x, o.first), beside("f", f, o.first)});
        a.h = rows_of(h);
        a.y = rows_of(y);
        a.stream = stream;
        Device d;
        take(&d, f, "f");
        take(&d, x, "x");
        take(&d, h, "h");
        take(&d, y, "y");
        take_weights(&d, a);
        d.enter();
        check_hip(launch_residual(a), "kernel launch");
    });
}

disco_status_t disco_residual_norm_workspace(const disco_rows_t* f, const disco_residual_t* options, size_t* bytes) {
    return guard([&] {
        if (!bytes) refuse(DISCO_ERR_INVALID_ARGUMENT, "bytes is NULL");
        *bytes = 0;
        ResidualArgs a;
        check_residual(nullptr, f, options, &a);
        *bytes = residual_grad_ws_bytes(a);
    });
}

disco_status_t disco_residual_norm_backward(const disco_rows_t* x, const disco_rows_t* f, const disco_residual_t* options,
                                            const disco_rows_t* dh, const disco_rows_t* dy, disco_rows_t* dx, disco_rows_t* df,
                                            disco_tensor_t* dpost_weight, disco_tensor_t* dgate, disco_tensor_t* dnext_weight,
                                            void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return guard([&] {
        TraceRange range("disco_residual_norm_backward");
        ResidualArgs a;
        check_residual(x, f, options, &a);
        if (!dh && !dy) refuse(DISCO_ERR_INVALID_ARGUMENT, "neither dh nor dy is given");
        if (dh) check_like(dh, "dh", f, "f", false);
        if (dy) check_like(dy, "dy", f, "f", false);
        if (dx && !x) refuse(DISCO_ERR_INVALID_ARGUMENT, "dx needs x");
        if (dx) check_like(dx, "dx", f, "f", true);
        if (df) check_like(df, "df", f, "f", true);
        const disco_tensor_t *w1 = options ? options->post_weight : nullptr, *g = options ? options->gate : nullptr,
                             *w2 = options ? options->next_weight : nullptr;
        a.dpost = check_sum(dpost_weight, "dpost_weight", w1, "post_weight", f->batch);
        a.dgate = check_sum(dgate, "dgate", g, "gate", f->batch);
        a.dnext = check_sum(dnext_weight, "dnext_weight", w2, "next_weight", f->batch);
        const bool sums = a.dpost || a.dgate || a.dnext;
        if (!sums && (empty(*f) || (!dx && !df))) return;
        const size_t need = sums ? residual_grad_ws_bytes(a) : 0;
        const Place pw = weight_place(a, "post_weight", a.post_w, a.post_sb), gate = weight_place(a, "gate", a.gate, a.gate_sb),
                    nw = weight_place(a, "next_weight", a.next_w, a.next_sb), c = counter_place(a.drop),
                    dpw = weight_place(a, "dpost_weight", a.dpost, a.post_sb), dg = weight_place(a, "dgate", a.dgate, a.gate_sb),
                    dnw = weight_place(a, "dnext_weight", a.dnext, a.next_sb), w = place("the workspace", workspace, (int64_t)need);
        check_apart({place("dx", dx), place("df", df), dpw, dg, dnw, w}, {pw, gate, nw, c});
        check_apart({dpw, dg, dnw, w}, {place("x", x), place("f", f), place("dh", dh), place("dy", dy)});
        for (const auto& o : {std::pair<const disco_rows_t*, const char*>{dx, "dx"}, {df, "df"}})
            check_apart({place(o.second, o.first)}, {beside("x", x, o.first), beside("f", f, o.first), beside("dh", dh, o.first),
                                                     beside("dy", dy, o.first)});
        a.dh = rows_of(dh);
        a.dy = rows_of(dy);
        a.dx = rows_of(dx);
        a.df = rows_of(df);
        a.stream = stream;
        Device d;
        take(&d, f, "f");
        take(&d, x, "x");
        take(&d, dh, "dh");
        take(&d, dy, "dy");
        take(&d, dx, "dx");
        take(&d, df, "df");
        d.take(a.dpost, "dpost_weight");
        d.take(a.dgate, "dgate");
        d.take(a.dnext, "dnext_weight");
        take_weights(&d, a);
        if (need && workspace) d.take(workspace, "workspace");
        d.enter();
        Workspace ws(workspace, workspace_bytes, need, stream);
        check_hip(launch_residual_grad(a, (float*)ws.p), "kernel launch");
    });
}

disco_status_t disco_gated_recurrence_workspace(const disco_rows_t* x, size_t* bytes) {
    return guard([&] {
        if (!bytes) refuse(DISCO_ERR_INVALID_ARGUMENT, "bytes is NULL");
        *bytes = 0;
        RecurArgs a;
        check_recur(x, nullptr, nullptr, nullptr, &a);
        if (a.batch > 0) *bytes = recur_ws_bytes(a);
    });
}

disco_status_t disco_gated_recurrence(const disco_rows_t* x, const disco_rows_t* gate, const disco_rows_t* out_gate,
                                      const disco_recurrence_t* options, const float* state, disco_rows_t* y, float* last,
                                      float* carries, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return guard([&] {
        TraceRange range("disco_gated_recurrence");
        if (!gate) refuse(DISCO_ERR_INVALID_ARGUMENT, "gate is NULL");
        RecurArgs a;
        check_recur(x, gate, out_gate, options, &a);
        check_like(y, "y", x, "x", true);
        if (a.batch == 0 || (a.steps == 0 && !last)) return;
        a.y = rows_of(y);
        a.state = state;
        a.last = last;
        a.carries = carries;
        a.stream = stream;
        const size_t need = recur_ws_bytes(a);
        const Place py = place("y", y), pl = states(a, "last", last), pc = carries_place(a),
                    w = place("the workspace", workspace, (int64_t)need), ps = states(a, "state", state), n = lengths_place(a);
        check_apart({py, pl, pc, w}, {n});
        check_apart({py, pc, w}, {ps});
        if (last != state) check_apart({pl}, {ps});
        check_apart({pl, pc, w}, {place("x", x), place("gate", gate), place("out_gate", out_gate)});
        check_apart({py}, {beside("x", x, y), beside("gate", gate, y), beside("out_gate", out_gate, y)});
        Device d;
        take(&d, x, "x");
        take(&d, gate, "gate");
        take(&d, out_gate, "out_gate");
        take(&d, y, "y");
        d.take(state, "state");
        d.take(last, "last");
        if (a.steps > 0) d.take(carries, "carries");
        d.take(a.lengths, "lengths");  // (read without steps too)
        if (need && workspace) d.take(workspace, "workspace");
        d.enter();
        Workspace ws(workspace, workspace_bytes, need, stream);
        check_hip(launch_recur(a, (float*)ws.p), "kernel launch");
    });
}

disco_status_t disco_gated_recurrence_backward(const disco_rows_t* x, const disco_rows_t* gate, const disco_rows_t* out_gate,
                                               const disco_recurrence_t* options, const float* carries, const disco_rows_t* dy,
                                               const float* dlast, disco_rows_t* dx, disco_rows_t* dgate, disco_rows_t* dout_gate,
                                               float* dstate, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return guard([&] {
        TraceRange range("disco_gated_recurrence_backward");
        if (!gate) refuse(DISCO_ERR_INVALID_ARGUMENT, "gate is NULL");
        RecurArgs a;
        check_recur(x, gate, out_gate, options, &a);
        check_like(dy, "dy", x, "x", false);
        if (dx) check_like(dx, "dx", x, "x", true);
        if (dgate) check_like(dgate, "dgate", x, "x", true);
        if (dout_gate && !out_gate) refuse(DISCO_ERR_INVALID_ARGUMENT, "dout_gate needs out_gate");
        if (dout_gate) check_like(dout_gate, "dout_gate", x, "x", true);
        if (a.batch == 0 || (a.steps == 0 && !dstate) || (!dx && !dgate && !dout_gate && !dstate)) return;
        if (a.steps > 0 && !carries) refuse(DISCO_ERR_INVALID_ARGUMENT, "carries is NULL");
        a.carries = const_cast<float*>(carries);
        a.dy = rows_of(dy);
        a.dx = rows_of(dx);
        a.dg = rows_of(dgate);
        a.dz = rows_of(dout_gate);
        a.dlast = dlast;
        a.dstate = dstate;
        a.stream = stream;
        const size_t need = recur_ws_bytes(a);
        const Place w = place("the workspace", workspace, (int64_t)need), ds = states(a, "dstate", dstate),
                    dl = states(a, "dlast", dlast), n = lengths_place(a), pc = carries_place(a);
        const std::pair<const disco_rows_t*, const char*> outs[] = {{dx, "dx"}, {dgate, "dgate"}, {dout_gate, "dout_gate"}};
        check_apart({place("dx", dx), place("dgate", dgate), place("dout_gate", dout_gate), ds, w}, {n, pc});
        check_apart({place("dx", dx), place("dgate", dgate), place("dout_gate", dout_gate), w}, {dl});
        if (dstate != dlast) check_apart({ds}, {dl});
        check_apart({ds, w}, {place("x", x), place("gate", gate), place("out_gate", out_gate), place("dy", dy)});
        for (const auto& o : outs)
            check_apart({place(o.second, o.first)}, {beside("x", x, o.first), beside("gate", gate, o.first),
                                                     beside("out_gate", out_gate, o.first), beside("dy", dy, o.first)});
        Device d;
        take(&d, x, "x");
        take(&d, gate, "gate");
        take(&d, out_gate, "out_gate");
        take(&d, dy, "dy");
        for (const auto& o : outs) take(&d, o.first, o.second);
        d.take(dlast, "dlast");
        d.take(dstate, "dstate");
        if (a.steps > 0) d.take(carries, "carries");
        d.take(a.lengths, "lengths");  // (read without steps too)
        if (need && workspace) d.take(workspace, "workspace");
        d.enter();
        Workspace ws(workspace, workspace_bytes, need, stream);
        check_hip(launch_recur_grad(a, (float*)ws.p), "kernel launch");
    });
}

}  // extern "C"
