// disco_heads_abi.cpp -- C entries of the token operators (head norm and
// rotation, cross attention) and of gradient clipping, declared in disco.h:
// argument validation, workspaces, dispatch to the launchers of disco_heads.h.
// Validation is synchronous and comes before anything is enqueued.
#include <rocprofiler-sdk-roctx/roctx.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "disco.h"
#include "disco_heads.h"
#include "disco_internal.h"

using namespace disco;

namespace {

struct TraceRange {
    explicit TraceRange(const char* name) { roctxRangePushA(name); }
    ~TraceRange() { roctxRangePop(); }
    TraceRange(const TraceRange&) = delete;
    TraceRange& operator=(const TraceRange&) = delete;
};

// A refusal, carried to the entry's guard().
struct Refusal {
    disco_status_t status;
    std::string why;
};

[[noreturn]] void refuse(disco_status_t s, std::string why) { throw Refusal{s, std::move(why)}; }

void check_hip(hipError_t e, const char* what) {
    if (e == hipSuccess) return;
    refuse(e == hipErrorOutOfMemory ? DISCO_ERR_OUT_OF_MEMORY : DISCO_ERR_DEVICE,
           std::string(what) + ": " + hipGetErrorString(e));
}

// Runs an entry's body; no exception leaves a C entry.
template <typename F>
disco_status_t guard(F&& body) {
    try {
        body();
        return set_last_error(DISCO_OK, "");
    } catch (const Refusal& r) {
        return set_last_error(r.status, r.why.c_str());
    } catch (const std::bad_alloc&) {
        return set_last_error(DISCO_ERR_OUT_OF_MEMORY, "out of host memory");
    } catch (const std::exception& e) {
        return set_last_error(DISCO_ERR_DEVICE, e.what());
    }
}

// The device the call runs on: that of the first tensor's memory.
struct Device {
    int id = -1, before = -1;
    void take(const void* p, const char* name) {
        if (!p) return;
        hipPointerAttribute_t attr;
        std::memset(&attr, 0, sizeof(attr));
        if (hipPointerGetAttributes(&attr, p) != hipSuccess) {
            (void)hipGetLastError();
            refuse(DISCO_ERR_DEVICE, std::string(name) + " is not a device pointer known to HIP");
        }
        if (attr.type != hipMemoryTypeDevice && attr.type != hipMemoryTypeManaged)
            refuse(DISCO_ERR_DEVICE, std::string(name) + " is not device memory");
        if (id < 0) id = attr.device;
        if (attr.device != id)
            refuse(DISCO_ERR_DEVICE, std::string(name) + " lives on device " + std::to_string(attr.device) +
                                         ", the other tensors on device " + std::to_string(id));
    }
    void enter() {
        int cur = 0;
        check_hip(hipGetDevice(&cur), "hipGetDevice");
        if (id >= 0 && cur != id) {
            check_hip(hipSetDevice(id), "hipSetDevice");
            before = cur;
        }
    }
    ~Device() {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

// The caller's workspace, or one of the stream-ordered pool.
struct Workspace {
    void* p = nullptr;
    bool own = false;
    hipStream_t stream = nullptr;
    Workspace(void* given, size_t given_bytes, size_t need, hipStream_t s) : stream(s) {
        if (need == 0) return;
        if (given) {
            if (given_bytes < need)
                refuse(DISCO_ERR_INVALID_ARGUMENT, "the workspace holds " + std::to_string(given_bytes) +
                                                       " bytes, this call needs " + std::to_string(need));
            if ((uintptr_t)given % 256 != 0)
                refuse(DISCO_ERR_INVALID_ARGUMENT, "the workspace is not 256-byte aligned");
            p = given;
            return;
        }
        check_hip(hipMallocAsync(&p, need, s), "hipMallocAsync(workspace)");
        own = true;
    }
    ~Workspace() {
        if (own) (void)hipFreeAsync(p, stream);
    }
    Workspace(const Workspace&) = delete;
    Workspace& operator=(const Workspace&) = delete;
};

size_t bytes_of(int32_t dtype) { return dtype == DISCO_BFLOAT16 ? 2 : 4; }

constexpr int64_t kMaxRows = (int64_t)1 << 31;       // tokens of all batch items
constexpr int64_t kMaxOffset = (int64_t)1 << 46;     // element offsets

bool empty(const disco_heads_t& t) { return t.batch == 0 || t.tokens == 0 || t.heads == 0; }

// Elements from the first to one past the last.
int64_t extent(const disco_heads_t& t) {
    return empty(t) ? 0
                    : (t.batch - 1) * t.stride_batch + (t.tokens - 1) * t.stride_token +
                          (t.heads - 1) * t.stride_head + t.dim;
}

void check_heads(const disco_heads_t* t, const char* name) {
    const std::string n(name);
    if (!t) refuse(DISCO_ERR_INVALID_ARGUMENT, n + " is NULL");
    if (t->dtype != DISCO_FLOAT32 && t->dtype != DISCO_BFLOAT16) refuse(DISCO_ERR_DTYPE, n + " has an unknown dtype");
    if (t->reserved != 0) refuse(DISCO_ERR_INVALID_ARGUMENT, n + ".reserved is not 0");
    if (t->dim < 1 || t->dim > kMaxHeadDim)
        refuse(DISCO_ERR_SHAPE, n + " needs heads of 1 to " + std::to_string(kMaxHeadDim) + " entries");
    if (t->batch < 0 || t->tokens < 0 || t->heads < 0 || t->heads > 4096 || t->batch > 65535)
        refuse(DISCO_ERR_SHAPE, n + " has a size out of range");
    if (t->stride_batch < 0 || t->stride_token < 0 || t->stride_head < 0)
        refuse(DISCO_ERR_INVALID_ARGUMENT, n + " has a negative stride");
    if (t->tokens >= kMaxRows || (t->batch > 0 && t->tokens * t->batch >= kMaxRows))
        refuse(DISCO_ERR_SHAPE, n + " has 2^31 tokens or more");
    if (empty(*t)) return;
    if (t->stride_batch > kMaxOffset || t->stride_token > kMaxOffset / t->tokens || t->stride_head > kMaxOffset ||
        extent(*t) > kMaxOffset)
        refuse(DISCO_ERR_INVALID_ARGUMENT, n + " spans more than 2^46 elements");
    if (!t->data) refuse(DISCO_ERR_INVALID_ARGUMENT, n + ".data is NULL");
    if ((uintptr_t)t->data % bytes_of(t->dtype) != 0)
        refuse(DISCO_ERR_INVALID_ARGUMENT, n + ".data is not aligned to its type");
}

// An output's rows must not overlap each other: by growing stride, each
// axis has to step over all that the ones before it span.
void check_output(const disco_heads_t* t, const char* name) {
    check_heads(t, name);
    if (empty(*t)) return;
    std::pair<int64_t, int64_t> ax[3] = {{t->stride_batch, t->batch}, {t->stride_token, t->tokens}, {t->stride_head, t->heads}};
    std::sort(ax, ax + 3);
    int64_t span = t->dim;
    for (const auto& a : ax) {
        if (a.second <= 1) continue;
        if (a.first < span) refuse(DISCO_ERR_INVALID_ARGUMENT, std::string(name) + " is written and its rows overlap");
        span += a.first * (a.second - 1);
    }
}

void check_same(const disco_heads_t* a, const char* na, const disco_heads_t* b, const char* nb) {
    if (a->dtype != b->dtype) refuse(DISCO_ERR_DTYPE, std::string(na) + " and " + nb + " have different dtypes");
    if (a->batch != b->batch || a->tokens != b->tokens || a->heads != b->heads || a->dim != b->dim)
        refuse(DISCO_ERR_SHAPE, std::string(na) + " and " + nb + " have different sizes");
}

// An axis that two tensors step along alike.
struct Axis {
    int64_t stride, na, nb;
};

// Whether some a0 + sum ia stride + ea, ea < dim_a, is some b0 + sum ib stride +
// eb, eb < dim_b, for d = b0 - a0: by falling stride each axis steps over all
// that the ones after it span, so that only two of its differences ia - ib can
// bring d within reach of those.
bool meets(const Axis* ax, int n, int64_t d, int64_t dim_a, int64_t dim_b) {
    if (n == 0) return d > -dim_b && d < dim_a;
    const int64_t s = ax->stride, k = d >= 0 ? d / s : -((-d + s - 1) / s);
    for (int64_t i : {k, k + 1})
        if (i > -ax->nb && i < ax->na && meets(ax + 1, n - 1, d - i * s, dim_a, dim_b)) return true;
    return false;
}

// Whether two tensors may share memory: exactly where they have the same
// strides along nested axes, as the parts of one joint buffer do in any order of
// its axes.  With other strides, tensors whose tokens lie equally far apart
// are told apart by their place within a token, all others by the memory from
// their first to their last entry.
bool may_overlap(const disco_heads_t& a, const disco_heads_t& b) {
    if (empty(a) || empty(b)) return false;
    const int64_t ea = (int64_t)bytes_of(a.dtype), eb = (int64_t)bytes_of(b.dtype);
    const uintptr_t a0 = (uintptr_t)a.data, b0 = (uintptr_t)b.data;
    const uintptr_t a1 = a0 + (uintptr_t)(extent(a) * ea), b1 = b0 + (uintptr_t)(extent(b) * eb);
    if (a1 <= b0 || b1 <= a0) return false;

    Axis ax[3];
    int n = 0;
    bool alike = ea == eb;
    const int64_t at[3][4] = {{a.stride_batch, a.batch, b.stride_batch, b.batch},
                              {a.stride_token, a.tokens, b.stride_token, b.tokens},
                              {a.stride_head, a.heads, b.stride_head, b.heads}};
    for (const auto& x : at) {
        const int64_t na = x[0] == 0 ? 1 : x[1], nb = x[2] == 0 ? 1 : x[3];
        if (na > 1 && nb > 1 && x[0] != x[2]) alike = false;
        if (na > 1 || nb > 1) ax[n++] = Axis{na > 1 ? x[0] : x[2], na, nb};
    }
    std::sort(ax, ax + n, [](const Axis& p, const Axis& q) { return p.stride > q.stride; });
    int64_t span_a = a.dim, span_b = b.dim;
    for (int i = n - 1; i >= 0 && alike; --i) {
        alike = ax[i].stride >= std::max(span_a, span_b);
        span_a += ax[i].stride * (ax[i].na - 1);
        span_b += ax[i].stride * (ax[i].nb - 1);
    }
    if (alike) return meets(ax, n, ((int64_t)b0 - (int64_t)a0) / ea, a.dim, b.dim);

    const int64_t step = a.stride_token * ea;
    if (step > 0 && step == b.stride_token * eb && (a.batch == 1 || a.stride_batch % a.stride_token == 0) &&
        (b.batch == 1 || b.stride_batch % b.stride_token == 0)) {
        const int64_t wa = ((a.heads - 1) * a.stride_head + a.dim) * ea, wb = ((b.heads - 1) * b.stride_head + b.dim) * eb;
        const int64_t d = (int64_t)((a0 >= b0 ? (a0 - b0) % (uintptr_t)step : (step - (b0 - a0) % (uintptr_t)step) % step));
        if (d >= wb && d + wa <= step) return false;
    }
    return true;
}

// Of tensors of one size: whether each entry of one lies where the other's does
// (the stride of a single entry leads nowhere).
bool same_place(const disco_heads_t& a, const disco_heads_t& b) {
    return a.data == b.data && (a.batch <= 1 || a.stride_batch == b.stride_batch) &&
           (a.tokens <= 1 || a.stride_token == b.stride_token) && (a.heads <= 1 || a.stride_head == b.stride_head);
}

void check_apart(const disco_heads_t* out, const char* no, const disco_heads_t* in, const char* ni) {
    if (may_overlap(*out, *in)) refuse(DISCO_ERR_INVALID_ARGUMENT, std::string(no) + " overlaps " + ni);
}

Heads heads_of(const disco_heads_t* t) { return Heads{t->data, t->stride_batch, t->stride_token, t->stride_head}; }

// ---- head norm and rotation ---------------------------------------------------
void check_rotate(const disco_heads_t* x, int32_t norm, const disco_tensor_t* w, double eps,
                  const disco_rotation_t* r, RotateArgs* a) {
    if (norm != 0 && norm != 1) refuse(DISCO_ERR_INVALID_ARGUMENT, "norm must be 0 or 1");
    if (!norm && w) refuse(DISCO_ERR_INVALID_ARGUMENT, "a weight needs the norm");
    if (norm && (!(eps >= 0.0) || !std::isfinite(eps))) refuse(DISCO_ERR_INVALID_ARGUMENT, "eps must be >= 0 and finite");
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
    if (r->position_stride_batch > kMaxOffset)
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
    if (!std::isfinite(scale)) refuse(DISCO_ERR_INVALID_ARGUMENT, "scale must be finite");
    a->batch = (int32_t)q->batch;
    a->heads = q->heads;
    a->kv_heads = k->heads;
    a->dim = q->dim;
    a->queries = q->tokens;
    a->keys = k->tokens;
    a->scale = (float)scale;
    a->scale2 = (float)(scale * 1.4426950408889634074);
    // (in units of log 2 too such a bias is finite)
    a->bias_limit = (float)std::min(0x1p+100, 0x1p+126 / std::fabs(scale * 1.4426950408889634074));
    a->bf16 = q->dtype == DISCO_BFLOAT16;
    a->q = heads_of(q);
    a->k = heads_of(k);
    if (v) a->v = heads_of(v);
    if (!o) return;
    if (o->bias_stride_batch < 0 || o->bias_stride_batch > kMaxOffset)
        refuse(DISCO_ERR_INVALID_ARGUMENT, "bias stride out of range");
    a->bias = o->key_bias;
    a->bias_sb = o->bias_stride_batch;
    a->lengths = o->key_lengths;
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
        if (!same_place(*x, *y)) check_apart(y, "y", x, "x");
        if (empty(*x)) return;
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
            const disco_heads_t row{dweight->data, dweight->dtype, dy->dim, weight->ndim == 2 ? dy->heads : 1, 0, 1, 1,
                                    0, 0, dy->dim};
            if (x) check_apart(&row, "dweight", x, "x");
            check_apart(&row, "dweight", dy, "dy");
            if (dx) check_apart(&row, "dweight", dx, "dx");
            disco_heads_t wt = row;
            wt.data = weight->data;
            check_apart(&row, "dweight", &wt, "weight");
        }
        if (dx) {
            if (!same_place(*dx, *dy)) check_apart(dx, "dx", dy, "dy");
            if (x) check_apart(dx, "dx", x, "x");
        }
        if (!a.dweight && (!dx || empty(*dy))) return;
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
        const size_t need = a.dweight ? rotate_grad_ws_bytes(a) : 0;
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
        for (auto& t : {std::make_pair(q, "q"), std::make_pair(k, "k"), std::make_pair(v, "v")})
            check_apart(out, "out", t.first, t.second);
        if (low) {
            if (!a.bf16) refuse(DISCO_ERR_DTYPE, "low is for bf16");
            check_output(low, "low");
            check_same(q, "q", low, "low");
            for (auto& t : {std::make_pair(q, "q"), std::make_pair(k, "k"), std::make_pair(v, "v"),
                            std::make_pair((const disco_heads_t*)out, "out")})
                check_apart(low, "low", t.first, t.second);
            a.low = heads_of(low);
        }
        if (empty(*q)) return;
        a.out = heads_of(out);
        a.stats = stats;
        a.stream = stream;
        Device d;
        take_attend(&d, a, q, k);
        d.take(out->data, "out");
        d.take(a.low.p, "low");
        d.take(stats, "stats");
        const size_t need = attend_ws_bytes(a);
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
        const std::pair<const disco_heads_t*, const char*> ins[] = {{q, "q"}, {k, "k"}, {v, "v"}, {out, "out"}, {dout, "dout"}};
        for (int i = 0; i < 3; ++i) {
            check_output(outs[i].first, outs[i].second);
            check_same(outs[i].first, outs[i].second, i == 0 ? q : k, i == 0 ? "q" : "k");
            for (const auto& in : ins) check_apart(outs[i].first, outs[i].second, in.first, in.second);
            if (low) check_apart(outs[i].first, outs[i].second, low, "low");
            for (int j = 0; j < i; ++j) check_apart(outs[i].first, outs[i].second, outs[j].first, outs[j].second);
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
        const size_t need = attend_grad_ws_bytes(a);
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
        const uintptr_t n0 = (uintptr_t)norm;
        Device d;
        d.take(norm, "norm");
        for (const ClipTensor& x : t) {
            if (x.n == 0) continue;
            const uintptr_t len = (uintptr_t)x.n * (x.bf16 ? 2 : 4);
            for (const void* p : {x.g, (const void*)x.out})
                if (p && n0 + sizeof(float) > (uintptr_t)p && n0 < (uintptr_t)p + len)
                    refuse(DISCO_ERR_INVALID_ARGUMENT, "norm overlaps a gradient");
            d.take(x.g, "a gradient");
            if (x.out && x.out != x.g) d.take(x.out, "a clipped gradient");
        }
        const size_t need = clip_ws_bytes(t.data(), (int)t.size());
        if (need && workspace) d.take(workspace, "workspace");
        d.enter();
        Workspace ws(workspace, workspace_bytes, need, stream);
        check_hip(launch_clip(t.data(), (int)t.size(), (float)max_norm, (float)eps, norm, ws.p, stream), "kernel launch");
    });
}

}  // extern "C"
