// disco_token_abi.h -- what the C entries of the token operators share: refusals
// and the guard that no exception passes, the device of a call, its workspace, and
// the checks of token tensors and of the places that a call writes.
#pragma once
#include <rocprofiler-sdk-roctx/roctx.h>

#include <algorithm>
#include <cstring>
#include <exception>
#include <initializer_list>
#include <new>
#include <string>
#include <utility>

#include "disco.h"
#include "disco_heads.h"
#include "disco_internal.h"

namespace disco {
namespace token {

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

[[noreturn]] inline void refuse(disco_status_t s, std::string why) { throw Refusal{s, std::move(why)}; }

inline void check_hip(hipError_t e, const char* what) {
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

inline size_t bytes_of(int32_t dtype) { return dtype == DISCO_BFLOAT16 ? 2 : 4; }

constexpr int64_t kMaxRows = (int64_t)1 << 31;       // tokens of all batch items
constexpr int64_t kMaxOffset = (int64_t)1 << 46;     // element offsets

inline bool empty(const disco_heads_t& t) { return t.batch == 0 || t.tokens == 0 || t.heads == 0; }

// Elements from the first to one past the last.
inline int64_t extent(const disco_heads_t& t) {
    return empty(t) ? 0
                    : (t.batch - 1) * t.stride_batch + (t.tokens - 1) * t.stride_token +
                          (t.heads - 1) * t.stride_head + t.dim;
}

inline void check_heads(const disco_heads_t* t, const char* name) {
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
inline void check_output(const disco_heads_t* t, const char* name) {
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

inline void check_same(const disco_heads_t* a, const char* na, const disco_heads_t* b, const char* nb) {
    if (a->dtype != b->dtype) refuse(DISCO_ERR_DTYPE, std::string(na) + " and " + nb + " have different dtypes");
    if (a->batch != b->batch || a->tokens != b->tokens || a->heads != b->heads || a->dim != b->dim)
        refuse(DISCO_ERR_SHAPE, std::string(na) + " and " + nb + " have different sizes");
}

// The memory of an argument: rows of `width` bytes, n[i] of them `stride[i]` bytes
// apart along batch, token and head; one row for a dense argument.
struct Place {
    const char* name;
    uintptr_t p;
    int64_t width, stride[3], n[3];
    bool none() const { return p == 0 || width == 0 || n[0] == 0 || n[1] == 0 || n[2] == 0; }
    uintptr_t end() const {
        uintptr_t e = p + (uintptr_t)width;
        for (int i = 0; i < 3; ++i) e += (uintptr_t)(stride[i] * (n[i] - 1));
        return e;
    }
};
inline Place place(const char* name, const disco_heads_t* t) {
    if (!t) return Place{name, 0, 0, {0, 0, 0}, {1, 1, 1}};
    const int64_t e = (int64_t)bytes_of(t->dtype);
    return Place{name, (uintptr_t)t->data, t->dim * e, {t->stride_batch * e, t->stride_token * e, t->stride_head * e},
                 {t->batch, t->tokens, t->heads}};
}
inline Place place(const char* name, const void* p, int64_t bytes) { return Place{name, (uintptr_t)p, p ? bytes : 0, {0, 0, 0}, {1, 1, 1}}; }

// An axis that two places step along alike, with what the axes after it span.
struct Axis {
    int64_t stride, na, nb, span_a, span_b;
};

// Whether some ia stride + ea along the axes is some ib stride + eb + d, ea < wa and eb
// < wb: along each axis few differences ia - ib bring d within reach of what the
// axes after it span, and where more than a few do, b covers rows of a.
inline bool meets(const Axis* ax, int n, int64_t d, int64_t wa, int64_t wb) {
    if (n == 0) return d > -wb && d < wa;
    auto below = [](int64_t x, int64_t s) { return x >= 0 ? x / s : -((-x + s - 1) / s); };
    const int64_t s = ax->stride;
    const int64_t lo = std::max(1 - ax->nb, below(d - ax->span_a, s)), hi = std::min(ax->na - 1, below(d + ax->span_b, s) + 1);
    if (hi - lo > 4) return true;
    for (int64_t i = lo; i <= hi; ++i)
        if (meets(ax + 1, n - 1, d - i * s, wa, wb)) return true;
    return false;
}

// Whether two places may share memory: exactly where they have the same
// strides along nested axes, as the parts of one joint buffer do in any order of
// its axes, or where one of them is a single row.  With other strides, tensors whose
// tokens lie equally far apart are told apart by their place within a token,
// all others by the memory from their first to their last byte.
inline bool may_overlap(const Place& a, const Place& b) {
    if (a.none() || b.none() || a.end() <= b.p || b.end() <= a.p) return false;
    Axis ax[3];
    int n = 0;
    bool alike = true, single_a = true, single_b = true;
    for (int i = 0; i < 3; ++i) {
        const int64_t na = a.stride[i] == 0 ? 1 : a.n[i], nb = b.stride[i] == 0 ? 1 : b.n[i];
        if (na > 1 && nb > 1 && a.stride[i] != b.stride[i]) alike = false;
        if (na > 1 || nb > 1) ax[n++] = Axis{na > 1 ? a.stride[i] : b.stride[i], na, nb, 0, 0};
        single_a = single_a && na == 1;
        single_b = single_b && nb == 1;
    }
    std::sort(ax, ax + n, [](const Axis& p, const Axis& q) { return p.stride > q.stride; });
    int64_t span_a = a.width, span_b = b.width;
    for (int i = n - 1; i >= 0 && alike; --i) {
        alike = (single_a || ax[i].stride >= span_a) && (single_b || ax[i].stride >= span_b);
        ax[i].span_a = span_a;
        ax[i].span_b = span_b;
        span_a += ax[i].stride * (ax[i].na - 1);
        span_b += ax[i].stride * (ax[i].nb - 1);
    }
    if (alike) return meets(ax, n, (int64_t)b.p - (int64_t)a.p, a.width, b.width);

    const int64_t step = a.stride[1];
    if (step > 0 && step == b.stride[1] && (a.n[0] == 1 || a.stride[0] % step == 0) && (b.n[0] == 1 || b.stride[0] % step == 0)) {
        const int64_t wa = (a.n[2] - 1) * a.stride[2] + a.width, wb = (b.n[2] - 1) * b.stride[2] + b.width;
        const int64_t d = a.p >= b.p ? (int64_t)((a.p - b.p) % (uintptr_t)step) : (step - (int64_t)((b.p - a.p) % (uintptr_t)step)) % step;
        if (d >= wb && d + wa <= step) return false;
    }
    return true;
}

// Of tensors of one size: whether each entry of one lies where the other's does
// (the stride of a single entry leads nowhere).
inline bool same_place(const disco_heads_t& a, const disco_heads_t& b) {
    return a.data == b.data && (a.batch <= 1 || a.stride_batch == b.stride_batch) &&
           (a.tokens <= 1 || a.stride_token == b.stride_token) && (a.heads <= 1 || a.stride_head == b.stride_head);
}

// Everything that a call writes lies apart from all else that it reads and writes.
inline void check_apart(std::initializer_list<Place> written, std::initializer_list<Place> read) {
    for (const Place* w = written.begin(); w != written.end(); ++w) {
        auto check = [&](const Place& o) {
            if (may_overlap(*w, o)) refuse(DISCO_ERR_INVALID_ARGUMENT, std::string(w->name) + " overlaps " + o.name);
        };
        for (const Place& r : read) check(r);
        for (const Place* o = written.begin(); o != w; ++o) check(*o);
    }
}

inline Heads heads_of(const disco_heads_t* t) { return Heads{t->data, t->stride_batch, t->stride_token, t->stride_head}; }

}  // namespace token
}  // namespace disco
