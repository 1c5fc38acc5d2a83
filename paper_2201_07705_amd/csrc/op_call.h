// What the calls of all operators share on the host: the state of a context's
// operators, workspaces, and checks of arguments.
#pragma once
#include <algorithm>
#include <cstring>
#include <map>
#include <memory>
#include <new>
#include <string>
#include <thread>
#include <utility>
#include <vector>

#ifdef __SANITIZE_ADDRESS__
#include <sanitizer/asan_interface.h>
#endif

#include "internal.h"
#include "op_args.h"

namespace gemel {
namespace op {

struct DeviceScope {
    int prev = -1;
    explicit DeviceScope(int d) {
        if (hipGetDevice(&prev) != hipSuccess) prev = -1;
        if (prev != d)
            (void)hipSetDevice(d);
        else
            prev = -1;
    }
    ~DeviceScope() {
        if (prev >= 0) (void)hipSetDevice(prev);
    }
};

inline gemel_status hip_fail(gemel_ctx *ctx, hipError_t e, const char *what) {
    return fail(ctx, e == hipErrorOutOfMemory ? GEMEL_ENOMEM : GEMEL_EDEVICE,
                std::string(what) + ": " + hipGetErrorString(e));
}
#define OPCHK(call, what)                                   \
    do {                                                    \
        const hipError_t e_ = (call);                       \
        if (e_ != hipSuccess) return hip_fail(ctx, e_, what); \
    } while (0)

// Requests grouped by adapter. Positions are rows sorted by adapter (rows
// without one first), in row order within one, so that a tile of positions
// meets few adapters whatever the order of the requests.
struct Batch {
    BatchTables t{};
    void *dev = nullptr;
    size_t bytes = 0;
    std::vector<hipStream_t> streams;   // that its calls ran on
    bool held = false;                  // a graph, or another thread's stream, may hold its addresses
};

// Tables given back that enqueued work may still read: until events, recorded
// on the streams that their calls ran on, have passed.
struct Retired {
    void *dev;
    size_t bytes;
    std::vector<hipStream_t> streams;   // without an event yet
    std::vector<hipEvent_t> events;
};

// A stretch of device memory that the kernels of one stream share.
struct Workspace {
    char *p = nullptr;
    size_t bytes = 0;
    bool captured = false;   // a graph may hold its address
};

struct State : OperatorState {
    int device;
    void *zero = nullptr;        // 256 zero bytes
    hipStream_t side = nullptr;  // uploads of tables
    void *pinned = nullptr;      // they are staged in
    size_t pinned_bytes = 0;
    std::vector<void *> outgrown;   // staging memory before (to free it would wait for the device)
    std::map<std::pair<hipStream_t, std::thread::id>, Workspace> ws;   // (each thread's own hipStreamPerThread)
    std::vector<char *> captured;   // outgrown workspaces that graphs may use
    std::vector<std::unique_ptr<Batch>> batches;
    // tables given back: nobody reads `spare` ones; work on streams that cannot
    // be asked (replays of graphs) may still read `held` ones
    std::vector<std::pair<void *, size_t>> spare, held;
    std::vector<Retired> retired;
    std::vector<hipEvent_t> events;   // not in use

    explicit State(int d) : device(d) {}
    bool release() override {
        DeviceScope scope(device);
        const bool ok = hipDeviceSynchronize() == hipSuccess;
        for (auto &w : ws)
            if (w.second.p) (void)hipFree(w.second.p);
        for (char *p : captured) (void)hipFree(p);
        for (auto &b : batches)
            if (b && b->dev) (void)hipFree(b->dev);
        for (auto *v : {&spare, &held})
            for (auto &b : *v) (void)hipFree(b.first);
        for (auto &r : retired) {
            (void)hipFree(r.dev);
            for (hipEvent_t e : r.events) (void)hipEventDestroy(e);
        }
        for (hipEvent_t e : events) (void)hipEventDestroy(e);
        if (zero) (void)hipFree(zero);
        if (pinned) (void)hipHostFree(pinned);
        for (void *p : outgrown) (void)hipHostFree(p);
        if (side) (void)hipStreamDestroy(side);
        ws.clear();
        captured.clear();
        batches.clear();
        spare.clear();
        held.clear();
        retired.clear();
        events.clear();
        outgrown.clear();
        zero = pinned = nullptr;
        side = nullptr;
        return ok;
    }
};

inline gemel_status ready(gemel_ctx *ctx, State **out) {
    if (ctx->operators) {
        *out = static_cast<State *>(ctx->operators.get());
        return GEMEL_OK;
    }
    int n = 0;
    OPCHK(hipGetDeviceCount(&n), "hipGetDeviceCount");
    if (ctx->device >= n) return fail(ctx, GEMEL_EINVAL, "device index beyond the visible devices");
    hipDeviceProp_t prop;
    OPCHK(hipGetDeviceProperties(&prop, ctx->device), "hipGetDeviceProperties");
    if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0)
        return fail(ctx, GEMEL_EDEVICE, std::string("libgemel is built for gfx950; device is ") + prop.gcnArchName);
    auto st = std::make_unique<State>(ctx->device);
    hipError_t e = hipMalloc(&st->zero, 256);
    if (e == hipSuccess) e = hipStreamCreateWithFlags(&st->side, hipStreamNonBlocking);
    if (e == hipSuccess) e = launch_fill_u32((uint32_t *)st->zero, 64, 0, Sink{st->side});
    if (e == hipSuccess) e = hipStreamSynchronize(st->side);
    if (e != hipSuccess) {
        st->release();
        return hip_fail(ctx, e, "operator state");
    }
    *out = st.get();
    ctx->operators = std::move(st);
    return GEMEL_OK;
}

// The same for a call on a stream: a context sets up nothing while that is
// captured.
inline gemel_status ready(gemel_ctx *ctx, hipStream_t stream, State **out) {
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (!ctx->operators && stream) OPCHK(hipStreamIsCapturing(stream, &cs), "hipStreamIsCapturing");
    if (cs != hipStreamCaptureStatusNone)
        return fail(ctx, GEMEL_ESTATE, "the context's first call cannot be captured: make it once before");
    return ready(ctx, out);
}

// Offsets of a call's buffers in its stream's workspace.
struct Layout {
    size_t bytes = 0;
    size_t take(int64_t n, size_t elem) {
        const size_t at = bytes;
        bytes += (size_t)op_round_up(n * (int64_t)elem, 256);
#ifdef __SANITIZE_ADDRESS__
        pieces.emplace_back(at, (size_t)n * elem);
        bytes += 256;
#endif
        return at;
    }
#ifdef __SANITIZE_ADDRESS__
    // CPU builds with AddressSanitizer: only the pieces themselves may be accessed
    std::vector<std::pair<size_t, size_t>> pieces;
    void fence(char *base, size_t all) const {
        ASAN_POISON_MEMORY_REGION(base, all);
        for (const auto &p : pieces) ASAN_UNPOISON_MEMORY_REGION(base + p.first, p.second);
    }
#else
    void fence(char *, size_t) const {}
#endif
};

// The call's pieces of its stream's workspace; `batch` (or null) is noted as
// used on the stream.
inline gemel_status workspace(gemel_ctx *ctx, State &st, hipStream_t stream, const Layout &lay, Batch *batch, char **out) {
    // one handle, a stream for each thread: another thread cannot ask for its
    // work, which is waited for with the device
    const bool per_thread = stream == hipStreamPerThread;
    Workspace &w = st.ws[{stream, per_thread ? std::this_thread::get_id() : std::thread::id()}];
    size_t bytes = lay.bytes;
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (stream) OPCHK(hipStreamIsCapturing(stream, &cs), "hipStreamIsCapturing");
    if (w.bytes < bytes) {
        if (cs != hipStreamCaptureStatusNone)
            return fail(ctx, GEMEL_ESTATE, "the stream's workspace is too small to be captured: make the call once before");
        bytes = (size_t)op_round_up((int64_t)bytes, 2 << 20);
        if (w.p) {
            OPCHK(hipDeviceSynchronize(), "hipDeviceSynchronize");
            if (w.captured)
                st.captured.push_back(w.p);
            else
                (void)hipFree(w.p);
            w = Workspace();
        }
        void *p = nullptr;
        OPCHK(hipMalloc(&p, bytes), "workspace");
        w.p = (char *)p;
        w.bytes = bytes;
    }
    if (cs != hipStreamCaptureStatusNone) w.captured = true;
    if (batch && (cs != hipStreamCaptureStatusNone || per_thread))
        batch->held = true;
    else if (batch && std::find(batch->streams.begin(), batch->streams.end(), stream) == batch->streams.end())
        batch->streams.push_back(stream);
    lay.fence(w.p, w.bytes);
    *out = w.p;
    return GEMEL_OK;
}

// Rows of device memory that a call reads or writes.
struct Range {
    const char *what;
    uintptr_t lo, hi;        // from the first row to the end of the last
    uintptr_t stride, width; // bytes (stride 0: one stretch)
    bool out;
};
inline Range range(const char *what, const void *p, int64_t bytes, bool out) {
    return {what, (uintptr_t)p, (uintptr_t)p + (p ? (uintptr_t)bytes : 0), 0, 0, out};
}
inline Range range(const char *what, const void *p, int64_t rows, int64_t cols, int64_t stride, int64_t elem, bool out) {
    Range r = range(what, p, rows > 0 ? ((rows - 1) * stride + cols) * elem : 0, out);
    r.stride = (uintptr_t)(stride * elem);
    r.width = (uintptr_t)(cols * elem);
    return r;
}
// Whether the rows of two ranges share bytes. Rows of one stride may lie side
// by side, as columns of one wider matrix; of different strides their whole
// spans count.
inline bool overlap(const Range &a, const Range &b) {
    if (a.lo >= b.hi || b.lo >= a.hi) return false;
    if (!a.stride || a.stride != b.stride) return true;
    const uintptr_t d = b.lo >= a.lo ? (b.lo - a.lo) % a.stride : (a.stride - (a.lo - b.lo) % a.stride) % a.stride;
    return d < a.width || d + b.width > a.stride;
}
inline gemel_status apart(gemel_ctx *ctx, const std::vector<Range> &r) {
    for (size_t i = 0; i < r.size(); ++i)
        for (size_t j = 0; j < r.size(); ++j)
            if (r[i].out && i != j && overlap(r[i], r[j]))
                return fail(ctx, GEMEL_EINVAL, std::string(r[i].what) + " overlaps " + r[j].what);
    return GEMEL_OK;
}

struct Call {
    gemel_ctx *ctx;
    State *st;
    hipStream_t stream;
    Batch *batch;
    Layout lay;
    char *base = nullptr;
    template <typename T>
    T *at(size_t off) const {
        return (T *)(base + off);
    }
};

inline gemel_status workspace(Call &c) { return workspace(c.ctx, *c.st, c.stream, c.lay, c.batch, &c.base); }

inline gemel_status check_aligned(gemel_ctx *ctx, const char *what, const void *p, int64_t elem) {
    if ((uintptr_t)p % (uintptr_t)elem) return fail(ctx, GEMEL_EINVAL, std::string(what) + " is not aligned to its type");
    return GEMEL_OK;
}

inline gemel_status check_rows(gemel_ctx *ctx, const char *what, const void *p, int64_t stride, int64_t cols, int64_t elem) {
    if (!p) return fail(ctx, GEMEL_EINVAL, std::string(what) + " is null");
    if (stride < cols || stride > INT32_MAX) return fail(ctx, GEMEL_EINVAL, std::string(what) + " has a bad row stride");
    return check_aligned(ctx, what, p, elem);
}

inline int64_t partial_floats(const MmArgs &a) {
    return a.splits > 1 ? (int64_t)a.splits * a.batch * a.M * a.ldp : 0;
}
// Rows that a product reads where they are; others are copied first.
inline bool in_place(const void *p, int64_t rows, int64_t ld, int64_t cols) {
    return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && cols % 8 == 0 && ld <= MM_MAX_LD && rows * ld <= 1ll << 30;
}

// Runs f, with host allocation failures as a status.
template <typename F>
inline gemel_status guarded(gemel_ctx *ctx, F &&f) {
    try {
        return f();
    } catch (const std::bad_alloc &) {
        return fail(ctx, GEMEL_ENOMEM, "out of host memory");
    } catch (const std::exception &e) {
        return fail(ctx, GEMEL_EDEVICE, e.what());
    }
}

}  // namespace op
}  // namespace gemel
