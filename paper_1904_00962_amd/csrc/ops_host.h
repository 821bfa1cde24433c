// Host-side helpers shared by the entry points of include/lamb_ops.h. Not
// installed.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include <algorithm>
#include <exception>
#include <new>
#include <vector>

#include "lamb_host.h"
#include "lamb_ops.h"

namespace lamb_mi355x {

constexpr int kXcds = 8;  // accelerator dies, each with its own L2; blocks go to them in turn

// Workgroup b runs on die b % kXcds. Deals the items to the dies in runs, so that tiles
// that read the same operand rows share an L2, and each die still gets its part of the
// long items, which come first.
template <class T>
std::vector<T> spread_over_dies(const std::vector<T> &items) {
    constexpr size_t kRun = 8;
    const size_t n = items.size(), whole = n / (kXcds * kRun) * (kXcds * kRun);
    std::vector<T> out(n);
    for (size_t b = 0; b < n; ++b) {
        const size_t die = b % kXcds, at = b / kXcds;
        out[b] = b < whole ? items[(at / kRun * kXcds + die) * kRun + at % kRun] : items[b];
    }
    return out;
}

// A launch has fewer than 2^32 threads along an axis: many workgroups go along two, and
// those past `blocks` find nothing to do.
inline dim3 grid_of(int64_t blocks) {
    constexpr int64_t kAxis = int64_t(1) << 21;
    return blocks <= kAxis ? dim3(uint32_t(blocks))
                           : dim3(uint32_t(kAxis), uint32_t((blocks + kAxis - 1) / kAxis));
}

// Runs an entry point's body; what it throws becomes a status.
template <class F>
lamb_status guarded(F body) noexcept {
    try {
        return body();
    } catch (const std::bad_alloc &) {
        return fail(LAMB_ENOMEM, "host allocation failed");
    } catch (const std::exception &e) {
        return fail(LAMB_EINVAL, "%s", e.what());
    }
}

inline bool aligned_to(const void *p, uintptr_t bytes) {
    return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
}

inline int64_t round_up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }

struct DeviceScope {
    int previous = -1;
    explicit DeviceScope(int device) {
        if (hipGetDevice(&previous) == hipSuccess && previous != device)
            (void)hipSetDevice(device);
        else
            previous = -1;
    }
    ~DeviceScope() {
        if (previous >= 0)
            (void)hipSetDevice(previous);
    }
};

// The end of a plan's last call outside a capture, and its stream: see ordered().
struct CallOrder {
    hipEvent_t done = nullptr;
    hipStream_t stream = nullptr;
    bool used = false;
};

// Calls of one plan share its workspace: one on another stream than the last waits for
// that one. A captured call is left out; when its graph runs is the caller's to order.
template <class F>
lamb_status ordered(CallOrder &order, hipStream_t stream, F enqueue) {
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    hipError_t err = hipStreamIsCapturing(stream, &capture);
    if (err != hipSuccess)
        return fail_hip(err, "hipStreamIsCapturing");
    if (capture != hipStreamCaptureStatusNone)
        return enqueue();
    if (order.used && order.stream != stream) {
        err = hipStreamWaitEvent(stream, order.done, 0);
        if (err != hipSuccess)
            return fail_hip(err, "hipStreamWaitEvent");
    }
    const lamb_status st = enqueue();
    // also after a failure: what went out before it uses the workspace
    err = hipEventRecord(order.done, stream);
    order.stream = stream;
    order.used = true;
    if (st == LAMB_OK && err != hipSuccess)
        return fail_hip(err, "hipEventRecord");
    return st;
}

// Memory that a call reads or writes, for the overlap check: bytes lo to hi, or of these
// `row` at every multiple of `stride` from lo on.
struct Span {
    uintptr_t lo, hi;
    bool written;
    int32_t index;
    const char *what;
    uint64_t row, stride;  // stride 0: every byte
};

inline Span span_of(const void *p, uint64_t bytes, bool written, int32_t index, const char *what) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return Span{lo, lo + uintptr_t(bytes), written, index, what, bytes, 0};
}

// `rows` rows of `cols` elements, `stride` elements apart; rows 0: no memory.
inline Span span_of_rows(const void *p, int64_t rows, int64_t stride, int64_t cols, int64_t size,
                         bool written, int32_t index, const char *what) {
    const uint64_t bytes = rows ? uint64_t((rows - 1) * stride + cols) * uint64_t(size) : 0;
    Span s = span_of(p, bytes, written, index, what);
    if (rows > 1) {
        s.row = uint64_t(cols * size);
        s.stride = uint64_t(stride * size);
    }
    return s;
}

// Whether two spans, s.lo <= t.lo, share a byte. Rows of one stride may lie between each
// other, as column slices of one buffer do; of two strides only the ends are looked at.
inline bool share_bytes(const Span &s, const Span &t) {
    if (t.lo >= s.hi || t.lo == t.hi)
        return false;
    if (s.stride == 0 || (t.stride != 0 && t.stride != s.stride))
        return true;
    const uint64_t at = uint64_t(t.lo - s.lo) % s.stride;
    return at < s.row || t.row > s.stride - at;
}

// Written memory overlaps nothing; what is only read may overlap. Sorts the spans.
inline lamb_status check_spans(Span *spans, size_t n) {
    std::sort(spans, spans + n, [](const Span &p, const Span &q) {
        return p.lo != q.lo ? p.lo < q.lo : p.hi < q.hi;
    });
    uintptr_t read_to = 0, written_to = 0;  // the furthest ends so far
    for (size_t i = 0; i < n; ++i) {
        const Span &s = spans[i];
        const bool near = s.lo < written_to || (s.written && s.lo < read_to);
        for (size_t k = 0; near && k < i; ++k)
            if ((s.written || spans[k].written) && share_bytes(spans[k], s))
                return fail(LAMB_EOVERLAP, "%s (%d) overlaps %s (%d)", s.what, s.index,
                            spans[k].what, spans[k].index);
        uintptr_t &far = s.written ? written_to : read_to;
        far = std::max(far, s.hi);
    }
    return LAMB_OK;
}

// The limits that the operators' entry points share. Rows times stride times 8 bytes stay
// below 2^63.
constexpr int64_t kMaxTokens = int64_t(1) << 24, kMaxVocab = int64_t(1) << 24,
                  kMaxDim = int64_t(1) << 16, kMaxStride = int64_t(1) << 36;

inline bool is_float(int32_t dtype) {
    return dtype == LAMB_DTYPE_F32 || dtype == LAMB_DTYPE_BF16;
}
inline bool is_id(int32_t dtype) { return dtype == LAMB_DTYPE_I32 || dtype == LAMB_DTYPE_I64; }
inline int64_t size_of(int32_t dtype) {
    return dtype == LAMB_DTYPE_BF16 ? 2 : dtype == LAMB_DTYPE_I64 ? 8 : 4;
}

inline lamb_status check_workspace(const void *workspace, size_t bytes, size_t need) {
    if (!workspace)
        return fail(LAMB_ENULL, "workspace must not be NULL");
    if (!aligned_to(workspace, 256))
        return fail(LAMB_EALIGN, "the workspace must be 256-byte aligned");
    if (bytes < need)
        return fail(LAMB_EINVAL, "the workspace has %zu bytes, the call needs %zu", bytes, need);
    return LAMB_OK;
}

}  // namespace lamb_mi355x
