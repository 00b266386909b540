// Checks of arguments that the C entries of the training operators share.
#pragma once

#include <new>

#include "dd_elem.h"
#include "dd_train.h"

namespace dd {

inline bool float_type(int32_t t) { return t == DD_F32 || t == DD_BF16 || t == DD_F16; }

inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// Whether work on s goes into a graph.
inline hipError_t captured(hipStream_t s, bool *yes) {
    hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
    const hipError_t e = hipStreamIsCapturing(s, &st);
    *yes = st != hipStreamCaptureStatusNone;
    return e;
}

// What every C entry runs in: nothing thrown gets out.
template <class F>
dd_status guarded(const F &f) {
    no_error();
    try {
        return f();
    } catch (const std::bad_alloc &) {
        return fail(DD_ENOMEM, "out of host memory");
    } catch (...) {
        return fail(DD_EHIP, "unexpected failure in host code");
    }
}

// Rows of an array: where they start, and how far apart.
inline dd_status check_rows(const char *name, const void *p, int64_t rows, int64_t cols, int64_t stride, int32_t type, bool output) {
    if (!p) return fail(DD_EINVAL, "%s is NULL", name);
    if (!aligned(p, elem_size(type))) return fail(DD_EINVAL, "%s is not aligned to its elements", name);
    if (rows <= 1) return DD_OK;
    if (stride < 0 || (output && stride < cols)) return fail(DD_EINVAL, "%s: stride %lld", name, (long long)stride);
    if (stride > (int64_t(1) << 60) / rows) return fail(DD_EINVAL, "%s: stride %lld is too large", name, (long long)stride);
    return DD_OK;
}

#define CHECK(x)                          \
    do {                                  \
        const dd_status st_ = (x);        \
        if (st_ != DD_OK) return st_;     \
    } while (0)

}  // namespace dd
