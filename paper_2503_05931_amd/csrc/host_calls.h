// What the host sides of include/aed_train.h and include/aed_vocab.h share: messages of failed calls, workspaces, handles' beginnings and ends.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <exception>
#include <new>
#include <vector>

#include "../../include/aed_train.h"

namespace aed {

extern thread_local char train_error[512];  // aed_train_last_error's

inline aed_status fail(aed_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(train_error, sizeof train_error, fmt, ap);
    va_end(ap);
    return st;
}
inline aed_status hip_status(hipError_t e, const char* what) { return e == hipSuccess ? AED_OK : fail(AED_EHIP, "%s: %s", what, hipGetErrorString(e)); }
// No exception leaves an entry point: what is thrown here is an allocation that failed.
template <typename F> aed_status guarded(F f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return fail(AED_ECAPACITY, "out of host memory");
    } catch (const std::exception& e) {
        return fail(AED_EINVAL, "%s", e.what());
    }
}

inline size_t rounded(size_t n) { return (n + 255) & ~(size_t)255; }

// Tables that go to the workspace's beginning in one copy, then scratch
struct Arena {
    std::vector<char> tables;
    size_t total = 0;
    template <typename T> size_t table(const std::vector<T>& v) {
        const size_t at = tables.size();
        tables.resize(rounded(at + v.size() * sizeof(T)));
        if (!v.empty()) memcpy(tables.data() + at, v.data(), v.size() * sizeof(T));
        return total = tables.size(), at;
    }
    size_t scratch(size_t bytes) {  // after all tables
        const size_t at = total;
        total = rounded(total + bytes);
        return at;
    }
};
inline aed_status check_workspace(const void* ws, size_t have, size_t need) {
    if (!ws) return fail(AED_EINVAL, "workspace is NULL");
    if ((uintptr_t)ws % 256 != 0) return fail(AED_EINVAL, "workspace must be 256-byte aligned");
    if (have < need) return fail(AED_EINVAL, "workspace has %zu bytes, %zu needed", have, need);
    return AED_OK;
}

// A handle whose tables are on their way to the workspace
template <typename P> aed_status start(P* p, void* workspace, size_t bytes, void* hip_stream, P** out) {
    aed_status st = check_workspace(workspace, bytes, p->arena.total);
    p->ws = static_cast<char*>(workspace);
    p->stream = static_cast<hipStream_t>(hip_stream);
    if (st == AED_OK && !p->arena.tables.empty())  // the source lives as long as the handle
        st = hip_status(hipMemcpyAsync(p->ws, p->arena.tables.data(), p->arena.tables.size(), hipMemcpyHostToDevice, p->stream), "copying the work lists");
    if (st != AED_OK) {
        delete p;
        return st;
    }
    *out = p;
    return AED_OK;
}
template <typename P> aed_status finish(P* p) {
    if (!p) return AED_OK;
    const hipError_t e = hipStreamSynchronize(p->stream);
    delete p;
    return hip_status(e, "hipStreamSynchronize");
}

}  // namespace aed
