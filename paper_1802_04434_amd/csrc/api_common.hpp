// What the files behind the C ABI (include/signsgd.h) share: validation of buffers, and the launch call.
#pragma once
#include "../../include/signsgd.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "common.hpp"

namespace host {

// of this thread's most recent SS_ERR_HIP, whichever file's call it was
inline thread_local int g_last_hip_error = 0;

constexpr size_t kMaxGrid = 0x7FFFFFFFull;

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline size_t grad_bytes(ss_dtype gdt) { return gdt == SS_BF16 ? 2 : 4; }

// A buffer of one call, for the check that nothing that is written shares a byte
// with anything else (buffers that are only read may coincide, e.g. one gradient
// handed in for two workers).
struct Span {
    uintptr_t lo, hi;   // [lo, hi); empty spans (NULL pointer or no bytes) never overlap
    bool written;
};

inline Span span(const void *p, size_t bytes, bool written) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return Span{lo, p ? lo + bytes : lo, written};
}

// sorts s; true iff a written span overlaps any other span
inline bool written_spans_overlap(Span *s, int n) {
    std::sort(s, s + n, [](const Span &a, const Span &b) { return a.lo < b.lo; });
    uintptr_t end_any = 0, end_written = 0;   // furthest end among the spans seen so far
    for (int i = 0; i < n; ++i) {
        if (s[i].lo == s[i].hi) continue;
        if (s[i].lo < (s[i].written ? end_any : end_written)) return true;
        end_any = std::max(end_any, s[i].hi);
        if (s[i].written) end_written = std::max(end_written, s[i].hi);
    }
    return false;
}

// Every kernel takes one argument struct by value.  The status is the launch
// call's own return value: an error left on this thread by an earlier, unrelated
// runtime call is neither reported as ours nor cleared.
template <typename Args>
int launch(void (*kernel)(Args), size_t grid, unsigned lds_bytes, hipStream_t stream, const Args &a,
           int block = ss::kBlock, int grid_y = 1) {
    void *params[1] = {const_cast<Args *>(&a)};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)grid, (unsigned)grid_y),
                                         dim3((unsigned)block), params, lds_bytes, stream);
    if (e != hipSuccess) {
        g_last_hip_error = (int)e;
        return SS_ERR_HIP;
    }
    return SS_OK;
}

}  // namespace host
