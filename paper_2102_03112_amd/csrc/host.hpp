// host.hpp -- what the C ABI's source files share on the host: the error
// message of the calling thread, the workspace check and the tracing mark of
// an entry point (api.hip holds them).
#pragma once

#include <hip/hip_runtime.h>

#include <stddef.h>
#include <stdint.h>

#include "deepreduce.h"

namespace dr {

// Set the thread's error message and return st.
dr_status fail(dr_status st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
dr_status hip_fail(hipError_t e, const char *where);

bool ws_ok(const void *ws, size_t ws_bytes, size_t need);

// Per-kernel timing: every entry point that launches work marks its start.
void trace_call(hipStream_t s);

constexpr uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
constexpr uint64_t align_up(uint64_t a, uint64_t b) { return ceil_div(a, b) * b; }

}  // namespace dr

#define DR_HIP(call)                                          \
    do {                                                      \
        hipError_t e_ = (call);                               \
        if (e_ != hipSuccess) return dr::hip_fail(e_, #call); \
    } while (0)
