// kt_host.h -- host helpers that the library's translation units share.
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/kt.h"

namespace kt {

// The calling thread's error text (kt_last_error); `fail` sets it and returns its first argument.
void clear_error();
__attribute__((format(printf, 2, 3))) kt_status fail(kt_status code, const char* fmt, ...);

// Raises a kernel's limit of dynamic LDS on the current device (once).
bool ensure_dynamic_lds(const void* kernel, size_t bytes);

static inline bool launch_ok() { return hipGetLastError() == hipSuccess; }

static inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

constexpr int kNumCUs = 256;

}  // namespace kt
