// Error reporting shared by the host-side translation units: fail() stores a
// formatted message as the calling thread's cp_last_error() and returns code.
#pragma once

#include <new>

#include "crosspool.h"

namespace cp {
cp_status fail(cp_status code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

// Runs the body of a C entry point: a host allocation that fails in it becomes
// CP_ENOMEM (no exception leaves the library).
template <class F>
cp_status guarded(F &&body) {
  try {
    return body();
  } catch (const std::bad_alloc &) {
    return fail(CP_ENOMEM, "host allocation failed");
  }
}
}  // namespace cp
