// Host-side helpers that every source of the library's C ABI uses (defined in deinfer_api.hip where not inline).
#pragma once
#include "../../include/deinfer.h"
#include "common.h"

#define DEINFER_HIDDEN __attribute__((visibility("hidden")))

namespace deinfer {

// Sets the calling thread's error text and returns code.
DEINFER_HIDDEN int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
// Compute units of the current device (asked once per device); -1: none can be asked.
DEINFER_HIDDEN int device_cus();
// DEINFER_OK, or the error that the launch `what` left.
DEINFER_HIDDEN int check_launch(const char *what);

inline int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t elem_size(int dtype) { return dtype == DEINFER_F32 ? 4 : 2; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Calls f with a value of the element type of `dtype` (float, uint16_t for bf16, f16_bits for fp16).
template <typename F>
int by_dtype(int dtype, F f) {
  if (dtype == DEINFER_F32) return f(float{});
  if (dtype == DEINFER_F16) return f(f16_bits{});
  return f(uint16_t{});
}

}  // namespace deinfer
