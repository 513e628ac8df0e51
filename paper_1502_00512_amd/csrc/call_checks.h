// Host side of the operators on caller's arrays (logit_ops.hip, adapt_ops.hip): checks of their arguments.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/rnnlm.h"
#include "rows.h"

namespace {

using namespace rnnlm_dev;

#define LAUNCHED()                                             \
  do {                                                         \
    if (hipGetLastError() != hipSuccess) return RNNLM_ERR_HIP; \
  } while (0)

// What a launch can hold is less than 2^32 threads, with up to 1024 of them to a row.
constexpr int32_t LOGITS_V_MAX = 1 << 20;
constexpr int64_t ROWS_MAX = (int64_t(1) << 22) - 64, THREADS_MAX = (int64_t(1) << 32) - 1;

size_t align256(size_t n) { return (n + 255) / 256 * 256; }
bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
size_t elem_bytes(int32_t dtype) { return dtype == RNNLM_DTYPE_FP32 ? 4 : 2; }
// 16-byte slots of a row, the last of them possibly not whole
int slots_of(int32_t V, int32_t dtype) { return (int)(((int64_t)V * (int64_t)elem_bytes(dtype) + 15) / 16); }
bool read_once(int64_t rows, int32_t V, int32_t dtype) { return (double)rows * V * (double)elem_bytes(dtype) > (double)READ_ONCE_BYTES; }
bool tau_ok(float tau) { return std::isfinite(tau) && tau >= 1e-3f && tau <= 1e3f; }

// rows of V elements, ld apart: addresses stay within what 64 bits and the kernels' 32-bit element counts reach
bool rows_ok(const void *p, int32_t dtype, int64_t rows, int32_t V, int64_t ld) {
  if ((!p && rows != 0) || (dtype != RNNLM_DTYPE_FP32 && dtype != RNNLM_DTYPE_BF16) || !aligned(p, elem_bytes(dtype))) return false;
  return rows >= 0 && V >= 1 && V <= LOGITS_V_MAX && ld >= V && ld <= (int64_t(1) << 40) && rows <= ROWS_MAX &&
         (rows == 0 || ld <= (int64_t(1) << 60) / rows);
}

struct Span {
  uintptr_t at, end;
};
Span span(const void *p, size_t bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return {a, p ? a + bytes : a};
}
bool meet(Span a, Span b) { return a.at < b.end && b.at < a.end; }

}  // namespace
