// The two ways of orthogonalising (ws_orthogonal.h): in tiles (ws_orthogonal.hip), and
// by the Gram matrix alone where a side is short (ws_orthogonal_few.hip).
#pragma once

#include <atomic>

#include "ws_error.hpp"
#include "ws_orthogonal.h"

namespace wsg {

// Lets a kernel use this much LDS on the current device; `allowed`: the kernel's own, the
// devices that have been asked.
inline ws_status allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>& allowed) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess && (dev >= 64 || !(allowed.load(std::memory_order_acquire) >> dev & 1))) {
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess && dev < 64) allowed.fetch_or(1ull << dev, std::memory_order_acq_rel);
  }
  return e == hipSuccess ? WS_OK : hip_fail("hipFuncSetAttribute", e);
}

constexpr int kFewRows = 64;  // of the shorter side, at the most
constexpr int kFewSteps = 6;  // see ws_orthogonal_few.hip

// Whether the Gram matrix alone is quicker.  us so and in tiles, five steps: 16 x 2048 15 and
// 146, 64 x 512 45 and 100, 64 x 2048 48 and 147; 128 rows in binary64 are more than a CU's LDS.
inline bool by_gram_matrix(int64_t rows, int64_t cols, int32_t steps) {
  return (rows < cols ? rows : cols) <= kFewRows && steps <= kFewSteps;
}

int64_t few_workspace(int64_t rows, int64_t cols, int64_t batch);
ws_status orthogonalize_few(const ws_matrix* G, int32_t steps, const ws_matrix* out, void* workspace, hipStream_t stream);

}  // namespace wsg
