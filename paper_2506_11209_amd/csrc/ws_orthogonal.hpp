// The two ways of orthogonalising (ws_orthogonal.h): in tiles (ws_orthogonal.hip), and
// by the Gram matrix alone where a side is short (ws_orthogonal_few.hip).
#pragma once

#include "ws_orthogonal.h"

namespace wsg {

constexpr int kFewRows = 64;  // of the shorter side, at the most
constexpr int kFewSteps = 6;  // see ws_orthogonal_few.hip

// Whether the Gram matrix alone is quicker.  us so and in tiles, five steps: 64 x 2048 32
// and 110, 128 x 1024 148 and 97, 128 x 4096 165 and 147.
inline bool by_gram_matrix(int64_t rows, int64_t cols, int32_t steps) {
  return (rows < cols ? rows : cols) <= kFewRows && steps <= kFewSteps;
}

int64_t few_workspace(int64_t rows, int64_t cols, int64_t batch);
ws_status orthogonalize_few(const ws_matrix* G, int32_t steps, const ws_matrix* out, void* workspace, hipStream_t stream);

}  // namespace wsg
