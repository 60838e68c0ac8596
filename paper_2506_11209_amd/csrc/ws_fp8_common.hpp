// Shared pieces of the 8-bit path: element types, unaligned vector access,
// reductions over 16 lanes, row groups, and host-side checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ws_error.hpp"
#include "ws_fp8.h"

namespace wsg {

constexpr int kBlock = WS_FP8_BLOCK;
constexpr int kScaleOne = 127;  // the E8M0 byte of 1

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

struct bf16_t {
  uint16_t bits;
};
struct f16_t {
  _Float16 v;
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return __uint_as_float((uint32_t)x.bits << 16); }
__device__ __forceinline__ float to_f32(f16_t x) { return (float)x.v; }
// Round to nearest even; NaN stays NaN.
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) {
  return x;
}
template <>
__device__ __forceinline__ bf16_t from_f32<bf16_t>(float x) {
  const __bf16 b = (__bf16)x;
  return bf16_t{__builtin_bit_cast(uint16_t, b)};
}
template <>
__device__ __forceinline__ f16_t from_f32<f16_t>(float x) {
  return f16_t{(_Float16)x};
}

// N consecutive elements, aligned to one: gfx950 loads and stores vectors at
// any element's address (a wave's access takes longer where it straddles more
// cache lines), so rows of any length take the vector path.
template <typename T, int N>
__device__ __forceinline__ void load_n(const T* p, T* out) {
  typedef uint32_t vec __attribute__((ext_vector_type(sizeof(T) * N / 4), aligned(sizeof(T))));
  const vec t = *(const vec*)p;
  __builtin_memcpy(out, &t, sizeof(t));
}
template <typename T, int N>
__device__ __forceinline__ void store_n(T* p, const T* in) {
  typedef uint32_t vec __attribute__((ext_vector_type(sizeof(T) * N / 4), aligned(sizeof(T))));
  vec t;
  __builtin_memcpy(&t, in, sizeof(t));
  *(vec*)p = t;
}

// Maximum over the 16 lanes of a DPP row, in all of them.
__device__ __forceinline__ uint32_t max16(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true));  // row_ror:8
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, true));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, true));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, true));
  return x;
}

// The rows of group i of `groups` among `rows`; i == groups: the rows after the
// last group, i == groups + 1: those before the first.  Offsets that decrease or
// leave the rows are cut to them.
__device__ __forceinline__ void group_rows(const int32_t* offsets, int groups, int64_t rows, int i, int64_t* lo,
                                           int64_t* hi) {
  // both loads at once and for every i; then what they mean at the ends
  int64_t a = offsets[i < groups ? i : groups], b = offsets[i < groups ? i + 1 : 0];
  if (i > groups) a = 0;
  if (i == groups) b = rows;
  a = a < 0 ? 0 : a > rows ? rows : a;
  *lo = a;
  *hi = b < a ? a : b > rows ? rows : b;
}

// x, which is the same in all lanes, as a scalar.
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// The tile of workgroup `id` of n when each XCD (workgroups go round the eight in
// turn) takes a run of neighbours: lines that two tiles share meet in one L2.
__device__ __forceinline__ uint32_t xcd_run(uint32_t id, uint32_t n) {
  const uint32_t share = n / 8, extra = n % 8, x = id % 8;
  return x * share + min(x, extra) + id / 8;
}

struct GroupTile {
  int group;       // -1: none; `groups` and more: rows of no group
  int64_t lo, hi;  // its rows
  int64_t index;   // the tile's number inside the group
  int64_t before;  // tiles of the groups before it
};

// Which group tile `t` belongs to when every group, and then the rows after the
// last and those before the first, are cut into tiles of `size` rows.  Called by
// whole waves; the answer is the same in all lanes.  Sums of 64 groups' tiles at a
// time.
__device__ __forceinline__ GroupTile find_group_tile(const int32_t* offsets, int groups, int64_t rows, int size,
                                                     int64_t t) {
  const int lane = threadIdx.x & 63, n = groups + 2;
  int64_t before = 0;
  for (int first = 0; first < n; first += 64) {
    const int i = first + lane;
    int64_t lo = 0, hi = 0;
    if (i < n) group_rows(offsets, groups, rows, i, &lo, &hi);
    const int tiles = (int)((hi - lo + size - 1) / size);
    int64_t upto = tiles;
    for (int d = 1; d < 64; d *= 2) {
      const int64_t o = __shfl_up(upto, d);
      if (lane >= d) upto += o;
    }
    upto += before;
    const uint64_t past = __ballot(t < upto);
    if (past) {
      const int k = __builtin_ctzll(past);
      GroupTile g;
      g.group = __builtin_amdgcn_readfirstlane(first + k);
      g.lo = uniform(__shfl(lo, k));
      g.hi = uniform(__shfl(hi, k));
      g.before = uniform(__shfl(upto - tiles, k));
      g.index = t - g.before;
      return g;
    }
    before = __shfl(upto, 63);
  }
  return GroupTile{-1, 0, 0, 0, before};
}

// All tiles of the groups and of the rows in none.
__device__ __forceinline__ int64_t count_group_tiles(const int32_t* offsets, int groups, int64_t rows, int size) {
  const GroupTile g = find_group_tile(offsets, groups, rows, size, (int64_t)1 << 60);
  return uniform(g.before);
}

// -- host ---------------------------------------------------------------------

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tiles of `size` rows that hold `rows` rows in `groups` groups and, with `outside`,
// the rows before and after them, whatever the offsets.
inline int64_t group_tiles(int64_t rows, int64_t groups, int size, bool outside) {
  const int64_t parts = groups + (outside ? 2 : 0);
  return (rows + (size - 1) * (parts < rows ? parts : rows)) / size;
}

constexpr int64_t kMaxDim = 1ll << 30;
// Workgroups of `block` threads in one launch: the runtime counts threads of a dimension in 32 bits.
constexpr int64_t max_workgroups(int block) { return ((1ll << 32) - 1) / block; }

inline int elem_size(int32_t dtype) {
  return dtype == WS_OUT_F32 ? 4 : dtype == WS_OUT_BF16 || dtype == WS_OUT_F16 ? 2 : 0;
}

// A dense operand: sizes, type, and data where it has elements.  `batched`: the call
// takes a batch, so that 0 matrices have none; elsewhere batch 0 is a single matrix.
inline bool valid(const ws_matrix* m, bool batched = false) {
  if (!m || m->rows < 0 || m->cols < 0 || m->rows > kMaxDim || m->cols > kMaxDim || m->batch < 0) return false;
  const int size = elem_size(m->dtype);
  if (!size || m->ld < m->cols || m->ld > kMaxDim) return false;
  if (m->batch > 1 && m->rows > 0 && m->cols > 0 && m->stride < (m->rows - 1) * m->ld + m->cols) return false;
  if (m->rows == 0 || m->cols == 0 || (batched && m->batch == 0)) return true;
  return m->data && (uintptr_t)m->data % size == 0;
}

inline bool valid(const ws_fp8_matrix* m, bool batched = false) {
  if (!m || m->rows < 0 || m->cols < 0 || m->rows > kMaxDim || m->cols > kMaxDim || m->batch < 0) return false;
  if (m->block_rows != 1 && m->block_rows != kBlock) return false;
  if (m->ld % 16 || m->ld < ceil_div(m->cols, 16) * 16 || m->ld > kMaxDim) return false;
  if (m->ld_scales < ceil_div(m->rows, m->block_rows) || m->ld_scales > kMaxDim) return false;
  if (m->batch > 1 && m->rows > 0 && m->cols > 0 &&
      (m->stride_codes % 16 || m->stride_codes < (m->rows - 1) * m->ld + ceil_div(m->cols, 16) * 16 ||
       m->stride_scales < (ceil_div(m->cols, kBlock) - 1) * m->ld_scales + ceil_div(m->rows, m->block_rows)))
    return false;
  if (m->rows == 0 || m->cols == 0 || (batched && m->batch == 0)) return true;
  return m->codes && m->scales && (uintptr_t)m->codes % 16 == 0;
}

}  // namespace wsg
