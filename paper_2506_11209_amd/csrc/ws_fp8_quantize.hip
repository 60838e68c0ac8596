// Quantisation by blocks of 128 (formulas: ws_fp8.h).
#include "ws_fp8_common.hpp"

namespace wsg {
namespace {

struct QuantArgs {
  const void* x;
  int64_t x_rows, ld;       // rows that index may name, elements between them
  int64_t rows, cols;       // of the result's row form
  const int32_t* index;     // source row of each row; null: itself
  const int32_t* offsets;   // groups + 1, or null
  int32_t groups;
  uint8_t *codes, *scales;  // row form (weight: of w)
  int64_t ld_codes, ld_scales;
  uint8_t *codes_t, *scales_t;  // column form (weight: of its transpose; may be null)
  int64_t ld_codes_t, ld_scales_t;
  int64_t padded;           // with groups: blocks of 128 of the column form
  int64_t stride_x, stride_codes, stride_scales, stride_codes_t, stride_scales_t;  // batch
  int64_t row_tiles, col_tiles;
  int32_t runs;             // rows do not start at cache lines: neighbouring tiles on one XCD
};

// Bits of |x|, 0 for infinities and NaN: they order like the values.
__device__ __forceinline__ uint32_t finite_abs(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}

// E8M0 byte of the smallest power of two s with amax <= 448 s.  448 = 1.75 2^8:
// s = 2^(E - 8) for amax = m 2^E with m <= 1.75, twice that above.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
  const int b = (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return amax == 0 ? (uint32_t)kScaleOne : (uint32_t)(b < 0 ? 0 : b);
}

// 1 / s, exact: the byte is at most 247.
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// What is rounded to a code: x / s, exact but where it is far below the least
// code; NaN for what is not finite.
__device__ __forceinline__ float scaled(float x, float by) {
  return (__float_as_uint(x) & 0x7fffffffu) < 0x7f800000u ? x * by : __uint_as_float(0x7fc00000u);
}

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

// Eight elements of a row from column c; zeros past its end and for a row that
// is not there.
template <typename T>
__device__ __forceinline__ void load_row8(const T* row, bool there, int64_t c, int64_t cols, T* v) {
  if (there && c + 8 <= cols) {
    load_n<T, 8>(row + c, v);
  } else {
    for (int j = 0; j < 8; ++j) v[j] = from_f32<T>(0.0f);
    if (there)
      for (int j = 0; j < 8; ++j)
        if (c + j < cols) v[j] = row[c + j];
  }
}

// 1 x 128: 16 lanes hold a block, eight elements each, and share its maximum; a
// wave takes four blocks of a row (1 KiB of codes and elements in 16 bits).  A
// workgroup's rows are `rows_per_wg` deep so that the scales, which lie along
// the rows, are written in runs and not byte by byte.  Bound: memory; 8192 x 4096
// bf16 in 24.2 us (4.2 TB/s), 16 x 4096 in 2.7, which is the launch.
template <typename T, int UNROLL>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantArgs a) {
  constexpr int kRows = 4 * UNROLL;  // rows of a workgroup
  __shared__ uint8_t sc[4][kRows];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t id = a.runs ? xcd_run(blockIdx.x, gridDim.x) : blockIdx.x, ct = id % a.col_tiles, r0 = id / a.col_tiles * kRows;
  const int64_t c = ct * 512 + lane * 8, end = (a.cols + 15) / 16 * 16;
  T v[UNROLL][8];
#pragma unroll
  for (int i = 0; i < UNROLL; ++i) {
    const int64_t r = r0 + wave + 4 * i;
    int64_t src = r;
    bool there = r < a.rows;
    if (a.index && there) {
      src = a.index[r];
      there = src >= 0 && src < a.x_rows;
    }
    load_row8<T>((const T*)a.x + src * a.ld, there, c, a.cols, v[i]);
  }
#pragma unroll
  for (int i = 0; i < UNROLL; ++i) {
    const int64_t r = r0 + wave + 4 * i;
    float f[8];
    uint32_t amax = 0;
    for (int j = 0; j < 8; ++j) {
      f[j] = to_f32(v[i][j]);
      amax = max(amax, finite_abs(f[j]));
    }
    const uint32_t byte = scale_byte(max16(amax));
    const float by = inverse_scale(byte);
    for (int j = 0; j < 8; ++j) f[j] = scaled(f[j], by);
    if (r < a.rows && c < end)
      *(uint2*)(a.codes + r * a.ld_codes + c) = make_uint2(codes4(f[0], f[1], f[2], f[3]), codes4(f[4], f[5], f[6], f[7]));
    if ((lane & 15) == 0) sc[lane >> 4][wave + 4 * i] = (uint8_t)byte;
  }
  __syncthreads();
  const int j = threadIdx.x / kRows, i = threadIdx.x % kRows;
  if (j < 4 && r0 + i < a.rows && (ct * 4 + j) * kBlock < a.cols) a.scales[(ct * 4 + j) * a.ld_scales + r0 + i] = sc[j][i];
}

// Eight elements as they lie in memory.  forget(): what was computed from them is
// not kept in registers (widened, a thread's 64 would take two waves' registers).
template <typename T>
struct Raw8 {
  uint32_t w[2 * sizeof(T)];
  __device__ __forceinline__ float operator[](int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
    const uint16_t h = (uint16_t)(w[j / 2] >> (j % 2 * 16));
    return to_f32(__builtin_bit_cast(T, h));
  }
  __device__ __forceinline__ void forget() {
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (sizeof(T) == 2) asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
#endif
  }
};
template <>
__device__ __forceinline__ float Raw8<float>::operator[](int j) const {
  return __uint_as_float(w[j]);
}

// A 128 x 128 tile: row codes as above, and codes of the transpose by way of
// LDS.  WEIGHT: one scale for the tile, else one for each row and, for the
// transpose, for each column.  A thread holds 8 x 8 elements, so that eight
// rows of one column convert straight into eight neighbouring bytes; they go
// to LDS in 8-byte pieces at a place that the column's upper bits permute (the
// 16 lanes of a row write 16 columns eight apart: one bank set without it), and
// leave as whole 128-byte lines.  Bound: memory, one read and two writes: 8192 x
// 4096 bf16 in 28.9 us (4.7 TB/s), a 4100 x 4104 f32 weight in 20 to 21 (5 TB/s).
template <typename T, bool WEIGHT>
__global__ __launch_bounds__(256, (WEIGHT || sizeof(T) == 2 ? 4 : 3)) void quantize_tile_kernel(QuantArgs a) {
  __shared__ uint8_t tile[kBlock * kBlock] __attribute__((aligned(16)));
  __shared__ uint32_t col_max[4][kBlock];
  __shared__ uint8_t row_byte[kBlock], col_byte[kBlock] __attribute__((aligned(16)));
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = tid >> 4, q = tid & 15;
  int64_t t = a.runs ? xcd_run(blockIdx.x, gridDim.x) : blockIdx.x;
  const int64_t cb = t % a.col_tiles;
  t /= a.col_tiles;
  const int64_t rb = t % a.row_tiles, batch = t / a.row_tiles;
  const T* x = (const T*)a.x + batch * a.stride_x;
  uint8_t* codes = a.codes + batch * a.stride_codes;
  uint8_t* scales = a.scales + batch * a.stride_scales;
  uint8_t* codes_t = a.codes_t ? a.codes_t + batch * a.stride_codes_t : nullptr;
  uint8_t* scales_t = a.codes_t ? a.scales_t + batch * a.stride_scales_t : nullptr;

  // The tile's rows; `there`: they have elements (else they are zeros).  The
  // transpose's block is number rb: groups follow each other in whole tiles.
  int64_t r0 = rb * kBlock, n = a.rows - r0;
  bool there = true;
  if (a.offsets) {
    const GroupTile gt = find_group_tile(a.offsets, a.groups, a.rows, kBlock, rb);
    r0 = gt.lo + gt.index * kBlock;
    n = gt.group < 0 ? 0 : gt.hi - r0;
    there = gt.group >= 0 && gt.group < a.groups;
  }
  n = n > kBlock ? kBlock : n;
  const int64_t c0 = cb * kBlock, c = c0 + q * 8, end = (a.cols + 15) / 16 * 16;

  Raw8<T> v[8];
  if (there && n == kBlock && c0 + kBlock <= a.cols && !a.index) {  // all of it: no lane branches
    const T* from = x + (r0 + 8 * g) * a.ld + c;
#pragma unroll
    for (int p = 0; p < 8; ++p, from += a.ld) load_n<T, 8>(from, (T*)v[p].w);
  } else {
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int64_t r = r0 + 8 * g + p;
      bool in = there && 8 * g + p < n;
      int64_t src = r;
      if (a.index && in) {
        src = a.index[r];
        in = src >= 0 && src < a.x_rows;
      }
      T t[8];
      load_row8<T>(x + src * a.ld, in, c, a.cols, t);
      __builtin_memcpy(v[p].w, t, sizeof(t));
    }
  }
  uint32_t cm[8] = {0, 0, 0, 0, 0, 0, 0, 0}, rm[8];
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    rm[p] = 0;
    for (int j = 0; j < 8; ++j) {
      const uint32_t b = finite_abs(v[p][j]);
      rm[p] = max(rm[p], b);
      cm[j] = max(cm[j], b);
    }
    v[p].forget();
  }
  uint32_t one = 0;  // WEIGHT: the tile's byte
  if constexpr (WEIGHT) {
    uint32_t m = 0;
    for (int j = 0; j < 8; ++j) m = max(m, cm[j]);
    m = max16(m);
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    if (lane == 0) col_max[wave][0] = m;
    __syncthreads();
    one = scale_byte(max(max(col_max[0][0], col_max[1][0]), max(col_max[2][0], col_max[3][0])));
  } else {
    for (int j = 0; j < 8; ++j) {
      cm[j] = max(cm[j], (uint32_t)__shfl_xor((int)cm[j], 16));
      cm[j] = max(cm[j], (uint32_t)__shfl_xor((int)cm[j], 32));
    }
    if (lane < 16)
      for (int j = 0; j < 8; ++j) col_max[wave][8 * q + j] = cm[j];
  }
  uint8_t* to = codes + (r0 + 8 * g) * a.ld_codes + c;
#pragma unroll
  for (int p = 0; p < 8; ++p, to += a.ld_codes) {
    const uint32_t byte = WEIGHT ? one : scale_byte(max16(rm[p]));
    const float by = inverse_scale(byte);
    float f[8];
    for (int j = 0; j < 8; ++j) f[j] = scaled(v[p][j], by);
    v[p].forget();
    if (8 * g + p < n && c < end)
      *(uint2*)to = make_uint2(codes4(f[0], f[1], f[2], f[3]), codes4(f[4], f[5], f[6], f[7]));
    if (!WEIGHT && q == 0) row_byte[8 * g + p] = (uint8_t)byte;
    if (p % 2) __builtin_amdgcn_sched_barrier(0);  // two rows at a time: fewer registers
  }
  uint32_t col_bytes[2] = {0, 0};
  if constexpr (!WEIGHT) {
    __syncthreads();
    if (tid < kBlock)
      col_byte[tid] = (uint8_t)scale_byte(max(max(col_max[0][tid], col_max[1][tid]), max(col_max[2][tid], col_max[3][tid])));
    __syncthreads();
    __builtin_memcpy(col_bytes, __builtin_assume_aligned(col_byte + 8 * q, 8), 8);
  }
  if (codes_t) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int k = 8 * q + j;
      const uint32_t byte = WEIGHT ? one : col_bytes[j / 4] >> (j % 4 * 8) & 255u;
      const float by = inverse_scale(byte);
      float f[8];
      for (int p = 0; p < 8; ++p) f[p] = scaled(v[p][j], by);
      *(uint2*)(tile + k * kBlock + ((8 * g) ^ (16 * (q & 7)))) =
          make_uint2(codes4(f[0], f[1], f[2], f[3]), codes4(f[4], f[5], f[6], f[7]));
      if (j % 2) __builtin_amdgcn_sched_barrier(0);
    }
  }
  __syncthreads();
  if constexpr (WEIGHT) {
    if (tid == 0) scales[cb * a.ld_scales + rb] = (uint8_t)one;
    if (codes_t && tid == 0) scales_t[rb * a.ld_scales_t + cb] = (uint8_t)one;
  } else {
    if (tid < n) scales[cb * a.ld_scales + r0 + tid] = row_byte[tid];
  }
  // columns of the transpose: all of a grouped block, else up to the rows' padding
  const int64_t left = a.offsets ? (rb < a.padded ? kBlock : 0) : (a.rows + 15) / 16 * 16 - rb * kBlock;
  if (!codes_t || left <= 0) return;
  if (!WEIGHT && tid < kBlock && c0 + tid < a.cols) scales_t[rb * a.ld_scales_t + c0 + tid] = col_byte[tid];
  for (int k = tid >> 3; k < kBlock; k += 32) {
    const int i = (tid & 7) * 16;
    if (c0 + k < a.cols && i < left)
      *(uint4*)(codes_t + (c0 + k) * a.ld_codes_t + rb * kBlock + i) =
          *(const uint4*)(tile + k * kBlock + (i ^ (16 * ((k >> 3) & 7))));
  }
}

template <typename T>
ws_status run_rows(const QuantArgs& in, hipStream_t stream) {
  QuantArgs a = in;
  a.col_tiles = ceil_div(a.cols, 512);
  // Deep workgroups write their scales in longer runs and load more at a time;
  // shallow ones spread few rows over the CUs (rows x columns below one round
  // of deep ones).
  const bool deep = ceil_div(a.rows, 32) * a.col_tiles >= 1024;
  const int depth = deep ? 32 : 4;
  const auto kernel = deep ? &quantize_rows_kernel<T, 8> : &quantize_rows_kernel<T, 1>;
  const int64_t most = max_workgroups(256) / a.col_tiles * depth;  // rows of one launch: any width has some
  for (int64_t left = a.rows; left > 0; left -= most) {
    a.rows = left < most ? left : most;
    const ws_status s = launch("quantize_rows", kernel, ceil_div(a.rows, depth) * a.col_tiles, 256, 0, stream, a);
    if (s != WS_OK) return s;
    if (a.index) a.index += most;
    else a.x = (const T*)a.x + most * a.ld;
    a.codes += most * a.ld_codes;
    a.scales += most;
  }
  return WS_OK;
}

template <bool WEIGHT>
ws_status run_tiles(const QuantArgs& a, int32_t dtype, int64_t batch, hipStream_t stream) {
  const int64_t grid = a.row_tiles * a.col_tiles;
  if (grid > max_workgroups(256) || grid * batch > max_workgroups(256)) return WS_ERR_INVALID_ARG;
  switch (dtype) {
    case WS_OUT_F32: return launch("quantize_tile", &quantize_tile_kernel<float, WEIGHT>, grid * batch, 256, 0, stream, a);
    case WS_OUT_BF16: return launch("quantize_tile", &quantize_tile_kernel<bf16_t, WEIGHT>, grid * batch, 256, 0, stream, a);
    default: return launch("quantize_tile", &quantize_tile_kernel<f16_t, WEIGHT>, grid * batch, 256, 0, stream, a);
  }
}

QuantArgs base_args(const ws_matrix* x, const int32_t* index, const ws_fp8_matrix* out) {
  QuantArgs a{};
  a.x = x->data;
  a.x_rows = x->rows;
  a.ld = x->ld;
  a.rows = out->rows;
  a.cols = out->cols;
  a.index = index;
  a.codes = (uint8_t*)out->codes;
  a.scales = out->scales;
  a.ld_codes = out->ld;
  a.ld_scales = out->ld_scales;
  // Rows that start inside a cache line share it with the next tile.  Runs of tiles
  // per XCD then merge their parts (4100 x 4104 f32 with transpose: 28.0 us, in turn
  // 30.5); where no line is shared, tiles in turn are better (8192 x 4096: 42.6, runs 45.6).
  a.runs = x->ld * elem_size(x->dtype) % 128 != 0 || out->ld % 128 != 0;
  return a;
}

void set_transposed(QuantArgs* a, const ws_fp8_matrix* t) {
  a->codes_t = (uint8_t*)t->codes;
  a->scales_t = t->scales;
  a->ld_codes_t = t->ld;
  a->ld_scales_t = t->ld_scales;
  a->runs |= t->ld % 128 != 0;
}

// x against a row form of it.
bool rows_fit(const ws_matrix* x, const int32_t* index, const ws_fp8_matrix* out) {
  return valid(x) && valid(out) && x->batch <= 1 && out->batch <= 1 && out->block_rows == 1 && out->cols == x->cols &&
         (index || out->rows == x->rows) && (uintptr_t)index % 4 == 0;
}

}  // namespace
}  // namespace wsg

using namespace wsg;

extern "C" {

int64_t ws_fp8_padded_blocks(int64_t rows, int32_t groups) {
  if (rows < 0 || rows > kMaxDim || groups < 0) return -1;
  return groups == 0 ? ceil_div(rows, kBlock) : group_tiles(rows, groups, kBlock, false);
}

ws_status ws_fp8_quantize_rows(const ws_matrix* x, const int32_t* index, const ws_fp8_matrix* out, hipStream_t stream) {
  if (!rows_fit(x, index, out)) return WS_ERR_INVALID_ARG;
  if (out->rows == 0 || out->cols == 0) return WS_OK;
  const QuantArgs a = base_args(x, index, out);
  switch (x->dtype) {
    case WS_OUT_F32: return run_rows<float>(a, stream);
    case WS_OUT_BF16: return run_rows<bf16_t>(a, stream);
    default: return run_rows<f16_t>(a, stream);
  }
}

ws_status ws_fp8_quantize_both(const ws_matrix* x, const int32_t* index, int32_t groups, const int32_t* offsets,
                               const ws_fp8_matrix* out_rows, const ws_fp8_matrix* out_columns, hipStream_t stream) {
  if (!rows_fit(x, index, out_rows) || !valid(out_columns) || out_columns->batch > 1 || out_columns->block_rows != 1 ||
      out_columns->rows != out_rows->cols || groups < 0 || groups > (1 << 20) || (groups > 0 && (!offsets || (uintptr_t)offsets % 4)))
    return WS_ERR_INVALID_ARG;
  const int64_t padded = ws_fp8_padded_blocks(out_rows->rows, groups);
  if (out_columns->cols != (groups ? padded * kBlock : out_rows->rows)) return WS_ERR_INVALID_ARG;
  if (out_rows->rows == 0 || out_rows->cols == 0) return WS_OK;
  QuantArgs a = base_args(x, index, out_rows);
  set_transposed(&a, out_columns);
  a.offsets = groups ? offsets : nullptr;
  a.groups = groups;
  a.padded = padded;
  a.row_tiles = groups ? group_tiles(a.rows, groups, kBlock, true) : padded;
  a.col_tiles = ceil_div(a.cols, kBlock);
  return run_tiles<false>(a, x->dtype, 1, stream);
}

ws_status ws_fp8_quantize_weight(const ws_matrix* w, const ws_fp8_matrix* out, const ws_fp8_matrix* out_transposed,
                                 hipStream_t stream) {
  if (!valid(w, true) || !valid(out, true) || out->block_rows != kBlock || out->rows != w->rows || out->cols != w->cols ||
      out->batch != w->batch)
    return WS_ERR_INVALID_ARG;
  const ws_fp8_matrix* t = out_transposed;
  if (t && (!valid(t, true) || t->block_rows != kBlock || t->rows != w->cols || t->cols != w->rows || t->batch != w->batch))
    return WS_ERR_INVALID_ARG;
  if (w->rows == 0 || w->cols == 0 || w->batch == 0) return WS_OK;
  QuantArgs a = base_args(w, nullptr, out);
  a.stride_x = w->stride;
  a.stride_codes = out->stride_codes;
  a.stride_scales = out->stride_scales;
  if (t) {
    set_transposed(&a, t);
    a.stride_codes_t = t->stride_codes;
    a.stride_scales_t = t->stride_scales;
  }
  a.row_tiles = ceil_div(a.rows, kBlock);
  a.col_tiles = ceil_div(a.cols, kBlock);
  return run_tiles<true>(a, w->dtype, w->batch, stream);
}

}  // extern "C"
