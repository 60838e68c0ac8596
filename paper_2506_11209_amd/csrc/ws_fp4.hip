// Weights in 4 bits: rounding, widening and products of a few rows (definitions:
// ws_fp4.h).
#include <math.h>

#include <type_traits>

#include "ws_fp4.h"
#include "ws_fp8_common.hpp"

namespace wsg {
namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// 2^(byte - 127); 2^-127 is subnormal, 255 is NaN.
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return __uint_as_float(byte == 0 ? 1u << 22 : byte == 255 ? 0x7fc00000u : byte << 23);
}

// -- rounding and widening -------------------------------------------------------

struct Fp4CastArgs {
  const void* w;
  void* out;
  uint8_t *codes, *scales;
  int64_t rows, cols, ld_w, ld, ld_scales, stride_w, stride_codes, stride_scales;
  int64_t tiles, down, across;  // of all matrices; of a matrix
};

template <typename T>
__device__ __forceinline__ void load8(const T* row, int64_t c, int64_t cols, float (&v)[8]) {
  if (c + 8 <= cols) {
    T t[8];
    if constexpr (sizeof(T) == 4) {
      load_n<T, 4>(row + c, t);
      load_n<T, 4>(row + c + 4, t + 4);
    } else {
      load_n<T, 8>(row + c, t);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_f32(t[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? to_f32(row[c + j]) : 0.0f;
  }
}

// A wave's tile: lane l has row l % 16, and of every 32 columns the 8 from 8 (l / 16).
struct CastTile {
  int64_t matrix, i, j;
  bool there;
};
__device__ __forceinline__ CastTile cast_tile(const Fp4CastArgs& a) {
  // of the wave: divided as scalars
  const int64_t t = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), plane = a.down * a.across;
  return CastTile{t / plane, t % plane / a.across, t % a.across, t < a.tiles};
}

// Bound: memory (16 of 4096 x 2048 of bf16 into the same codes 75 us, 4.5 TB/s; two tiles a
// wave 79, four 101).
template <typename T>
__global__ __launch_bounds__(256) void fp4_quantize_kernel(Fp4CastArgs a) {
  const CastTile t = cast_tile(a);
  if (!t.there) return;  // whole waves
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int64_t b = t.j, row_at = 16 * t.i + r;
  const T* row = (const T*)a.w + t.matrix * a.stride_w + row_at * a.ld_w;
  const int64_t cols = row_at < a.rows ? a.cols : 0;  // rows of padding are zeros
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) load8<T>(row, 128 * b + 32 * i + 8 * g, cols, v[i]);
  uint32_t code[4], scale = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t amax = 0;  // of the magnitudes' bits, which are in their order; NaN above infinity
#pragma unroll
    for (int j = 0; j < 8; ++j) amax = max(amax, __float_as_uint(v[i][j]) & 0x7fffffffu);
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 16));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 32));
    // amax = f 2^e, 1 <= f < 2: 2^(e - 2) where f <= 1.5, else 2^(e - 1)
    const int e = (int)(amax >> 23) - ((amax & 0x7fffffu) <= 0x400000u ? 2 : 1);
    const int byte = amax >= 0x7f800000u ? 255 : amax == 0 ? kScaleOne : min(max(e, 0), 252);
    scale |= (uint32_t)byte << (8 * i);
    uint32_t c = 0;
    if (byte != 255) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = ldexpf(v[i][j], kScaleOne - byte);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[0], y[1], 1.0f, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], 1.0f, 1);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], 1.0f, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], 1.0f, 3);
    }
    code[i] = c;
  }
  *(i32x4_t*)(a.codes + t.matrix * a.stride_codes + t.i * a.ld + 1024 * b + 16 * lane) =
      i32x4_t{(int)code[0], (int)code[1], (int)code[2], (int)code[3]};
  if (g == 0) *(uint32_t*)(a.scales + t.matrix * a.stride_scales + t.i * a.ld_scales + 64 * b + 4 * r) = scale;
}

// Eight codes of a dword times a scale, exactly.
__device__ __forceinline__ bf16x8_t widen_bf16(uint32_t c, float scale) {
  const bf16x2_t p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
  const bf16x2_t r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2), s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
  return bf16x8_t{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
__device__ __forceinline__ f16x8_t widen_f16(uint32_t c) {
  const f16x2_t p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 0), q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 1);
  const f16x2_t r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 2), s = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, 1.0f, 3);
  return f16x8_t{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}

// As fp4_quantize_kernel, the other way.  T: float or bf16_t.
template <typename T>
__global__ __launch_bounds__(256) void fp4_dequantize_kernel(Fp4CastArgs a) {
  const CastTile t = cast_tile(a);
  if (!t.there) return;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int64_t b = t.j, row_at = 16 * t.i + r;
  const i32x4_t code = *(const i32x4_t*)(a.codes + t.matrix * a.stride_codes + t.i * a.ld + 1024 * b + 16 * lane);
  const uint32_t scale = *(const uint32_t*)(a.scales + t.matrix * a.stride_scales + t.i * a.ld_scales + 64 * b + 4 * r);
  if (row_at >= a.rows) return;
  T* row = (T*)a.out + t.matrix * a.stride_w + row_at * a.ld_w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float by = scale_value(scale >> (8 * i) & 255u);
    const f16x8_t h = widen_f16((uint32_t)code[i]);
    const int64_t c = 128 * b + 32 * i + 8 * g;
    T v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = from_f32<T>((float)h[j] * by);
    if (c + 8 <= a.cols) {
      if constexpr (sizeof(T) == 4) {
        store_n<T, 4>(row + c, v);
        store_n<T, 4>(row + c + 4, v + 4);
      } else {
        store_n<T, 8>(row + c, v);
      }
    } else {
      for (int j = 0; j < 8; ++j)
        if (c + j < a.cols) row[c + j] = v[j];
    }
  }
}

struct Fp4ScaleArgs {
  const uint8_t* scales;
  uint8_t* out;
  int64_t rows, across, cols, ld_scales, stride_scales, ld, stride;  // cols: of out
  int64_t down, fours, all;  // of a matrix; of a row of tiles; of them all
};

// A wave takes four tiles next to each other: lane l the scales of row l % 16 in the
// l / 16-th of them.
__global__ __launch_bounds__(256) void fp4_scales_kernel(Fp4ScaleArgs a) {
  const int64_t t = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t >= a.all) return;
  const int lane = threadIdx.x & 63;
  const int64_t line = t / a.fours, m = line / a.down, i = line % a.down, b = t % a.fours * 4 + lane / 16, r = 16 * i + lane % 16;
  if (b >= a.across || r >= a.rows) return;
  const uint32_t s = *(const uint32_t*)(a.scales + m * a.stride_scales + i * a.ld_scales + 64 * b + lane % 16 * 4);
  uint8_t* to = a.out + m * a.stride + r * a.ld + 4 * b;
  if (4 * b + 4 <= a.cols) {
    __builtin_memcpy(to, &s, 4);
  } else {
    for (int k = 0; 4 * b + k < a.cols; ++k) to[k] = (uint8_t)(s >> (8 * k));
  }
}

// -- products --------------------------------------------------------------------

struct Fp4Args {
  const void* x;
  const uint8_t *codes, *scales;
  void* C;
  const int32_t *index, *offsets;
  int64_t ldx, ld, ld_scales, stride_codes, stride_scales, ldc;
  uint8_t* arranged;  // A by operands (fp4_arrange_kernel), or null
  int64_t M, x_rows, N, K;
  int64_t tiles_m, strips;
  int32_t groups, dtype;
};

__device__ __forceinline__ f32x4_t multiply(bf16x8_t x, bf16x8_t w, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t multiply(f16x8_t x, f16x8_t w, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w, c, 0, 0, 0);
}

// Eight of a row's columns from k, zeros past its end.
template <typename T>
__device__ __forceinline__ i32x4_t load_end(const T* row, int k, int K) {
  T t[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) t[j] = k + j < K ? row[k + j] : from_f32<T>(0.0f);
  i32x4_t v;
  __builtin_memcpy(&v, t, 16);
  return v;
}

template <typename T>
__device__ __forceinline__ void store_value(void* C, int64_t at, float v) {
  ((T*)C)[at] = from_f32<T>(v);
}

// The rows of one tile of 16 MT rows.
struct RowTile {
  int64_t m0, m_end;
  int group;  // -1: there is no such tile; `groups` and more: rows of no group
};
template <int MT, bool GROUPED>
__device__ __forceinline__ RowTile row_tile(const Fp4Args& a, int64_t tm) {
  if constexpr (GROUPED) {
    const GroupTile gt = find_group_tile(a.offsets, a.groups, a.M, 16 * MT, tm);
    return RowTile{gt.lo + gt.index * 16 * MT, gt.hi, gt.group};
  }
  return RowTile{tm * 16 * MT, a.M, 0};
}

// A by operands of the matrix instruction: for 16 rows and 128 columns 4 KiB, lane l's 16
// bytes of the k-th quarter at 1024 k + 16 l.  A wave's load of it is one piece; of A itself
// it is 64 bytes each of 16 rows (choose() has what both take).  Zeros past the last column
// and for rows that are not there.  Bound: latency, one trip to memory and back.
template <typename X, int MT, bool GROUPED>
__global__ __launch_bounds__(256) void fp4_arrange_kernel(Fp4Args a) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int blocks = (int)((a.K + 127) / 128), per = (blocks + 3) / 4;  // a workgroup has four blocks of a tile
  const int64_t tm = blockIdx.x / per;
  const int b = blockIdx.x % per * 4 + (threadIdx.x >> 6);
  const RowTile t = row_tile<MT, GROUPED>(a, tm);
  if (b >= blocks || t.group < 0 || (GROUPED && t.group >= a.groups)) return;
  const int K = (int)a.K - 8 * g;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = t.m0 + 16 * i + r;
    int64_t from = m < t.m_end ? (a.index ? a.index[m] : m) : -1;
    if (from >= a.x_rows) from = -1;
    const X* x = (const X*)a.x + (from < 0 ? 0 : from) * a.ldx + 8 * g;
    uint8_t* to = a.arranged + ((tm * MT + i) * (int64_t)blocks + b) * 4096 + 16 * lane;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int k = 128 * b + 32 * q;
      i32x4_t v = {0, 0, 0, 0};
      if (from >= 0) {
        if (k + 8 <= K) load_n<X, 8>(x + k, (X*)&v);
        else v = load_end(x, k, K);
      }
      *(i32x4_t*)(to + 1024 * q) = v;
    }
  }
}

// A workgroup computes 16 MT rows of 16 NT columns: its waves share out the contraction,
// 256 columns of A at a time, and add up their parts through LDS in a fixed order.
// Operands go from memory straight to registers, a step's weights before the products of
// the one before.  Rows that are not there read those of another and are not stored.
// Bound: reading the weights (1 x 8192 x 8192: 8.6 us, 4.2 TB/s; by rows of codes instead
// of tiles, 64 bytes of 16 rows a load and scales 4 bytes of each, 14.1; 128 rows in 53 to 56 of
// 64 groups of 4096 x 2048 43 to 55 us, by rows of codes 83); from about 16 rows on by this
// split, in which A is read once for every 32 columns (256 x 4096 x 4096: 24 us, 1024 x 8192 x
// 8192: 205, 0.67 PFLOP/s).
// (Of 64 rows with the registers of four waves; of fewer with those of eight, and so more
// workgroups a CU.)
template <typename X, int MT, int NT, bool GROUPED, bool ARRANGED>
__global__ __launch_bounds__(MT > 2 ? 256 : 512) void fp4_product_kernel(Fp4Args a) {
  constexpr bool kBf16 = std::is_same<X, bf16_t>::value;
  extern __shared__ __align__(16) f32x4_t part[];  // waves x MT x NT x 64
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
  const int waves = blockDim.x >> 6;
  // Strips of columns go round the XCDs, all of a tile of rows before the next, whose rows
  // stay in the L2: they are more bytes than a strip's codes.  All tiles of a strip before
  // the next strip instead: 2048 x 2048 x 2048 84 us for 42, 1024 x 8192 x 8192 337 for 205,
  // 2048 rows of 64 groups of 4096 x 2048 266 for 133, 128 rows 60 for 56.
  const uint32_t turn = ((uint32_t)a.strips + 7) / 8 * 8, strip = blockIdx.x % turn, tm = blockIdx.x / turn;
  if (strip >= a.strips) return;
  const RowTile rows = row_tile<MT, GROUPED>(a, tm);
  if (rows.group < 0) return;
  const int64_t m0 = rows.m0, m_end = rows.m_end;
  const bool zero = a.x_rows == 0 || (GROUPED && rows.group >= a.groups);
  const uint8_t *codes = a.codes, *scales = a.scales;
  if (GROUPED && !zero) {
    codes += rows.group * a.stride_codes;
    scales += rows.group * a.stride_scales;
  }
  const int64_t n0 = (int64_t)strip * 16 * NT;
  const X* x[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    if constexpr (ARRANGED) {
      x[i] = (const X*)(a.arranged + ((int64_t)tm * MT + i) * ((a.K + 127) / 128) * 4096 + 16 * lane);
    } else {
      int64_t from = min(m0 + 16 * i + r, m_end - 1);
      if (a.index) from = a.index[from];
      x[i] = (const X*)a.x + (from >= 0 && from < a.x_rows ? from : 0) * a.ldx + 8 * g;
    }
  }
  const uint8_t *code_at[NT], *scale_at[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t tile = min(n0 / 16 + t, (a.N - 1) / 16);  // past the last column: computed and not stored
    code_at[t] = codes + tile * a.ld + 16 * lane;
    scale_at[t] = scales + tile * a.ld_scales + 4 * r;
  }
  f32x4_t acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[i][t] = f32x4_t{0, 0, 0, 0};
  const int blocks = zero ? 0 : (int)((a.K + 127) / 128), K = (int)a.K;
  const auto load_codes = [&](int b0, i32x4_t (&code)[2][NT], uint32_t (&scale)[2][NT]) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int b = min(b0 + u, blocks - 1);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        code[u][t] = *(const i32x4_t*)(code_at[t] + 1024 * (int64_t)b);
        scale[u][t] = *(const uint32_t*)(scale_at[t] + 64 * (int64_t)b);
      }
    }
  };
  const auto load_x = [&](int b, i32x4_t (&xv)[4][MT]) {
    if constexpr (ARRANGED) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < MT; ++i) xv[q][i] = *(const i32x4_t*)(x[i] + 2048 * (int64_t)b + 512 * q);
    } else if (128 * b + 128 <= K) {  // the same for the wave
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < MT; ++i) load_n<X, 8>(x[i] + 128 * b + 32 * q, (X*)&xv[q][i]);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < MT; ++i) xv[q][i] = load_end(x[i], 128 * b + 32 * q, K - 8 * g);
    }
  };
  const auto multiply_block = [&](const i32x4_t (&code)[NT], const uint32_t (&scale)[NT], const i32x4_t (&xv)[4][MT]) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float by = scale_value(scale[t] >> (8 * q) & 255u);
        if constexpr (kBf16) {
          const bf16x8_t w = widen_bf16((uint32_t)code[t][q], by);
#pragma unroll
          for (int i = 0; i < MT; ++i) acc[i][t] = multiply(__builtin_bit_cast(bf16x8_t, xv[q][i]), w, acc[i][t]);
        } else {  // binary16 does not reach as far as scales do: they are applied to the sums
          const f16x8_t w = widen_f16((uint32_t)code[t][q]);
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            const f32x4_t p = multiply(__builtin_bit_cast(f16x8_t, xv[q][i]), w, f32x4_t{0, 0, 0, 0});
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][t][j] = fmaf(by, p[j], acc[i][t][j]);
          }
        }
      }
  };
  int b0 = 2 * wave;
  if (b0 < blocks) {
    i32x4_t code[2][NT], next_code[2][NT], xv[2][4][MT];
    uint32_t scale[2][NT], next_scale[2][NT];
    load_codes(b0, next_code, next_scale);
    for (; b0 < blocks; b0 += 2 * waves) {
      load_x(b0, xv[0]);
      if (b0 + 1 < blocks) load_x(b0 + 1, xv[1]);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          code[u][t] = next_code[u][t];
          scale[u][t] = next_scale[u][t];
        }
      load_codes(b0 + 2 * waves, next_code, next_scale);
      multiply_block(code[0], scale[0], xv[0]);
      if (b0 + 1 < blocks) multiply_block(code[1], scale[1], xv[1]);
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) part[((wave * MT + i) * NT + t) * 64 + lane] = acc[i][t];
  __syncthreads();
  // lane l of a piece: rows 4 (l / 16) .., column l % 16
  for (int j = tid; j < MT * NT * 64; j += blockDim.x) {
    f32x4_t sum = part[j];
    for (int w = 1; w < waves; ++w) sum += part[w * MT * NT * 64 + j];
    const int64_t m = m0 + j / (NT * 64) * 16 + (j & 63) / 16 * 4, n = n0 + j / 64 % NT * 16 + (j & 15);
    if (n >= a.N) continue;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (m + k >= m_end) break;
      if (a.index) {
        const int32_t from = a.index[m + k];
        if (from < 0 || from >= a.x_rows) sum[k] = 0.0f;
      }
      const int64_t at = (m + k) * a.ldc + n;
      switch (a.dtype) {  // the same for the whole launch
        case WS_OUT_F32: store_value<float>(a.C, at, sum[k]); break;
        case WS_OUT_BF16: store_value<bf16_t>(a.C, at, sum[k]); break;
        default: store_value<f16_t>(a.C, at, sum[k]);
      }
    }
  }
}

// -- host ---------------------------------------------------------------------

bool valid_fp4(const ws_fp4_matrix* q, bool batched) {
  if (!q || q->rows < 0 || q->cols < 0 || q->rows > kMaxDim || q->cols > kMaxDim || q->batch < 0) return false;
  const int64_t across = ceil_div(q->cols, 128), down = ceil_div(q->rows, 16);
  if (q->ld % 16 || q->ld < 1024 * across || q->ld > kMaxDim || q->ld_scales % 4 || q->ld_scales < 64 * across || q->ld_scales > kMaxDim)
    return false;
  if (q->rows == 0 || q->cols == 0 || (batched && q->batch == 0)) return true;
  if (q->batch > 1 && (q->stride_codes % 16 || q->stride_scales % 4 || q->stride_codes < (down - 1) * q->ld + 1024 * across ||
                       q->stride_scales < (down - 1) * q->ld_scales + 64 * across))
    return false;
  return q->codes && (uintptr_t)q->codes % 16 == 0 && q->scales && (uintptr_t)q->scales % 4 == 0;
}

ws_status cast(const char* what, const ws_matrix* w, const ws_fp4_matrix* q, bool out, hipStream_t stream) {
  if (!valid(w, true) || !valid_fp4(q, true) || w->rows != q->rows || w->cols != q->cols) return WS_ERR_INVALID_ARG;
  if (w->batch != q->batch) return WS_ERR_INVALID_ARG;
  if (!out && w->dtype == WS_OUT_F16) return WS_ERR_INVALID_ARG;  // values of 2^17 and more
  if (w->rows == 0 || w->cols == 0 || w->batch == 0) return WS_OK;
  Fp4CastArgs a{};
  a.w = w->data;
  a.out = w->data;
  a.codes = (uint8_t*)q->codes;
  a.scales = q->scales;
  a.rows = w->rows;
  a.cols = w->cols;
  a.ld_w = w->ld;
  a.stride_w = w->stride;
  a.ld = q->ld;
  a.ld_scales = q->ld_scales;
  a.stride_codes = q->stride_codes;
  a.stride_scales = q->stride_scales;
  a.across = ceil_div(w->cols, 128);
  a.down = ceil_div(w->rows, 16);
  a.tiles = a.across * a.down * w->batch;
  const int64_t grid = ceil_div(a.tiles, 4);
  if (grid > max_workgroups(256)) return WS_ERR_INVALID_ARG;
  if (out)
    return launch(what, w->dtype == WS_OUT_F32 ? &fp4_quantize_kernel<float> : w->dtype == WS_OUT_BF16 ? &fp4_quantize_kernel<bf16_t>
                                                                                                          : &fp4_quantize_kernel<f16_t>,
                  grid, 256, 0, stream, a);
  return launch(what, w->dtype == WS_OUT_F32 ? &fp4_dequantize_kernel<float> : &fp4_dequantize_kernel<bf16_t>, grid, 256, 0, stream, a);
}

template <typename X, int MT, int NT, bool GROUPED>
ws_status launch_product(const char* what, int waves, hipStream_t stream, Fp4Args a) {
  a.strips = ceil_div(a.N, 16 * NT);
  a.tiles_m = GROUPED ? group_tiles(a.M, a.groups, 16 * MT, true) : ceil_div(a.M, 16 * MT);
  while (waves > 1 && waves * 128 >= a.K) waves /= 2;  // of 256 columns each
  const int64_t grid = ceil_div(a.strips, 8) * 8 * a.tiles_m, lds = waves * MT * NT * 1024;
  if (grid > max_workgroups(64 * waves) || a.tiles_m > 1 << 28) return WS_ERR_INVALID_ARG;
  if constexpr (MT > 1)
    if (a.arranged) {
      const int64_t first = a.tiles_m * ceil_div(ceil_div(a.K, 128), 4);
      if (first > max_workgroups(256)) return WS_ERR_INVALID_ARG;
      const ws_status s = launch(what, &fp4_arrange_kernel<X, MT, GROUPED>, first, 256, 0, stream, a);
      return s != WS_OK ? s : launch(what, &fp4_product_kernel<X, MT, NT, GROUPED, true>, grid, 64 * waves, lds, stream, a);
    }
  return launch(what, &fp4_product_kernel<X, MT, NT, GROUPED, false>, grid, 64 * waves, lds, stream, a);
}

// Rows of a group on average, and what follows from them.
struct Choice {
  int mt;         // tiles of 16 rows a workgroup has
  bool many;      // strips, of 16 rows
  int64_t bytes;  // of A by operands, 0 where it is read as it lies
};
// Of 16 rows, workgroups of 2 tiles' columns and eight waves where there are few strips, of
// 4 and four waves where there are many and starting waves costs more than it hides.  us so
// and so, by strips of 32 columns: 256 (1 x 8192 x 8192) 11.2 and 14.7, of 16 rows 14.5 and 16.5;
// 384 (12288 x 4096) 11.0 and 10.4, 14.6 and 11.5; 512 (16384 x 4096) 10.8 and 11.1, 14.7 and
// 12.4; 768 14.4 and 15.5, 19.9 and 18.8; 1024 17.4 and 17.1, 24.8 and 20.1; 2048 29.6 and
// 28.6, 44.3 and 34.4; 128 rows of 57 of 64 groups of 4096 x 2048 92 and 53.  More rows have
// many strips, and four waves.
// Rows of a group on average: one full group among empty ones runs in tiles of 16 rows too
// (256 rows in one of 64 of 4096 x 2048 24.8 us, in a matrix by itself 17.9, in all of them 58;
// 1024 rows 60.6, 44.1 and 73.1).
// A workgroup takes fewer rows where the launch has under three workgroups a CU.  us of all
// 64 (or 32) rows in one and so: 40 x 4104 x 4100 17.0 and 11.5, 64 x 4096 x 4096 15.5 and
// 10.2, 64 x 100 x 8192 22.3 and 11.5, 256 x 2048 x 2048 13.1 and 9.5; of two a CU
// 512 x 2048 x 2048 18.1 and 16.4, but 64 x 8192 x 8192 23.4 and 26.7.
// A by operands takes a launch more, about 4 us of the host's, and pays from 2^15 blocks of
// 16 rows and 128 columns on.  us from A and by operands: 512 x 2048 x 2048 21.5 and 18.0,
// 256 x 4096 x 4096 38 and 25, 2048 x 2048 x 2048 73 and 42; below, 512 x 1024 x 1024 9.2 and
// 13.1, 256 x 2048 x 2048 13.0 and 13.6.
Choice choose(int64_t M, int64_t N, int64_t K, int64_t groups) {
  const int64_t rows = groups > 0 ? ceil_div(M, groups) : M;
  Choice c{};
  c.mt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  const auto count = [&] { return groups > 0 ? group_tiles(M, groups, 16 * c.mt, false) : ceil_div(M, 16 * c.mt); };
  while (c.mt > 1 && ceil_div(N, 32) * count() < 768) c.mt /= 2;
  const int64_t tiles = count();
  const int64_t strips = ceil_div(N, 32) * tiles, blocks = c.mt * ceil_div(K, 128);  // blocks: a workgroup's
  c.many = strips > 500;
  if (c.mt > 1 && groups != 0 && blocks > 0 && strips >= ceil_div(1 << 15, blocks))
    c.bytes = (groups >= 0 ? group_tiles(M, groups, 16 * c.mt, true) : tiles) * blocks * 4096;
  return c;
}

template <typename X, bool GROUPED>
ws_status launch_product(const char* what, const Choice& c, hipStream_t stream, const Fp4Args& a) {
  if (c.mt == 1)
    return c.many ? launch_product<X, 1, 4, GROUPED>(what, 4, stream, a) : launch_product<X, 1, 2, GROUPED>(what, 8, stream, a);
  if (c.mt == 2) return launch_product<X, 2, 2, GROUPED>(what, 4, stream, a);
  return launch_product<X, 4, 2, GROUPED>(what, 4, stream, a);
}

ws_status product(const char* what, const ws_matrix* A, const int32_t* index, const ws_fp4_matrix* B, int32_t groups,
                  const int32_t* offsets, const ws_matrix* C, void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  const bool grouped = groups >= 0;
  if (!valid(A) || A->batch > 1 || !valid(C) || C->batch > 1 || !valid_fp4(B, grouped)) return WS_ERR_INVALID_ARG;
  if (A->dtype == WS_OUT_F32 || A->cols != B->cols || C->cols != B->rows || (!index && A->rows != C->rows) || (uintptr_t)index % 4)
    return WS_ERR_INVALID_ARG;
  if (grouped ? B->batch != groups || groups > 1 << 20 || !offsets || (uintptr_t)offsets % 4 : B->batch > 1) return WS_ERR_INVALID_ARG;
  if (C->rows == 0 || C->cols == 0) return WS_OK;
  const Choice c = choose(C->rows, C->cols, A->cols, groups);
  if (workspace_bytes < c.bytes || (c.bytes > 0 && (!workspace || (uintptr_t)workspace % 16))) return WS_ERR_INVALID_ARG;
  Fp4Args a{};
  a.arranged = c.bytes > 0 ? (uint8_t*)workspace : nullptr;
  a.x = A->data;
  a.codes = (const uint8_t*)B->codes;
  a.scales = B->scales;
  a.C = C->data;
  a.index = index;
  a.offsets = offsets;
  a.ldx = A->ld;
  a.ld = B->ld;
  a.ld_scales = B->ld_scales;
  a.stride_codes = B->stride_codes;
  a.stride_scales = B->stride_scales;
  a.ldc = C->ld;
  a.M = C->rows;
  a.x_rows = A->rows;
  a.N = C->cols;
  a.K = A->cols;
  a.groups = groups;
  a.dtype = C->dtype;
  if (A->dtype == WS_OUT_BF16)
    return grouped ? launch_product<bf16_t, true>(what, c, stream, a) : launch_product<bf16_t, false>(what, c, stream, a);
  return grouped ? launch_product<f16_t, true>(what, c, stream, a) : launch_product<f16_t, false>(what, c, stream, a);
}

}  // namespace
}  // namespace wsg

using namespace wsg;

extern "C" {

ws_status ws_fp4_quantize(const ws_matrix* w, const ws_fp4_matrix* out, hipStream_t stream) {
  return cast("fp4_quantize", w, out, true, stream);
}

ws_status ws_fp4_dequantize(const ws_fp4_matrix* q, const ws_matrix* out, hipStream_t stream) {
  return cast("fp4_dequantize", out, q, false, stream);
}

ws_status ws_fp4_scales(const ws_fp4_matrix* q, uint8_t* out, int64_t ld, int64_t stride, hipStream_t stream) {
  if (!valid_fp4(q, true) || ld < ceil_div(q->cols, WS_FP4_BLOCK) || ld > kMaxDim) return WS_ERR_INVALID_ARG;
  if (q->rows == 0 || q->cols == 0 || q->batch == 0) return WS_OK;
  Fp4ScaleArgs a{};
  a.cols = ceil_div(q->cols, WS_FP4_BLOCK);
  if (!out || (q->batch > 1 && stride < (q->rows - 1) * ld + a.cols)) return WS_ERR_INVALID_ARG;
  a.scales = q->scales;
  a.out = out;
  a.rows = q->rows;
  a.across = ceil_div(q->cols, 128);
  a.ld_scales = q->ld_scales;
  a.stride_scales = q->stride_scales;
  a.ld = ld;
  a.stride = stride;
  a.down = ceil_div(q->rows, 16);
  a.fours = ceil_div(a.across, 4);
  a.all = a.fours * a.down * q->batch;
  const int64_t grid = ceil_div(a.all, 4);
  if (grid > max_workgroups(256)) return WS_ERR_INVALID_ARG;
  return launch("fp4_scales", &fp4_scales_kernel, grid, 256, 0, stream, a);
}

int64_t ws_fp4_product_workspace(int64_t M, int64_t N, int64_t K, int32_t groups) {
  if (M < 0 || N < 0 || K < 0 || M > kMaxDim || N > kMaxDim || K > kMaxDim || groups < -1 || groups > 1 << 20) return -1;
  return M == 0 || N == 0 ? 0 : choose(M, N, K, groups).bytes;
}

ws_status ws_fp4_product(const ws_matrix* A, const int32_t* index, const ws_fp4_matrix* B, const ws_matrix* C, void* workspace,
                         int64_t workspace_bytes, hipStream_t stream) {
  return product("fp4_product", A, index, B, -1, nullptr, C, workspace, workspace_bytes, stream);
}

ws_status ws_fp4_grouped_product(const ws_matrix* A, const int32_t* index, const ws_fp4_matrix* B, int32_t groups,
                                 const int32_t* offsets, const ws_matrix* C, void* workspace, int64_t workspace_bytes,
                                 hipStream_t stream) {
  if (groups < 0) return WS_ERR_INVALID_ARG;
  return product("fp4_grouped_product", A, index, B, groups, offsets, C, workspace, workspace_bytes, stream);
}

}  // extern "C"
