// Orthogonalised updates of matrices with a short side, n <= 64 (definitions:
// ws_orthogonal.h).
//
// Every step multiplies X with a polynomial of A = X X^T, so all of them together
// multiply the first X with one n x n matrix Q: with T = a + b A + c A^2, Q <- T Q and
// A <- T A T.  Three launches whatever the number of steps: A_0 = G G^T over parts of the
// long side, the iteration by one workgroup in LDS, and Q G.  All in binary32: an error
// of A in a direction grows as A itself does there, 12 times a step, so that directions
// of singular value s (of G / |G|) come out within about 2^-23 / s^2, where products in
// binary16 would leave them 2^-10 / s^2.  A is not made from X again, and so parts from
// it a little more with every step: more than kFewSteps run in tiles.
//
// Sums: a part of G with very large or small values is scaled by a power of two of its
// own, so that squares neither overflow nor vanish.
#include <math.h>

#include "ws_fp8_common.hpp"
#include "ws_orthogonal.hpp"

namespace wsg {
namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;

struct FewArgs {
  const void* G;
  uint16_t* out;
  int64_t ld, stride, ld_out, stride_out;
  int32_t n, m, tall, steps;  // tall: rows of G are the long side
  int32_t parts, each;        // of the long side, a multiple of 16
  float* sums;                // batch x parts x tiles x 64 x 4: lower triangle of G G^T
  int32_t* scales;            // batch x parts: their values are those of G times 2^-scale; kNotFinite
  float* Q;                   // batch x (16 NT)^2, by 1 / sqrt(trace)
  int32_t* scale;             // batch: the scale of Q G
};
constexpr int kNotFinite = 1 << 20;

constexpr int lower_tiles(int nt) { return nt * (nt + 1) / 2; }
// Tile t of the lower triangle, row after row.
__device__ __forceinline__ void tile_at(int t, int* ti, int* tj) {
  int i = 0;
  while ((i + 1) * (i + 2) / 2 <= t) ++i;
  *ti = i;
  *tj = t - i * (i + 1) / 2;
}

// G's element of the short side's row and the long side's column.
template <typename T>
__device__ __forceinline__ float at(const T* G, const FewArgs& a, int row, int col) {
  return row < a.n && col < a.m ? to_f32(a.tall ? G[col * a.ld + row] : G[row * a.ld + col]) : 0.0f;
}

// Four neighbours of the long side.
template <typename T>
__device__ __forceinline__ f32x4_t four(const T* G, const FewArgs& a, int row, int col) {
  f32x4_t v;
  if (!a.tall && row < a.n && col + 4 <= a.m) {
    T t[4];
    load_n<T, 4>(G + row * a.ld + col, t);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = to_f32(t[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = at(G, a, row, col + i);
  }
  return v;
}

__device__ __forceinline__ f32x4_t multiply(float x, float y, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(x, y, c, 0, 0, 0); }

constexpr int kGramWaves = 4;

// A part's share of G G^T: wave w takes every fourth 16 columns of the part, all tiles
// of the lower triangle; their sums add up in turn in LDS.
template <typename T, int NT>
__global__ __launch_bounds__(64 * kGramWaves) void few_gram_kernel(FewArgs a) {
  constexpr int kTiles = lower_tiles(NT);
  __shared__ f32x4_t sums[kTiles * 64];
  __shared__ uint32_t top[kGramWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4;
  const int64_t matrix = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts, lo = part * a.each, hi = min(lo + a.each, a.m);
  const T* G = (const T*)a.G + matrix * a.stride;
  f32x4_t acc[kTiles];
  uint32_t most = 0;  // magnitudes' bits are in their order; NaN above infinity
  // All of the part with values times 2^-scale; a step's loads go out before the one
  // before it is multiplied.  Parts are whole 16s, but for the last one's end.
  const auto add_up = [&](int scale) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) acc[t] = f32x4_t{0, 0, 0, 0};
    f32x4_t f[NT], next[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) next[t] = four(G, a, 16 * t + r, lo + 16 * wave + 4 * g);
    for (int k0 = lo + 16 * wave; k0 < hi; k0 += 16 * kGramWaves) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        f[t] = next[t];
        next[t] = four(G, a, 16 * t + r, min(k0 + 16 * kGramWaves, a.m) + 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          most = max(most, __float_as_uint(f[t][i]) & 0x7fffffffu);
          f[t][i] = ldexpf(f[t][i], -scale);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j <= i; ++j) acc[i * (i + 1) / 2 + j] = multiply(f[i][k], f[j][k], acc[i * (i + 1) / 2 + j]);
    }
  };
  add_up(0);
  for (int d = 32; d; d /= 2) most = max(most, (uint32_t)__shfl_xor((int)most, d));
  if (lane == 0) top[wave] = most;
  __syncthreads();
  for (int w = 0; w < kGramWaves; ++w) most = max(most, top[w]);
  // Gradients between 2^-40 and 2^40 at the largest need no scale.
  int scale = 0;
  if (most >= 0x7f800000u) scale = kNotFinite;
  else if (most == 0) scale = -kNotFinite;
  else if (most < (87u << 23) || most >= (167u << 23)) {
    scale = ilogbf(__uint_as_float(most));
    add_up(scale);
  }
  if (tid == 0) a.scales[blockIdx.x] = scale;
  for (int w = 0; w < kGramWaves; ++w) {
    if (wave == w)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) sums[t * 64 + lane] = w ? sums[t * 64 + lane] + acc[t] : acc[t];
    __syncthreads();
  }
  f32x4_t* to = (f32x4_t*)a.sums + (int64_t)blockIdx.x * kTiles * 64;
  for (int i = tid; i < kTiles * 64; i += 64 * kGramWaves) to[i] = sums[i];
}

template <int NT>
struct FewShape {
  static constexpr int kWaves = lower_tiles(NT);  // a tile each
  static constexpr int kSide = 16 * NT, kPitch = kSide + 4;  // floats: rows spread over the banks
};

// One workgroup's iteration.  Matrices are symmetric (polynomials of A_0): a wave has a
// tile of the lower triangle and writes it to both its places in a matrix in LDS.  Bound:
// latency, of the way to memory and of three products in a row a step (T Q beside T A)
// with the meetings between them (n = 16: 6.4 us, n = 32: 8.3, n = 64, where it is the
// products themselves on one CU: 19).
template <int NT>
__global__ __launch_bounds__(64 * FewShape<NT>::kWaves) void few_iterate_kernel(FewArgs a) {
  typedef FewShape<NT> S;
  __shared__ __align__(16) float L[S::kSide * S::kPitch], R[S::kSide * S::kPitch], Z[S::kSide * S::kPitch];
  __shared__ float trace;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
  const int64_t matrix = blockIdx.x;
  int ti, tj;
  tile_at(wave, &ti, &tj);
  const int row = 16 * ti + 4 * g, col = 16 * tj + r;  // the lane's: rows row .. row + 3
  const auto put = [&](float* to, const f32x4_t& v) {
#pragma unroll
    for (int k = 0; k < 4; ++k) to[(row + k) * S::kPitch + col] = v[k];
    if (ti != tj) *(f32x4_t*)(to + col * S::kPitch + row) = v;
  };
  const auto product = [&](const float* x, const float* y) {
    f32x4_t u = {0, 0, 0, 0}, v = {0, 0, 0, 0};  // two sums, for half the way through each
#pragma unroll
    for (int k = 0; k < NT; ++k) {
      const f32x4_t p = *(const f32x4_t*)(x + (16 * ti + r) * S::kPitch + 16 * k + 4 * g);
      const f32x4_t q = *(const f32x4_t*)(y + (16 * tj + r) * S::kPitch + 16 * k + 4 * g);
      u = multiply(p[0], q[0], u);
      v = multiply(p[1], q[1], v);
      u = multiply(p[2], q[2], u);
      v = multiply(p[3], q[3], v);
    }
    return u + v;
  };
  // G G^T, all parts with the largest one's scale
  constexpr int kAtOnce = NT == 1 ? 32 : 16;  // parts in flight
  const f32x4_t* from = (const f32x4_t*)a.sums + (matrix * a.parts * S::kWaves + wave) * 64 + lane;
  f32x4_t s[kAtOnce];
  const auto load = [&](int p0) {
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) s[u] = from[min(p0 + u, a.parts - 1) * S::kWaves * 64];
  };
  const int its = lane < a.parts ? a.scales[matrix * a.parts + lane] : -kNotFinite;  // at most 64 parts
  load(0);
  int scale = its;
  for (int d = 32; d; d /= 2) scale = max(scale, __shfl_xor(scale, d));
  const int of_lane = 2 * max(its - scale, -200);  // what is left out is below 2^-149
  f32x4_t A = {0, 0, 0, 0}, Q = {0, 0, 0, 0};
  if (scale > -kNotFinite && scale < kNotFinite) {
    for (int p0 = 0; p0 < a.parts; p0 += kAtOnce) {
      if (p0 > 0) load(p0);
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        if (p0 + u >= a.parts) break;
        const int by = __builtin_amdgcn_readlane(of_lane, p0 + u);
#pragma unroll
        for (int k = 0; k < 4; ++k) A[k] += ldexpf(s[u][k], by);
      }
    }
  }
  put(L, A);
  __syncthreads();
  if (wave == 0) {
    float sum = lane < S::kSide ? L[lane * S::kPitch + lane] : 0.0f;  // a side has 64 at the most
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) trace = sum;
  }
  __syncthreads();
  const float sum = scale == kNotFinite ? NAN : trace;
  A *= sum == 0.0f ? 0.0f : 1.0f / sum;
  put(L, A);  // each value's own thread has put it there before
  __syncthreads();
  for (int step = 0; step < a.steps; ++step) {
    const bool last = step + 1 == a.steps;
    f32x4_t T = product(L, L);  // A^2
#pragma unroll
    for (int k = 0; k < 4; ++k) T[k] = fmaf(kC, T[k], fmaf(kB, A[k], row + k == col ? kA : 0.0f));
    put(R, T);
    if (step > 0) put(Z, Q);
    __syncthreads();
    f32x4_t v = A;
    if (!last) v = product(R, L);  // T A
    Q = step > 0 ? product(R, Z) : T;
    if (last) break;
    __syncthreads();
    put(L, v);
    __syncthreads();
    A = product(R, L);  // T A T: all of them commute
    __syncthreads();
    put(L, A);
    __syncthreads();
  }
  Q *= sum == 0.0f ? 0.0f : 1.0f / sqrtf(sum);
  float* to = a.Q + matrix * S::kSide * S::kSide;
#pragma unroll
  for (int k = 0; k < 4; ++k) to[(row + k) * S::kSide + col] = Q[k];
  if (ti != tj) *(f32x4_t*)(to + col * S::kSide + row) = Q;
  if (tid == 0) a.scale[matrix] = scale > -kNotFinite && scale < kNotFinite ? scale : 0;
}

// Q G: a wave takes 16 of the long side.  The operands are passed in the order that
// leaves a lane four neighbours of a row of the result.
template <typename T, int NT>
__global__ __launch_bounds__(256) void few_apply_kernel(FewArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int blocks = (a.m + 63) / 64, m0 = blockIdx.x % blocks * 64 + wave * 16;
  const int64_t matrix = blockIdx.x / blocks;
  if (m0 >= a.m) return;
  const T* G = (const T*)a.G + matrix * a.stride;
  const float* Q = a.Q + matrix * (16 * NT) * (16 * NT);
  const int scale = a.scale[matrix];
  // all of G at once, Q a step ahead
  f32x4_t acc[NT], x[NT], q[2][NT];
#pragma unroll
  for (int k = 0; k < NT; ++k) {
    const int row = 16 * k + 4 * g, col = m0 + r;
    if (a.tall && row + 4 <= a.n && col < a.m) {
      T t[4];
      load_n<T, 4>(G + col * a.ld + row, t);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[k][e] = to_f32(t[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[k][e] = at(G, a, row + e, col);
    }
  }
  const auto fetch = [&](int k, f32x4_t (&q)[NT]) {
#pragma unroll
    for (int t = 0; t < NT; ++t) q[t] = *(const f32x4_t*)(Q + (16 * t + r) * (16 * NT) + 16 * k + 4 * g);
  };
  fetch(0, q[0]);
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = f32x4_t{0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < NT; ++k) {
    if (k + 1 < NT) fetch(k + 1, q[(k + 1) % 2]);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[k][e] = ldexpf(x[k][e], -scale);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[t] = a.tall ? multiply(q[k % 2][t][e], x[k][e], acc[t]) : multiply(x[k][e], q[k % 2][t][e], acc[t]);
  }
  bf16_t* out = (bf16_t*)a.out + matrix * a.stride_out;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    // lane: tall: rows m0 + r, columns 16 t + 4 g ..; else rows 16 t + r, columns m0 + 4 g ..
    const int row = a.tall ? m0 + r : 16 * t + r, col = a.tall ? 16 * t + 4 * g : m0 + 4 * g;
    const int rows = a.tall ? a.m : a.n, cols = a.tall ? a.n : a.m;
    if (row >= rows) continue;
    bf16_t v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = from_f32<bf16_t>(acc[t][e]);
    bf16_t* to = out + row * a.ld_out + col;
    if (col + 4 <= cols) {
      store_n<bf16_t, 4>(to, v);
    } else {
      for (int e = 0; e < 4; ++e)
        if (col + e < cols) to[e] = v[e];
    }
  }
}

// -- host ---------------------------------------------------------------------

struct FewLayout {
  int nt, parts, each;
  int64_t n, m, sums, scales, Q, scale, all;
};

FewLayout few_layout(int64_t rows, int64_t cols, int64_t batch) {
  FewLayout l{};
  l.n = rows < cols ? rows : cols;
  l.m = rows < cols ? cols : rows;
  l.nt = l.n <= 16 ? 1 : l.n <= 32 ? 2 : 4;
  // Parts: as many as the iteration's workgroup adds up quickly (64 KiB to 160 KiB of sums)
  const int most = l.nt == 1 ? 64 : l.nt == 2 ? 32 : 16;
  l.each = (int)(ceil_div(ceil_div(l.m, most), 64) * 64);
  l.parts = (int)ceil_div(l.m, l.each);
  const auto take = [&](int64_t bytes) {
    const int64_t at = l.all;
    l.all += ceil_div(bytes, 256) * 256;
    return at;
  };
  l.sums = take(batch * l.parts * lower_tiles(l.nt) * 1024);
  l.scales = take(batch * l.parts * 4);
  l.Q = take(batch * 256 * l.nt * l.nt * 4);
  l.scale = take(batch * 4);
  return l;
}

template <typename T, int NT>
ws_status run_few(const FewArgs& a, int64_t batch, hipStream_t stream) {
  ws_status s = launch("orthogonalize", &few_gram_kernel<T, NT>, batch * a.parts, 64 * kGramWaves, 0, stream, a);
  if (s == WS_OK) s = launch("orthogonalize", &few_iterate_kernel<NT>, batch, 64 * FewShape<NT>::kWaves, 0, stream, a);
  if (s == WS_OK) s = launch("orthogonalize", &few_apply_kernel<T, NT>, batch * ceil_div(a.m, 64), 256, 0, stream, a);
  return s;
}

template <typename T>
ws_status run_few(const FewArgs& a, int nt, int64_t batch, hipStream_t stream) {
  switch (nt) {
    case 1: return run_few<T, 1>(a, batch, stream);
    case 2: return run_few<T, 2>(a, batch, stream);
    default: return run_few<T, 4>(a, batch, stream);
  }
}

}  // namespace

int64_t few_workspace(int64_t rows, int64_t cols, int64_t batch) { return few_layout(rows, cols, batch).all; }

ws_status orthogonalize_few(const ws_matrix* G, int32_t steps, const ws_matrix* out, void* workspace, hipStream_t stream) {
  const FewLayout l = few_layout(G->rows, G->cols, G->batch);
  uint8_t* w = (uint8_t*)workspace;
  FewArgs a{};
  a.G = G->data;
  a.out = (uint16_t*)out->data;
  a.ld = G->ld;
  a.stride = G->stride;
  a.ld_out = out->ld;
  a.stride_out = out->stride;
  a.n = (int32_t)l.n;
  a.m = (int32_t)l.m;
  a.tall = G->rows > G->cols;
  a.steps = steps;
  a.parts = l.parts;
  a.each = l.each;
  a.sums = (float*)(w + l.sums);
  a.scales = (int32_t*)(w + l.scales);
  a.Q = (float*)(w + l.Q);
  a.scale = (int32_t*)(w + l.scale);
  if (G->dtype == WS_OUT_F32) return run_few<float>(a, l.nt, G->batch, stream);
  if (G->dtype == WS_OUT_BF16) return run_few<bf16_t>(a, l.nt, G->batch, stream);
  return run_few<f16_t>(a, l.nt, G->batch, stream);
}

}  // namespace wsg
