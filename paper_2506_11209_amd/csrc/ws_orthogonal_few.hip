// Orthogonalised updates of matrices with a short side, n <= 64 (definitions:
// ws_orthogonal.h).
//
// Every step multiplies X with a polynomial of A = X X^T, so all of them together
// multiply the first X with one n x n matrix Q: with T = a + b A + c A^2, Q <- T Q and
// A <- T A T.  Three launches whatever the number of steps: A_0 = G G^T over parts of the
// long side, the iteration by one workgroup in LDS, and Q G.
//
// A and the iteration are in binary64: A is not made from X again, so that its error in a
// direction grows as A itself does there, 12 times a step, and a direction of singular
// value s (of G / |G|) comes out within a few u / s^2.  With binary32's u = 2^-24, five
// steps were off by up to 1.3e-3 (in norm) and six by up to 2e-2, where one value is 1 and
// the others 1/1000; now what is left is Q and its product with G in binary32, 2^-24 of the
// largest value of Q, 3.5^steps, and so 1e-4 for kFewSteps.  More steps run in tiles.
// Squares of binary32 values neither overflow nor vanish in binary64.
#include <math.h>

#include "ws_fp8_common.hpp"
#include "ws_orthogonal.hpp"

namespace wsg {
namespace {

constexpr double kA = 3.4445, kB = -4.7750, kC = 2.0315;

struct FewArgs {
  const void* G;
  uint16_t* out;
  int64_t ld, stride, ld_out, stride_out;
  int32_t n, m, tall, steps;  // tall: rows of G are the long side
  int32_t parts, each;        // of the long side, a multiple of 16
  double* sums;               // batch x parts x tiles x 64 x 4: lower triangle of G G^T
  float* Q;                   // batch x (16 NT)^2, by 2^scale / sqrt(trace)
  int32_t* scale;             // batch: Q belongs to G times 2^-scale
};

typedef double f64x4_t __attribute__((ext_vector_type(4)));

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
// Of its sums lane (r, g) has rows g, g + 4 .. of column r; in binary32 rows 4 g, 4 g + 1 ..
__device__ __forceinline__ f64x4_t multiply(double x, double y, f64x4_t c) { return __builtin_amdgcn_mfma_f64_16x16x4f64(x, y, c, 0, 0, 0); }

constexpr int kGramWaves = 4;

// A part's share of G G^T: wave w takes every fourth 16 columns of the part, all tiles
// of the lower triangle; their sums add up in turn in LDS.
template <typename T, int NT>
__global__ __launch_bounds__(64 * kGramWaves) void few_gram_kernel(FewArgs a) {
  constexpr int kTiles = lower_tiles(NT);
  __shared__ f64x4_t sums[kTiles * 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4;
  const int64_t matrix = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts, lo = part * a.each, hi = min(lo + a.each, a.m);
  const T* G = (const T*)a.G + matrix * a.stride;
  f64x4_t acc[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) acc[t] = f64x4_t{0, 0, 0, 0};
  // A step's loads go out before the one before it is multiplied.  Parts are whole 16s, but
  // for the last one's end.
  f32x4_t f[NT], next[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) next[t] = four(G, a, 16 * t + r, lo + 16 * wave + 4 * g);
  for (int k0 = lo + 16 * wave; k0 < hi; k0 += 16 * kGramWaves) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f[t] = next[t];
      next[t] = four(G, a, 16 * t + r, min(k0 + 16 * kGramWaves, a.m) + 4 * g);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j <= i; ++j)
          acc[i * (i + 1) / 2 + j] = multiply((double)f[i][k], (double)f[j][k], acc[i * (i + 1) / 2 + j]);
  }
  for (int w = 0; w < kGramWaves; ++w) {
    if (wave == w)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) sums[t * 64 + lane] = w ? sums[t * 64 + lane] + acc[t] : acc[t];
    __syncthreads();
  }
  f64x4_t* to = (f64x4_t*)a.sums + (int64_t)blockIdx.x * kTiles * 64;
  for (int i = tid; i < kTiles * 64; i += 64 * kGramWaves) to[i] = sums[i];
}

template <int NT>
struct FewShape {
  static constexpr int kWaves = lower_tiles(NT);  // a tile each
  static constexpr int kSide = 16 * NT, kPitch = kSide + 2;  // doubles: rows spread over the banks
  static constexpr int kBytes = 3 * kSide * kPitch * 8;
};

// One workgroup's iteration.  Matrices are symmetric (polynomials of A_0): a wave has a
// tile of the lower triangle and writes it to both its places in a matrix in LDS.  Bound:
// latency, of the way to memory and of three products in a row a step (T Q beside T A)
// with the meetings between them (n = 16: 8.0 us, n = 32: 11.8, n = 64, where it is the
// products themselves on one CU: 33).
template <int NT>
__global__ __launch_bounds__(64 * FewShape<NT>::kWaves) void few_iterate_kernel(FewArgs a) {
  typedef FewShape<NT> S;
  extern __shared__ __align__(16) uint8_t smem[];
  double* L = (double*)smem;
  double *R = L + S::kSide * S::kPitch, *Z = R + S::kSide * S::kPitch;
  __shared__ double trace;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, g = lane >> 4;
  const int64_t matrix = blockIdx.x;
  int ti, tj;
  tile_at(wave, &ti, &tj);
  const int row = 16 * ti + g, col = 16 * tj + r;  // the lane's: rows row, row + 4 ..
  const auto put = [&](double* to, const f64x4_t& v) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      to[(row + 4 * k) * S::kPitch + col] = v[k];
      if (ti != tj) to[col * S::kPitch + row + 4 * k] = v[k];
    }
  };
  const auto product = [&](const double* x, const double* y) {
    f64x4_t u = {0, 0, 0, 0}, v = {0, 0, 0, 0};  // two sums, for half the way through each
#pragma unroll
    for (int k = 0; k < NT; ++k) {
      const double* p = x + (16 * ti + r) * S::kPitch + 16 * k + 4 * g;
      const double* q = y + (16 * tj + r) * S::kPitch + 16 * k + 4 * g;
      u = multiply(p[0], q[0], u);
      v = multiply(p[1], q[1], v);
      u = multiply(p[2], q[2], u);
      v = multiply(p[3], q[3], v);
    }
    return u + v;
  };
  // G G^T
  constexpr int kAtOnce = 16;  // parts in flight
  const f64x4_t* from = (const f64x4_t*)a.sums + (matrix * a.parts * S::kWaves + wave) * 64 + lane;
  f64x4_t A = {0, 0, 0, 0}, Q = {0, 0, 0, 0};
  for (int p0 = 0; p0 < a.parts; p0 += kAtOnce) {
    f64x4_t s[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) s[u] = from[min(p0 + u, a.parts - 1) * S::kWaves * 64];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
      if (p0 + u < a.parts) A += s[u];
  }
  put(L, A);
  __syncthreads();
  if (wave == 0) {
    double sum = lane < S::kSide ? L[lane * S::kPitch + lane] : 0.0;  // a side has 64 at the most
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) trace = sum;
  }
  __syncthreads();
  // Sums of finite squares stay below 2^256 2^22; an infinity or NaN makes all of Q NaN.
  const double sum = trace < INFINITY ? trace : (double)NAN;
  A *= sum == 0.0 ? 0.0 : 1.0 / sum;
  put(L, A);  // each value's own thread has put it there before
  __syncthreads();
  for (int step = 0; step < a.steps; ++step) {
    const bool last = step + 1 == a.steps;
    f64x4_t T = product(L, L);  // A^2
#pragma unroll
    for (int k = 0; k < 4; ++k) T[k] = fma(kC, T[k], fma(kB, A[k], row + 4 * k == col ? kA : 0.0));
    put(R, T);
    if (step > 0) put(Z, Q);
    __syncthreads();
    f64x4_t v = A;
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
  // G's largest value is within sqrt(trace) and 1 / sqrt(n m) of it: both factors of Q G
  // stay inside binary32's range
  const double norm = sqrt(sum);
  const int scale = sum > 0.0 ? ilogb(norm) : 0;
  Q *= sum == 0.0 ? 0.0 : ldexp(1.0, scale) / norm;
  float* to = a.Q + matrix * S::kSide * S::kSide;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    to[(row + 4 * k) * S::kSide + col] = (float)Q[k];
    if (ti != tj) to[col * S::kSide + row + 4 * k] = (float)Q[k];
  }
  if (tid == 0) a.scale[matrix] = scale;
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
  int64_t n, m, sums, Q, scale, all;
};

FewLayout few_layout(int64_t rows, int64_t cols, int64_t batch) {
  FewLayout l{};
  l.n = rows < cols ? rows : cols;
  l.m = rows < cols ? cols : rows;
  l.nt = l.n <= 16 ? 1 : l.n <= 32 ? 2 : 4;
  // Parts: as many as the iteration's workgroup adds up quickly (128 KiB to 320 KiB of sums)
  const int most = l.nt == 1 ? 64 : l.nt == 2 ? 32 : 16;
  l.each = (int)(ceil_div(ceil_div(l.m, most), 64) * 64);
  l.parts = (int)ceil_div(l.m, l.each);
  const auto take = [&](int64_t bytes) {
    const int64_t at = l.all;
    l.all += ceil_div(bytes, 256) * 256;
    return at;
  };
  l.sums = take(batch * l.parts * lower_tiles(l.nt) * 2048);
  l.Q = take(batch * 256 * l.nt * l.nt * 4);
  l.scale = take(batch * 4);
  return l;
}

template <typename T, int NT>
ws_status run_few(const FewArgs& a, int64_t batch, hipStream_t stream) {
  ws_status s = launch("orthogonalize", &few_gram_kernel<T, NT>, batch * a.parts, 64 * kGramWaves, 0, stream, a);
  static std::atomic<uint64_t> allowed;
  if (s == WS_OK) s = allow_lds((const void*)&few_iterate_kernel<NT>, FewShape<NT>::kBytes, allowed);
  if (s == WS_OK) s = launch("orthogonalize", &few_iterate_kernel<NT>, batch, 64 * FewShape<NT>::kWaves, FewShape<NT>::kBytes, stream, a);
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
  a.sums = (double*)(w + l.sums);
  a.Q = (float*)(w + l.Q);
  a.scale = (int32_t*)(w + l.scale);
  if (G->dtype == WS_OUT_F32) return run_few<float>(a, l.nt, G->batch, stream);
  if (G->dtype == WS_OUT_BF16) return run_few<bf16_t>(a, l.nt, G->batch, stream);
  return run_few<f16_t>(a, l.nt, G->batch, stream);
}

}  // namespace wsg
