// The router's choice of experts, its balance loss and its gradient (definitions:
// ws_experts.h).
#include <math.h>

#include <type_traits>

#include "ws_experts.h"
#include "ws_fp8_common.hpp"

namespace wsg {
namespace {

struct ChooseArgs {
  const void* logits;
  void* dlogits;
  float *weights, *loss, *sums;  // sums: blocks x (experts + 1), of probabilities; null for one workgroup alone
  int32_t *ids, *counts, *parts;  // parts: blocks x (experts + 1), counts
  const float *dweights, *dloss;
  double* products;  // choose_finish_kernel's workgroups x 3
  uint32_t* ended;   // of them
  int64_t tokens, ld, ld_d;
  int32_t experts, k, blocks;
};

template <int CTRL>
__device__ __forceinline__ float rotated(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
// Sum over L lanes (16 or 64), the same bits in all of them.
template <int L>
__device__ __forceinline__ float sum_lanes(float x) {
  x += rotated<0x128>(x);  // row_ror:8
  x += rotated<0x124>(x);
  x += rotated<0x122>(x);
  x += rotated<0x121>(x);
  if constexpr (L == 64) {
    x += __shfl_xor(x, 16);
    x += __shfl_xor(x, 32);
  }
  return x;
}
template <int L>
__device__ __forceinline__ float largest(float x) {
  x = fmaxf(x, rotated<0x128>(x));
  x = fmaxf(x, rotated<0x124>(x));
  x = fmaxf(x, rotated<0x122>(x));
  x = fmaxf(x, rotated<0x121>(x));
  if constexpr (L == 64) {
    x = fmaxf(x, __shfl_xor(x, 16));
    x = fmaxf(x, __shfl_xor(x, 32));
  }
  return x;
}
template <int L>
__device__ __forceinline__ uint32_t max_lanes(uint32_t x) {
  x = max16(x);
  if constexpr (L == 64) {
    x = max(x, (uint32_t)__shfl_xor((int)x, 16));
    x = max(x, (uint32_t)__shfl_xor((int)x, 32));
  }
  return x;
}

// Logits in the order in which they are chosen: larger is earlier, NaN first of all,
// both zeros the same, what is below kLeast is not chosen.  A rank of 16 bits leaves room
// for the element's number, so that no two ranks are alike (kOwn) and the next below one
// is found without a mark on what went before.
template <typename T>
struct Rank {
  static constexpr bool kOwn = sizeof(T) == 2;
  // above -inf, whose bits are ff80 of bf16, fc00 of f16 and ff800000
  static constexpr uint32_t kLeast = std::is_same<T, f16_t>::value ? 0x04000000u : 0x00800000u;
  // What of() takes of an element's number.
  static __device__ __forceinline__ uint32_t mark(int e) { return kOwn ? 0x8000ffffu - (uint32_t)e : 0x80000000u; }
  static __device__ __forceinline__ uint32_t nan(uint32_t mark) { return kOwn ? 0xffff0000u | mark : 0xffffffffu; }
  // Of all but NaN.
  static __device__ __forceinline__ uint32_t of(T v, uint32_t mark) {
    uint32_t b;
    if constexpr (std::is_same<T, f16_t>::value) {
      const _Float16 h = v.v + (_Float16)0.0f;  // -0 becomes +0
      uint16_t bits;
      __builtin_memcpy(&bits, &h, 2);
      b = (uint32_t)bits << 16;
    } else {
      b = __float_as_uint(to_f32(v) + 0.0f);
    }
    return b ^ (((uint32_t)((int32_t)b >> 31) & (kOwn ? 0x7fff0000u : 0x7fffffffu)) | mark);
  }
  static __device__ __forceinline__ float value(uint32_t rank) {
    const uint32_t b = rank & 0x80000000u ? rank ^ 0x80000000u : ~rank;
    if constexpr (kOwn) {
      const uint16_t h = (uint16_t)(b >> 16);
      T v;
      __builtin_memcpy(&v, &h, 2);
      return to_f32(v);
    }
    return __uint_as_float(b);
  }
  static __device__ __forceinline__ int element(uint32_t rank) { return 0xffff - (int)(rank & 0xffffu); }
};

// e^(x - top) by the power of two: the difference and its product with log2(e) round,
// by 2^-23 of the exponent together.
__device__ __forceinline__ float exp_from(float x, float top) { return __builtin_amdgcn_exp2f((x - top) * 1.44269504088896341f); }

// A row of up to L V logits on L lanes: lane i holds elements W i .. W i + W - 1 of
// every W L, W as many as 16 bytes hold.
template <typename T, int L, int V>
struct Row {
  static constexpr int kWide = 16 / (int)sizeof(T), W = V < kWide ? V : kWide;
  static __device__ __forceinline__ int element(int sub, int v) { return v / W * (L * W) + sub * W + v % W; }
  // -inf past the row's n elements.  readable: elements from its first on that are the
  // caller's, so that a row's end is read along with what follows it and is not taken.
  static __device__ __forceinline__ void load(const T* row, int sub, int n, int64_t readable, T (&x)[V]) {
#pragma unroll
    for (int v = 0; v < V; v += W) {
      const int e = element(sub, v);
      const T none = from_f32<T>(-INFINITY);
#pragma unroll
      for (int w = 0; w < W; ++w) x[v + w] = none;
      if constexpr (W * sizeof(T) >= 4) {
        if (e < n && e + W <= readable) {
          load_n<T, W>(row + e, x + v);
        } else {
#pragma unroll
          for (int w = 0; w < W; ++w)
            if (e + w < n) x[v + w] = row[e + w];
        }
        if (n % W)  // the same for the launch
#pragma unroll
          for (int w = 0; w < W; ++w) x[v + w] = e + w < n ? x[v + w] : none;
      } else {
        if (e < n) x[v] = row[e];
      }
    }
  }
  static __device__ __forceinline__ void store(T* row, int sub, int n, const T (&x)[V]) {
#pragma unroll
    for (int v = 0; v < V; v += W) {
      const int e = element(sub, v), left = n - e;
      if constexpr (W * sizeof(T) >= 4) {
        if (left >= W) {
          store_n<T, W>(row + e, x + v);
          continue;
        }
        if (left <= 0) continue;
        T r[W];  // the row's end: the larger pieces first
#pragma unroll
        for (int w = 0; w < W; ++w) r[w] = x[v + w];
        T* to = row + e;
        if constexpr (W >= 8) {
          if (left & 4) {
            store_n<T, 4>(to, r);
            to += 4;
#pragma unroll
            for (int w = 0; w < 4; ++w) r[w] = r[w + 4];
          }
        }
        if constexpr (W >= 4) {
          if (left & 2) {
            to[0] = r[0];
            to[1] = r[1];
            to += 2;
            r[0] = r[2];
          }
        }
        if (left & 1) to[0] = r[0];
      } else {
        if (left > 0) row[e] = x[v];
      }
    }
  }
};

// Waves of a workgroup: the sums of a wave's tokens pass LDS.
template <int L>
constexpr int choose_waves() { return L == 16 ? 16 : 8; }

// What the sums of probabilities and the counts give, S_e and c_e in LDS.
__device__ __forceinline__ void finish(const ChooseArgs& a, const float* sums, const int32_t* counts, double* scratch) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
  double dot = 0.0, all = 0.0;
  for (int e = tid; e < a.experts; e += blockDim.x) {
    dot += (double)counts[e] * (double)sums[e];
    all += (double)counts[e];
    a.counts[e] = counts[e];
  }
  for (int d = 32; d; d /= 2) {
    dot += __shfl_xor(dot, d);
    all += __shfl_xor(all, d);
  }
  if (lane == 0) {
    scratch[2 * wave] = dot;
    scratch[2 * wave + 1] = all;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < waves; ++w) {
      dot += scratch[2 * w];
      all += scratch[2 * w + 1];
    }
    const double n = (double)counts[a.experts];
    a.counts[a.experts] = counts[a.experts];
    *a.loss = n > 0.0 ? (float)((double)a.experts * dot / (all * n)) : 0.0f;
  }
}

// L lanes take a token: its row stays in registers, the choices are k searches for the
// largest (and lowest) left, the first of which is the softmax's maximum too.  Sums of
// probabilities and counts stay in the lanes over a workgroup's tokens and pass LDS at
// the end, in a fixed order.  ALONE: one workgroup.
// Bound: instructions, some 35 for a logit and 8 choices, about 15 us of issue, and the
// latency of the lanes' maxima, one choice after the other with four waves a SIMD (65536 x
// 256 of bf16, 8 choices: 25.8 us, 1.4 TB/s; with ranks cleared of what went before instead of differences 34.6;
// with the next token's row under way meanwhile 26.7).
template <typename T, int L, int V, bool ALONE>
__global__ __launch_bounds__(64 * choose_waves<L>()) void choose_kernel(ChooseArgs a) {
  typedef Row<T, L, V> R;
  constexpr int kWaves = choose_waves<L>(), kGroups = kWaves * 64 / L, kMine = (WS_MAX_CHOICES + L - 1) / L;
  extern __shared__ __align__(16) uint8_t smem[];
  const int n = a.experts + 1;  // the last: tokens with a choice
  if (!ALONE && blockIdx.x == 0 && threadIdx.x == 0) *a.ended = 0;  // read by the next launch
  float* lds_sums = (float*)smem;                    // waves x n
  int32_t* lds_counts = (int32_t*)(lds_sums + kWaves * n);  // waves x n
  __shared__ double scratch[2 * kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = tid % L;
  float sums[V];
  int32_t counts[V], with = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    sums[v] = 0.0f;
    counts[v] = 0;
  }
  typedef Rank<T> K;
  const int64_t step = (int64_t)a.blocks * kGroups;
  for (int64_t t = (int64_t)blockIdx.x * kGroups + tid / L; t < a.tokens; t += step) {
    T raw[V];
    R::load((const T*)a.logits + t * a.ld, sub, a.experts, a.experts + (a.tokens - 1 - t) * a.ld, raw);
    uint32_t key[V], best = 0;
    bool nan = false;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      key[v] = K::of(raw[v], K::mark(R::element(sub, v)));  // -inf past the last expert
      nan |= __builtin_isunordered(to_f32(raw[v]), to_f32(raw[v ^ (V > 1)]));
    }
    if (__any(nan))
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = to_f32(raw[v]) != to_f32(raw[v]) ? K::nan(K::mark(R::element(sub, v))) : key[v];
#pragma unroll
    for (int v = 0; v < V; ++v) best = max(best, key[v]);
    best = max_lanes<L>(best);
    const bool some = best >= K::kLeast;
    const float top = K::value(best);
    if (some) {
      float p[V], sum = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        p[v] = exp_from(to_f32(raw[v]), top);
        sum += p[v];
      }
      const float by = 1.0f / sum_lanes<L>(sum);
#pragma unroll
      for (int v = 0; v < V; ++v) sums[v] = fmaf(p[v], by, sums[v]);
    }
    // a lane has the choices j = sub, sub + L ..
    uint32_t rank[kMine], last = ~0u;
    int32_t id[kMine];
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      rank[q] = 0;
      id[q] = -1;
      for (int j = q * L; j < a.k && j < (q + 1) * L; ++j) {
        if (j > 0) {
          uint32_t next = 0;
          if constexpr (K::kOwn) {  // of the differences, those of ranks below wrap and are the largest
#pragma unroll
            for (int v = 0; v < V; ++v) next = max(next, key[v] - best);
            next = max_lanes<L>(next) + best;
            best = next < best ? next : 0;
          } else {
#pragma unroll
            for (int v = 0; v < V; ++v) next = max(next, key[v]);
            best = max_lanes<L>(next);
          }
        }
        if (best < K::kLeast) break;
        last = best;
        const bool mine = j - q * L == sub;
        rank[q] = mine ? best : rank[q];
        if constexpr (!K::kOwn) {
          uint32_t low = 0;  // the lowest element with it, as a large number
#pragma unroll
          for (int v = V - 1; v >= 0; --v) low = key[v] == best ? ~(uint32_t)R::element(sub, v) : low;
          const int e = (int)~max_lanes<L>(low);
          id[q] = mine ? e : id[q];
#pragma unroll
          for (int v = 0; v < V; ++v) key[v] = R::element(sub, v) == e ? 0 : key[v];
        }
      }
    }
    float w[kMine], all = 0.0f;
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      if (K::kOwn && rank[q] != 0) id[q] = K::element(rank[q]);
      w[q] = rank[q] != 0 ? exp_from(K::value(rank[q]), top) : 0.0f;
      all += w[q];
    }
    const float by = 1.0f / sum_lanes<L>(all);
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      const int j = q * L + sub;
      if (j < a.k) {
        a.ids[t * a.k + j] = id[q];
        a.weights[t * a.k + j] = rank[q] != 0 ? w[q] * by : 0.0f;
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) counts[v] += K::kOwn ? key[v] >= last : key[v] == 0;
    with += some;
  }
  // the wave's tokens, then the workgroup's
  const auto add_groups = [](auto x) {
    if constexpr (L == 16) {
      x += __shfl_xor(x, 16);
      x += __shfl_xor(x, 32);
    }
    return x;
  };
#pragma unroll
  for (int v = 0; v < V; ++v) {
    sums[v] = add_groups(sums[v]);
    counts[v] = add_groups(counts[v]);
    const int e = R::element(sub, v);
    if (lane < L && e < a.experts) {
      lds_sums[wave * n + e] = sums[v];
      lds_counts[wave * n + e] = counts[v];
    }
  }
  with = add_groups(with);
  if (lane == 0) {
    lds_sums[wave * n + a.experts] = 0.0f;
    lds_counts[wave * n + a.experts] = with;
  }
  __syncthreads();
  for (int e = tid; e < n; e += 64 * kWaves) {
    float s = lds_sums[e];
    int32_t c = lds_counts[e];
    for (int w = 1; w < kWaves; ++w) {
      s += lds_sums[w * n + e];
      c += lds_counts[w * n + e];
    }
    if constexpr (ALONE) {
      lds_sums[e] = s;
      lds_counts[e] = c;
    } else {
      a.sums[(int64_t)blockIdx.x * n + e] = s;
      a.parts[(int64_t)blockIdx.x * n + e] = c;
    }
  }
  if constexpr (ALONE) {
    __syncthreads();
    finish(a, lds_sums, lds_counts, scratch);
  }
}

// Adds up what the workgroups left: a workgroup takes 16 columns, in a fixed order, and
// the last to end the products of all of them.  Bound: latency (256 times 257 columns:
// 5.0 us; by one workgroup 11.9).
constexpr int kFinishCols = 16, kFinishSlices = 16, kFinishReads = 16;  // blocks: at most slices x reads
constexpr int finish_groups(int experts) { return experts / kFinishCols + 1; }

__global__ __launch_bounds__(kFinishCols* kFinishSlices) void choose_finish_kernel(ChooseArgs a) {
  __shared__ float sums[kFinishSlices][kFinishCols];
  __shared__ int32_t counts[kFinishSlices][kFinishCols];
  __shared__ double scratch[3][4];
  __shared__ bool last;
  const int tid = threadIdx.x, col = tid % kFinishCols, slice = tid / kFinishCols;
  const int n = a.experts + 1, e = blockIdx.x * kFinishCols + col, groups = gridDim.x;
  float x[kFinishReads], s = 0.0f;
  int32_t y[kFinishReads], c = 0;
#pragma unroll
  for (int u = 0; u < kFinishReads; ++u) {
    const int64_t at = (int64_t)min(slice + kFinishSlices * u, a.blocks - 1) * n + min(e, n - 1);
    x[u] = a.sums[at];
    y[u] = a.parts[at];
  }
#pragma unroll
  for (int u = 0; u < kFinishReads; ++u) {
    s += slice + kFinishSlices * u < a.blocks ? x[u] : 0.0f;
    c += slice + kFinishSlices * u < a.blocks ? y[u] : 0;
  }
  sums[slice][col] = s;
  counts[slice][col] = c;
  __syncthreads();
  double dot = 0.0, all = 0.0, with = 0.0;
  if (slice == 0 && e < n) {
    for (int i = 1; i < kFinishSlices; ++i) {
      s += sums[i][col];
      c += counts[i][col];
    }
    a.counts[e] = c;
    dot = e < a.experts ? (double)c * (double)s : 0.0;
    all = e < a.experts ? (double)c : 0.0;
    with = e < a.experts ? 0.0 : (double)c;
  }
  for (int d = kFinishCols / 2; d; d /= 2) {
    dot += __shfl_xor(dot, d);
    all += __shfl_xor(all, d);
    with += __shfl_xor(with, d);
  }
  if (tid == 0) {
    double* mine = a.products + 3 * blockIdx.x;
    mine[0] = dot;
    mine[1] = all;
    mine[2] = with;
    __threadfence();
    last = atomicAdd(a.ended, 1u) == (uint32_t)groups - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  const auto take = [&](int k) {
    return tid < groups ? __hip_atomic_load(a.products + 3 * tid + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
  };
  dot = take(0);
  all = take(1);
  with = take(2);
  for (int d = 32; d; d /= 2) {
    dot += __shfl_xor(dot, d);
    all += __shfl_xor(all, d);
    with += __shfl_xor(with, d);
  }
  if (tid % 64 == 0) {
    scratch[0][tid / 64] = dot;
    scratch[1][tid / 64] = all;
    scratch[2][tid / 64] = with;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < 4; ++w) {
      dot += scratch[0][w];
      all += scratch[1][w];
      with += scratch[2][w];
    }
    *a.loss = with > 0.0 ? (float)((double)a.experts * dot / (all * with)) : 0.0f;
  }
}

// L lanes take a token: its softmax again from its logits, what its weights ask of its
// choices by way of a row in LDS, and one write; the next token's values are under way
// meanwhile.  Bound: instructions and latency (65536 x 256 of bf16: 22 us, 67 MB, 3.1 TB/s,
// of f32 24 us, 5.5 TB/s; 30001 x 100 of bf16 9.5; 8192 x 64 of f32 4.0, 1 TB/s).
template <typename T, int L, int V>
__global__ __launch_bounds__(256) void choose_gradient_kernel(ChooseArgs a) {
  typedef Row<T, L, V> R;
  constexpr int kGroups = 256 / L, kMine = (WS_MAX_CHOICES + L - 1) / L;
  __shared__ float rows[kGroups][L * V];
  const int tid = threadIdx.x, sub = tid % L;
  float* row = rows[tid / L];
  T raw[V], next[V];
  int32_t id[kMine], next_id[kMine];
  float w[kMine], next_w[kMine], dw[kMine], next_dw[kMine];
  const auto load = [&](int64_t t) {
    if (t >= a.tokens) return;
    R::load((const T*)a.logits + t * a.ld, sub, a.experts, a.experts + (a.tokens - 1 - t) * a.ld, next);
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      const int j = q * L + sub;
      next_id[q] = -1;
      next_w[q] = next_dw[q] = 0.0f;
      if (a.dweights && j < a.k) {
        next_id[q] = a.ids[t * a.k + j];
        next_w[q] = a.weights[t * a.k + j];
        next_dw[q] = a.dweights[t * a.k + j];
      }
    }
  };
  const int64_t step = (int64_t)gridDim.x * kGroups;
  int64_t t = (int64_t)blockIdx.x * kGroups + tid / L;
  load(t);
  // counts, and what of the loss belongs to one choice of one token
  float c[V], all = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {  // loads without a branch, so that they are under way together
    c[v] = (float)a.counts[min(R::element(sub, v), a.experts - 1)];
    row[R::element(sub, v)] = 0.0f;
  }
  const float n = (float)a.counts[a.experts], dloss = a.dloss ? *a.dloss : 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    c[v] = R::element(sub, v) < a.experts ? c[v] : 0.0f;
    all += c[v];
  }
  all = sum_lanes<L>(all);
  const float scale = a.dloss && all > 0.0f && n > 0.0f ? dloss * (float)a.experts / all / n : 0.0f;
  __builtin_amdgcn_wave_barrier();
  for (; t < a.tokens; t += step) {
    float dot = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) raw[v] = next[v];
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      id[q] = next_id[q];
      w[q] = next_w[q];
      dw[q] = next_dw[q];
    }
    load(t + step);
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      if ((uint32_t)id[q] >= (uint32_t)a.experts) {
        id[q] = -1;
        w[q] = dw[q] = 0.0f;
      }
      dot = fmaf(w[q], dw[q], dot);
    }
    // the largest that is no NaN: a NaN makes the sum one
    float x[V], top = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[v] = to_f32(raw[v]);  // -inf past the last expert
      top = fmaxf(top, x[v]);
    }
    top = largest<L>(top);
    const float from = top == -INFINITY ? 0.0f : top;  // a masked token's exponentials are zeros
    float sum = 0.0f, of_counts = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[v] = exp_from(x[v], from);
      sum += x[v];
      of_counts = fmaf(c[v], x[v], of_counts);
    }
    sum = sum_lanes<L>(sum);
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
    of_counts = sum_lanes<L>(of_counts) * by;
    dot = sum_lanes<L>(dot);
    // what a choice is asked, added up where an id comes twice: the same for all its places;
    // then the row holds another place than one's own
    float asked[kMine];
    bool twice = false;
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      asked[q] = w[q] * (dw[q] - dot);
      if (id[q] >= 0) __hip_atomic_store(row + id[q], (float)(q * L + sub), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int q = 0; q < kMine; ++q)
      if (id[q] >= 0)
        twice |= __hip_atomic_load(row + id[q], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT) != (float)(q * L + sub);
    __builtin_amdgcn_wave_barrier();
    if (__any(twice)) {
      float of[kMine];
#pragma unroll
      for (int q = 0; q < kMine; ++q) {
        of[q] = asked[q];
        asked[q] = 0.0f;
      }
#pragma unroll
      for (int o = 0; o < kMine; ++o)
#pragma unroll 1
        for (int j = 0; j < L && o * L + j < a.k; ++j) {
          const int other = __shfl(id[o], j, L);
          const float more = __shfl(of[o], j, L);
#pragma unroll
          for (int q = 0; q < kMine; ++q) asked[q] += other == id[q] ? more : 0.0f;
        }
    }
#pragma unroll
    for (int q = 0; q < kMine; ++q)
      if (id[q] >= 0) row[id[q]] = asked[q];
    __builtin_amdgcn_wave_barrier();  // a wave's LDS accesses keep their order
    T d[V];
#pragma unroll
    for (int v = 0; v < V; ++v) d[v] = from_f32<T>(fmaf(scale * (x[v] * by), c[v] - of_counts, row[R::element(sub, v)]));
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int q = 0; q < kMine; ++q)
      if (id[q] >= 0) row[id[q]] = 0.0f;
    __builtin_amdgcn_wave_barrier();
    R::store((T*)a.dlogits + t * a.ld_d, sub, a.experts, d);
  }
}

// -- host ---------------------------------------------------------------------

constexpr int kMostBlocks = 256;  // one a CU
static_assert(kMostBlocks <= kFinishSlices * kFinishReads && finish_groups(WS_MAX_EXPERTS) <= kFinishCols * kFinishSlices, "sizes");
// Tokens that one workgroup takes by itself (256 x 64: 12.2 us, by several and a second
// launch 14.8).
constexpr int64_t kAloneTokens = 256;

bool choose_sizes(int64_t tokens, int32_t experts, int32_t k) {
  return tokens >= 0 && experts >= 1 && experts <= WS_MAX_EXPERTS && k >= 1 && k <= experts && k <= WS_MAX_CHOICES &&
         tokens <= kMaxDim && tokens * k <= kMaxDim;
}

int lanes_of(int experts) { return experts <= 256 ? 16 : 64; }

int choose_blocks(int64_t tokens, int experts) {
  if (tokens <= kAloneTokens) return 1;
  const int64_t groups = experts <= 256 ? choose_waves<16>() * 4 : choose_waves<64>(), n = ceil_div(tokens, groups);
  return (int)(n < kMostBlocks ? n : kMostBlocks);
}

// f(type, lanes, elements a lane) of the smallest that holds a row.
template <typename T, typename F>
ws_status by_experts(int experts, const F& f) {
  typedef std::integral_constant<int, 16> L16;
  typedef std::integral_constant<int, 64> L64;
  if (experts <= 16) return f(T{}, L16{}, std::integral_constant<int, 1>{});
  if (experts <= 64) return f(T{}, L16{}, std::integral_constant<int, 4>{});
  if (experts <= 128) return f(T{}, L16{}, std::integral_constant<int, 8>{});
  if (experts <= 256) return f(T{}, L16{}, std::integral_constant<int, 16>{});
  if (experts <= 512) return f(T{}, L64{}, std::integral_constant<int, 8>{});
  return f(T{}, L64{}, std::integral_constant<int, 16>{});
}
template <typename F>
ws_status by_type(int32_t dtype, int experts, const F& f) {
  if (dtype == WS_OUT_F32) return by_experts<float>(experts, f);
  if (dtype == WS_OUT_BF16) return by_experts<bf16_t>(experts, f);
  return by_experts<f16_t>(experts, f);
}

bool aligned4(const void* p) { return p && (uintptr_t)p % 4 == 0; }

}  // namespace
}  // namespace wsg

using namespace wsg;

extern "C" {

int64_t ws_expert_choose_workspace(int64_t tokens, int32_t experts, int32_t k) {
  if (!choose_sizes(tokens, experts, k)) return -1;
  const int blocks = choose_blocks(tokens, experts);
  return blocks == 1 ? 0 : (int64_t)finish_groups(experts) * 24 + 8 + (int64_t)blocks * (experts + 1) * 8;
}

ws_status ws_expert_choose(const ws_matrix* logits, int32_t k, float* weights, int32_t* ids, int32_t* counts, float* loss,
                           void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  if (!valid(logits) || logits->batch > 1 || logits->cols > WS_MAX_EXPERTS) return WS_ERR_INVALID_ARG;
  const int64_t need = ws_expert_choose_workspace(logits->rows, (int32_t)logits->cols, k);
  if (need < 0 || workspace_bytes < need || (need > 0 && (!workspace || (uintptr_t)workspace % 8)) || !aligned4(counts) || !aligned4(loss) ||
      (logits->rows > 0 && (!aligned4(weights) || !aligned4(ids))))
    return WS_ERR_INVALID_ARG;
  ChooseArgs a{};
  a.logits = logits->data;
  a.weights = weights;
  a.loss = loss;
  a.ids = ids;
  a.counts = counts;
  a.tokens = logits->rows;
  a.ld = logits->ld;
  a.experts = (int32_t)logits->cols;
  a.k = k;
  a.blocks = choose_blocks(a.tokens, a.experts);
  if (a.blocks > 1) {
    a.products = (double*)workspace;
    a.ended = (uint32_t*)(a.products + 3 * finish_groups(a.experts));
    a.sums = (float*)(a.ended + 2);
    a.parts = (int32_t*)(a.sums + (int64_t)a.blocks * (a.experts + 1));
  }
  const ws_status s = by_type(logits->dtype, a.experts, [&](auto type, auto lanes, auto each) {
    typedef decltype(type) T;
    constexpr int L = decltype(lanes)::value, V = decltype(each)::value, waves = choose_waves<L>();
    const int lds = waves * (a.experts + 1) * 8;
    if (a.blocks == 1) return launch("expert_choose", &choose_kernel<T, L, V, true>, 1, 64 * waves, lds, stream, a);
    return launch("expert_choose", &choose_kernel<T, L, V, false>, a.blocks, 64 * waves, lds, stream, a);
  });
  if (s != WS_OK || a.blocks == 1) return s;
  return launch("expert_choose", &choose_finish_kernel, finish_groups(a.experts), kFinishCols * kFinishSlices, 0, stream, a);
}

ws_status ws_expert_choose_gradient(const ws_matrix* logits, int32_t k, const float* dweights, const float* dloss,
                                    const float* weights, const int32_t* ids, const int32_t* counts, const ws_matrix* dlogits,
                                    hipStream_t stream) {
  if (!valid(logits) || logits->batch > 1 || !valid(dlogits) || dlogits->batch > 1 || logits->rows != dlogits->rows ||
      logits->cols != dlogits->cols || logits->dtype != dlogits->dtype || logits->cols > WS_MAX_EXPERTS ||
      !choose_sizes(logits->rows, (int32_t)logits->cols, k))
    return WS_ERR_INVALID_ARG;
  if (logits->rows == 0) return WS_OK;
  if (!aligned4(counts) || (dloss && (uintptr_t)dloss % 4) || (dweights && (!aligned4(dweights) || !aligned4(weights) || !aligned4(ids))))
    return WS_ERR_INVALID_ARG;
  ChooseArgs a{};
  a.logits = logits->data;
  a.dlogits = dlogits->data;
  a.weights = const_cast<float*>(weights);
  a.ids = const_cast<int32_t*>(ids);
  a.counts = const_cast<int32_t*>(counts);
  a.dweights = dweights;
  a.dloss = dloss;
  a.tokens = logits->rows;
  a.ld = logits->ld;
  a.ld_d = dlogits->ld;
  a.experts = (int32_t)logits->cols;
  a.k = k;
  // us with 512, 1024 and 2048 workgroups at the most: 65536 x 256 of bf16 24.0, 22.1 and 27.8
  const int64_t most = 1024, n = ceil_div(a.tokens, 256 / lanes_of(a.experts));
  return by_type(logits->dtype, a.experts, [&](auto type, auto lanes, auto each) {
    return launch("expert_choose_gradient", &choose_gradient_kernel<decltype(type), decltype(lanes)::value, decltype(each)::value>,
                  n < most ? n : most, 256, 0, stream, a);
  });
}

}  // extern "C"
