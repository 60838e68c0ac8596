// Routing of tokens to experts and back (definitions: ws_experts.h).
#include "ws_experts.h"
#include "ws_fp8_common.hpp"

namespace wsg {
namespace {

// -- sort ----------------------------------------------------------------------

constexpr int kSortWaves = 8;
constexpr int kSortThreads = 64 * kSortWaves;
constexpr int kSortSteps = 4;          // steps of 64 slots whose ids a wave loads at once
constexpr int64_t kSortChunk = kSortSteps * kSortThreads;  // slots of a workgroup
// Slots that one workgroup sorts by itself, where two launches of several take less of
// the GPU but more of the caller.  us of one workgroup and of several, for 64 experts:
// calls back to back from Python 8.9 and 13.3 (2048 slots), 11.3 and 13.5 (4096), 15.7
// and 13.4 (6144); one call waited for 23.1 and 25.5, 27.4 and 25.5, 32.3 and 25.5; in
// a captured graph 7.1 and 7.1, 11.5 and 7.3, 16.0 and 7.4.
constexpr int64_t kSortAlone = 4096;
constexpr int64_t kSortBlocks = 256;   // chunks at the most; beyond, chunks grow

struct SortArgs {
  const void* ids;
  int64_t slots, chunk, blocks;
  int32_t k, experts, id_bytes, bits;  // bits: of an expert's number
  int32_t *offsets, *token, *place;
  int32_t* counts;  // blocks x experts; null for one workgroup alone
};

// The expert of slot s, -1 for none.
__device__ __forceinline__ int slot_expert(const SortArgs& a, int64_t s, int64_t end) {
  if (s >= end) return -1;
  const int64_t id = a.id_bytes == 8 ? ((const int64_t*)a.ids)[s] : (int64_t)((const int32_t*)a.ids)[s];
  return id >= 0 && id < a.experts ? (int)id : -1;
}

// A wave's share of the workgroup's chunk: whole steps of 64 slots.
__device__ __forceinline__ void wave_share(const SortArgs& a, int64_t* lo, int64_t* hi) {
  const int64_t c0 = blockIdx.x * a.chunk, c1 = min(c0 + a.chunk, a.slots);
  const int64_t share = (a.chunk + kSortThreads - 1) / kSortThreads * 64;
  *lo = min(c0 + (int64_t)(threadIdx.x >> 6) * share, c1);
  *hi = min(*lo + share, c1);
}

// One step of a wave: adds its lanes' slots to mine[e] and returns how many slots
// of the lane's expert came before its own.  The lanes of one expert find each
// other by ballots over the bits of its number; the first of them adds for all,
// so the counts need no atomics and the order is that of the slots.
__device__ __forceinline__ int take_step(const SortArgs& a, int e, int32_t* mine) {
  const int lane = threadIdx.x & 63;
  uint64_t same = __ballot(e >= 0);
  for (int b = 0; b < a.bits; ++b) {
    const bool set = (e >> b) & 1;
    const uint64_t m = __ballot(set);
    same &= set ? m : ~m;
  }
  int before = 0;
  if (e >= 0) {
    const int rank = __popcll(same & ((1ull << lane) - 1));
    const int at = __hip_atomic_load(&mine[e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    __builtin_amdgcn_wave_barrier();  // every lane has read before the first of each expert writes
    if (rank == 0) __hip_atomic_store(&mine[e], at + __popcll(same), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    before = at + rank;
  }
  __builtin_amdgcn_wave_barrier();
  return before;
}

__device__ __forceinline__ void load_steps(const SortArgs& a, int64_t s0, int64_t hi, int (&e)[kSortSteps]) {
#pragma unroll
  for (int i = 0; i < kSortSteps; ++i) e[i] = slot_expert(a, s0 + 64 * i + (threadIdx.x & 63), hi);
}

// counts[w][e] of this workgroup's waves, in LDS.
__device__ __forceinline__ void count_slots(const SortArgs& a, int32_t* counts) {
  for (int i = threadIdx.x; i < kSortWaves * a.experts; i += kSortThreads) counts[i] = 0;
  __syncthreads();
  int64_t lo, hi;
  wave_share(a, &lo, &hi);
  int32_t* mine = counts + (threadIdx.x >> 6) * a.experts;
  for (int64_t s0 = lo; s0 < hi; s0 += 64 * kSortSteps) {
    int e[kSortSteps];
    load_steps(a, s0, hi, e);
#pragma unroll
    for (int i = 0; i < kSortSteps; ++i)
      if (s0 + 64 * i < hi) take_step(a, e[i], mine);
  }
  __syncthreads();
}

// First of two launches: how many slots of each expert a chunk has.  Bound, both:
// latency, a chain of loads, ballots and meetings (8192 x 4 slots of 64 experts: 2.2 to
// 3.6 us, and 7.2 for place_kernel).
__global__ __launch_bounds__(kSortThreads) void count_kernel(SortArgs a) {
  extern __shared__ int32_t lds[];
  count_slots(a, lds);
  for (int e = threadIdx.x; e < a.experts; e += kSortThreads) {
    int n = 0;
    for (int w = 0; w < kSortWaves; ++w) n += lds[w * a.experts + e];
    a.counts[blockIdx.x * a.experts + e] = n;
  }
}

// Gives every slot its place: the first row of its expert, after the slots of
// earlier chunks, of earlier waves and of earlier steps.  ALONE: one workgroup.
template <bool ALONE>
__global__ __launch_bounds__(kSortThreads) void place_kernel(SortArgs a) {
  extern __shared__ int32_t lds[];
  int32_t* counts = lds;                            // waves x experts
  int32_t* first = lds + kSortWaves * a.experts;    // experts: rows of it, then its first row
  int32_t* sums = first + a.experts;                // one for each wave
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  count_slots(a, counts);
  // rows of each expert; counts[w][e] becomes the slots before wave w's
  for (int e = tid; e < a.experts; e += kSortThreads) {
    int run = 0, all = 0;
    if constexpr (!ALONE)
      for (int b0 = 0; b0 < (int)a.blocks; b0 += 16) {  // 16 loads at once
        int n[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) n[i] = b0 + i < (int)a.blocks ? a.counts[(int64_t)(b0 + i) * a.experts + e] : 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          run += b0 + i < (int)blockIdx.x ? n[i] : 0;
          all += n[i];
        }
      }
    for (int w = 0; w < kSortWaves; ++w) {
      const int n = counts[w * a.experts + e];
      counts[w * a.experts + e] = run;
      run += n;
    }
    first[e] = ALONE ? run : all;
  }
  __syncthreads();
  // exclusive sum over the experts, two a thread (WS_MAX_EXPERTS == 2 kSortThreads)
  const int e0 = 2 * tid, n0 = e0 < a.experts ? first[e0] : 0, n1 = e0 + 1 < a.experts ? first[e0 + 1] : 0;
  int upto = n0 + n1;
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int before = upto - n0 - n1, total = 0;
  for (int w = 0; w < kSortWaves; ++w) {
    if (w < wave) before += sums[w];
    total += sums[w];
  }
  if (e0 < a.experts) first[e0] = before;
  if (e0 + 1 < a.experts) first[e0 + 1] = before + n0;
  __syncthreads();
  if (blockIdx.x == 0) {
    for (int e = tid; e < a.experts; e += kSortThreads) a.offsets[e] = first[e];
    if (tid == 0) a.offsets[a.experts] = total;
  }
  for (int64_t r = total + (int64_t)blockIdx.x * kSortThreads + tid; r < a.slots; r += a.blocks * kSortThreads)
    a.token[r] = -1;
  int64_t lo, hi;
  wave_share(a, &lo, &hi);
  int32_t* mine = counts + wave * a.experts;
  for (int64_t s0 = lo; s0 < hi; s0 += 64 * kSortSteps) {
    int e[kSortSteps];
    load_steps(a, s0, hi, e);
#pragma unroll
    for (int i = 0; i < kSortSteps; ++i) {
      if (s0 + 64 * i >= hi) break;
      const int64_t s = s0 + 64 * i + lane;
      const int before = take_step(a, e[i], mine);
      if (e[i] >= 0) {
        const int row = first[e[i]] + before;
        a.place[s] = row;
        a.token[row] = (int32_t)((uint32_t)s / (uint32_t)a.k);
      } else if (s < hi) {
        a.place[s] = -1;
      }
    }
  }
}

// -- rows ----------------------------------------------------------------------

struct RowArgs {
  const void *x, *dy;
  void* out;
  const int32_t *index, *offsets;
  const float* weights;
  float* dweights;
  int64_t x_rows, rows, cols, ld_x, ld_dy, ld_out;
  int64_t first;  // token of this launch
  int32_t k, experts, parts;
};

// Up to N elements of a row from column c, zeros past its end.
template <typename T, int N>
__device__ __forceinline__ void load_part(const T* row, int64_t c, int64_t cols, T* v) {
  if (c + N <= cols) {
    load_n<T, N>(row + c, v);
  } else {
    for (int j = 0; j < N; ++j) v[j] = c + j < cols ? row[c + j] : from_f32<T>(0.0f);
  }
}
template <typename T, int N>
__device__ __forceinline__ void store_part(T* row, int64_t c, int64_t cols, const T* v) {
  if (c + N <= cols) {
    store_n<T, N>(row + c, v);
  } else {
    for (int j = 0; j < N; ++j)
      if (c + j < cols) row[c + j] = v[j];
  }
}

// A wave takes 4 x 64 x 16 bytes of a token's row and writes them to the rows of all
// its choices: each token is read once, where a copy by sorted row reads it once
// for every expert, on as many XCDs (8192 tokens of 2048 to 4 of 64 experts: 27 us,
// by sorted row 39).  Bound: memory, 168 MB at 6.2 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void gather_kernel(RowArgs a) {
  constexpr int N = 16 / sizeof(T), kSteps = 4;
  const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = a.first + item / a.parts, c0 = item % a.parts * (64 * N * kSteps) + (threadIdx.x & 63) * N;
  if (t >= a.x_rows) return;
  T v[kSteps][N];
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
    if (c0 + i * 64 * N < a.cols) load_part<T, N>((const T*)a.x + t * a.ld_x, c0 + i * 64 * N, a.cols, v[i]);
  for (int j = 0; j < a.k; ++j) {
    const int64_t r = a.index[t * a.k + j];
    if (r < 0 || r >= a.rows) continue;
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      if (c0 + i * 64 * N < a.cols) store_part<T, N>((T*)a.out + r * a.ld_out, c0 + i * 64 * N, a.cols, v[i]);
  }
  // rows of no slot
  int64_t r = a.offsets[a.experts];
  for (r = (r < 0 ? 0 : r) + t; r < a.rows; r += a.x_rows) {
    T zero[N];
    for (int j = 0; j < N; ++j) zero[j] = from_f32<T>(0.0f);
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      if (c0 + i * 64 * N < a.cols) store_part<T, N>((T*)a.out + r * a.ld_out, c0 + i * 64 * N, a.cols, zero);
  }
}

constexpr int kRowsAtOnce = 4;  // rows of h in flight

// A wave sums 512 columns of a token.  Bound: memory (8192 tokens of 4 times 2048
// columns: 32.6 us, 5.2 TB/s; 32 tokens 3.5 us, which is the launch and two trips).
template <typename T>
__global__ __launch_bounds__(256) void combine_kernel(RowArgs a) {
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t t = a.first + item / a.parts, c = item % a.parts * 512 + (threadIdx.x & 63) * 8;
  if (t >= a.rows || c >= a.cols) return;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int j0 = 0; j0 < a.k; j0 += kRowsAtOnce) {
    T v[kRowsAtOnce][8];
    float w[kRowsAtOnce];
    bool there[kRowsAtOnce];
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      const int64_t s = t * a.k + j0 + i;
      const int64_t p = j0 + i < a.k ? a.index[s] : -1;
      there[i] = p >= 0 && p < a.x_rows;
      w[i] = there[i] && a.weights ? a.weights[s] : 1.0f;
      if (there[i]) load_part<T, 8>((const T*)a.x + p * a.ld_x, c, a.cols, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i)
      if (there[i])
        for (int e = 0; e < 8; ++e) sum[e] = fmaf(w[i], to_f32(v[i][e]), sum[e]);
  }
  T r[8];
  for (int e = 0; e < 8; ++e) r[e] = from_f32<T>(sum[e]);
  store_part<T, 8>((T*)a.out + t * a.ld_out, c, a.cols, r);
}

// A workgroup takes a token: its gradient row is read once for four of its
// experts at a time, scaled into their rows, and multiplied with what they had
// given.  Dot products: a lane's columns, then the lanes by a tree, then the
// waves in order; always the same order.  Bound: memory (8192 tokens of 4 times 2048
// columns: 302 MB in 51 us back to back, 5.9 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void combine_gradient_kernel(RowArgs a) {
  __shared__ float part[4][kRowsAtOnce];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
  const int64_t t = a.first + blockIdx.x;
  const T* dy = (const T*)a.dy + t * a.ld_dy;
  for (int j0 = 0; j0 < a.k; j0 += kRowsAtOnce) {
    int64_t p[kRowsAtOnce];
    float w[kRowsAtOnce], dot[kRowsAtOnce];
    bool there[kRowsAtOnce];
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      const int64_t s = t * a.k + j0 + i;
      p[i] = j0 + i < a.k ? a.index[s] : -1;
      there[i] = p[i] >= 0 && p[i] < a.x_rows;
      w[i] = there[i] && a.weights ? a.weights[s] : 1.0f;
      dot[i] = 0.0f;
    }
    for (int64_t c = tid * 8; c < a.cols; c += blockDim.x * 8) {
      T d[8], h[kRowsAtOnce][8];
      load_part<T, 8>(dy, c, a.cols, d);
#pragma unroll
      for (int i = 0; i < kRowsAtOnce; ++i)
        if (there[i] && a.dweights) load_part<T, 8>((const T*)a.x + p[i] * a.ld_x, c, a.cols, h[i]);
#pragma unroll
      for (int i = 0; i < kRowsAtOnce; ++i)
        if (there[i]) {
          T r[8];
          for (int e = 0; e < 8; ++e) r[e] = from_f32<T>(w[i] * to_f32(d[e]));
          store_part<T, 8>((T*)a.out + p[i] * a.ld_out, c, a.cols, r);
          if (a.dweights)
            for (int e = 0; e < 8; ++e) dot[i] = fmaf(to_f32(d[e]), to_f32(h[i][e]), dot[i]);
        }
    }
    if (a.dweights) {
#pragma unroll
      for (int i = 0; i < kRowsAtOnce; ++i) {
        for (int d = 32; d; d /= 2) dot[i] += __shfl_xor(dot[i], d);
        if (lane == 0) part[wave][i] = dot[i];
      }
      __syncthreads();
      if (tid < kRowsAtOnce && j0 + tid < a.k) {
        float sum = part[0][tid];
        for (int v = 1; v < waves; ++v) sum += part[v][tid];
        a.dweights[t * a.k + j0 + tid] = sum;
      }
      __syncthreads();
    }
  }
  // rows of no slot
  int64_t r = a.offsets[a.experts];
  T zero[8];
  for (int e = 0; e < 8; ++e) zero[e] = from_f32<T>(0.0f);
  for (r = (r < 0 ? 0 : r) + t; r < a.x_rows; r += a.rows)
    for (int64_t c = tid * 8; c < a.cols; c += blockDim.x * 8) store_part<T, 8>((T*)a.out + r * a.ld_out, c, a.cols, zero);
}

#define WSG_BY_TYPE(dtype, kernel) \
  ((dtype) == WS_OUT_F32 ? &kernel<float> : (dtype) == WS_OUT_BF16 ? &kernel<bf16_t> : &kernel<f16_t>)

// Launches kernel(a) for all tokens, each of which has `parts` items; a workgroup of
// `block` threads takes `items` of them.  What one launch does not hold, in turn.
ws_status launch_tokens(const char* what, void (*kernel)(RowArgs), int64_t tokens, int64_t parts, int items, int block,
                        hipStream_t stream, RowArgs a) {
  const int64_t most = max_workgroups(block) / parts * items;  // whole workgroups
  for (a.first = 0; a.first < tokens; a.first += most) {
    const int64_t n = tokens - a.first < most ? tokens - a.first : most;
    const ws_status s = launch(what, kernel, ceil_div(n * parts, items), block, 0, stream, a);
    if (s != WS_OK) return s;
  }
  return WS_OK;
}

bool sort_sizes(int64_t tokens, int32_t k, int32_t experts) {
  return tokens >= 0 && k >= 1 && experts >= 1 && experts <= WS_MAX_EXPERTS && tokens <= kMaxDim && tokens * k <= kMaxDim;
}

// Slots of a workgroup.  Beyond what one sorts alone, small chunks for short kernels
// (32768 slots of 64 experts as 64 chunks: 9.5 us, as 16: 11.5), but not so many that
// summing their counts takes longer (131072 slots of 1024 experts as 64 chunks: 21
// us, as 256: 34); then whole rounds of loads, and at last kSortBlocks of what it takes.
int64_t sort_chunk(int64_t slots) {
  const auto chunk = [&](int64_t blocks) { return ceil_div(ceil_div(slots, blocks), kSortThreads) * kSortThreads; };
  if (slots <= kSortAlone) return chunk(1);
  const int64_t few = chunk(64), most = chunk(kSortBlocks);
  return most > kSortChunk ? most : few < kSortChunk ? few : kSortChunk;
}

bool plain(const ws_matrix* m) { return valid(m) && m->batch <= 1; }

}  // namespace
}  // namespace wsg

using namespace wsg;

extern "C" {

int64_t ws_expert_sort_workspace(int64_t tokens, int32_t k, int32_t experts) {
  if (!sort_sizes(tokens, k, experts)) return -1;
  const int64_t slots = tokens * k;
  return slots <= kSortAlone ? 0 : ceil_div(slots, sort_chunk(slots)) * experts * 4;
}

ws_status ws_expert_sort(int64_t tokens, int32_t k, int32_t experts, const void* ids, int32_t id_bytes,
                         int32_t* offsets, int32_t* token, int32_t* place, void* workspace, int64_t workspace_bytes,
                         hipStream_t stream) {
  const int64_t need = ws_expert_sort_workspace(tokens, k, experts);
  if (need < 0 || (id_bytes != 4 && id_bytes != 8) || !offsets || (uintptr_t)offsets % 4 || workspace_bytes < need ||
      (need > 0 && (!workspace || (uintptr_t)workspace % 4)))
    return WS_ERR_INVALID_ARG;
  if (tokens > 0 && (!ids || !token || !place || (uintptr_t)ids % id_bytes || (uintptr_t)token % 4 || (uintptr_t)place % 4))
    return WS_ERR_INVALID_ARG;
  SortArgs a{};
  a.ids = ids;
  a.slots = tokens * k;
  a.chunk = sort_chunk(a.slots);
  a.blocks = a.slots > 0 ? ceil_div(a.slots, a.chunk) : 1;  // without slots the offsets are written all the same
  a.k = k;
  a.experts = experts;
  a.id_bytes = id_bytes;
  while ((1 << a.bits) < experts) ++a.bits;
  a.offsets = offsets;
  a.token = token;
  a.place = place;
  const int count_lds = kSortWaves * experts * 4, place_lds = count_lds + experts * 4 + kSortWaves * 4;
  if (a.slots <= kSortAlone) return launch("expert_sort", &place_kernel<true>, 1, kSortThreads, place_lds, stream, a);
  a.counts = (int32_t*)workspace;
  const ws_status s = launch("expert_sort", &count_kernel, a.blocks, kSortThreads, count_lds, stream, a);
  return s != WS_OK ? s : launch("expert_sort", &place_kernel<false>, a.blocks, kSortThreads, place_lds, stream, a);
}

ws_status ws_expert_gather(const ws_matrix* x, int32_t k, int32_t experts, const int32_t* offsets, const int32_t* place,
                           const ws_matrix* out, hipStream_t stream) {
  if (!plain(x) || !plain(out) || x->cols != out->cols || x->dtype != out->dtype || k < 1 || experts < 1) return WS_ERR_INVALID_ARG;
  if (x->rows == 0) return out->rows == 0 ? WS_OK : WS_ERR_INVALID_ARG;  // no tokens: no rows of theirs
  if (out->rows == 0 || out->cols == 0) return WS_OK;
  if (!offsets || !place || (uintptr_t)offsets % 4 || (uintptr_t)place % 4) return WS_ERR_INVALID_ARG;
  RowArgs a{};
  a.x = x->data;
  a.out = out->data;
  a.index = place;
  a.offsets = offsets;
  a.x_rows = x->rows;
  a.rows = out->rows;
  a.cols = out->cols;
  a.ld_x = x->ld;
  a.ld_out = out->ld;
  a.k = k;
  a.experts = experts;
  a.parts = (int32_t)ceil_div(a.cols * elem_size(x->dtype), 4096);
  return launch_tokens("expert_gather", elem_size(x->dtype) == 4 ? &gather_kernel<float> : &gather_kernel<bf16_t>, a.x_rows, a.parts, 4,
                       256, stream, a);
}

ws_status ws_expert_combine(const ws_matrix* h, int32_t k, const int32_t* place, const float* weights,
                            const ws_matrix* out, hipStream_t stream) {
  if (!plain(h) || !plain(out) || h->cols != out->cols || h->dtype != out->dtype || k < 1 || (uintptr_t)weights % 4)
    return WS_ERR_INVALID_ARG;
  if (out->rows == 0 || out->cols == 0) return WS_OK;
  if (!place || (uintptr_t)place % 4) return WS_ERR_INVALID_ARG;
  RowArgs a{};
  a.x = h->data;
  a.out = out->data;
  a.index = place;
  a.weights = weights;
  a.x_rows = h->rows;
  a.rows = out->rows;
  a.cols = out->cols;
  a.ld_x = h->ld;
  a.ld_out = out->ld;
  a.k = k;
  a.parts = (int32_t)ceil_div(a.cols, 512);
  return launch_tokens("expert_combine", WSG_BY_TYPE(h->dtype, combine_kernel), a.rows, a.parts, 4, 256, stream, a);
}

ws_status ws_expert_combine_gradient(const ws_matrix* dy, const ws_matrix* h, int32_t k, int32_t experts,
                                     const int32_t* offsets, const int32_t* place, const float* weights,
                                     const ws_matrix* dh, float* dweights, hipStream_t stream) {
  if (!plain(dy) || !plain(dh) || dy->cols != dh->cols || dy->dtype != dh->dtype || k < 1 || experts < 1 ||
      (uintptr_t)weights % 4 || (uintptr_t)dweights % 4)
    return WS_ERR_INVALID_ARG;
  if (dweights && (!plain(h) || h->rows != dh->rows || h->cols != dh->cols || h->dtype != dh->dtype))
    return WS_ERR_INVALID_ARG;
  if (dy->rows == 0) {  // no tokens: no rows of theirs
    if (dh->rows != 0) return WS_ERR_INVALID_ARG;
    return WS_OK;
  }
  if (!offsets || !place || (uintptr_t)offsets % 4 || (uintptr_t)place % 4) return WS_ERR_INVALID_ARG;
  RowArgs a{};
  a.x = dweights ? h->data : nullptr;
  a.dy = dy->data;
  a.out = dh->data;
  a.index = place;
  a.offsets = offsets;
  a.weights = weights;
  a.dweights = dweights;
  a.x_rows = dh->rows;
  a.rows = dy->rows;
  a.cols = dy->cols;
  a.ld_x = dweights ? h->ld : 0;
  a.ld_dy = dy->ld;
  a.ld_out = dh->ld;
  a.k = k;
  a.experts = experts;
  const int block = a.cols <= 512 ? 64 : a.cols <= 1024 ? 128 : 256;
  return launch_tokens("expert_combine_gradient", WSG_BY_TYPE(dy->dtype, combine_gradient_kernel), a.rows, 1, 1, block, stream, a);
}

}  // extern "C"
