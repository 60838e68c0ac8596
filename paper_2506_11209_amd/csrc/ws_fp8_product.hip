// The block-scaled 8-bit product and its grouped forms (definitions: ws_fp8.h).
//
// Two matrix instructions, chosen by the type of the result:
//
//  * 16 bits: v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 codes with
//    16 x 128 codes and applies an E8M0 scale to each operand row, so a scale
//    of 128 columns costs no arithmetic of its own and accumulation runs on in
//    binary32 across blocks.  It adds products in groups of eight neighbouring
//    columns, each group aligned to its largest product with 13 bits below that
//    product's leading one, the rest cut (measured with single products; the older
//    8-bit instructions do the same); the groups' sums add up in binary32.  Taken
//    for the rate: measured before the rounding, it is 1.5e-5 of the result in norm
//    on normal values and 4.6e-5 where one column in a hundred is 20 times larger,
//    beside a rounding of 1.7e-3 (bf16) or 2.1e-4 (f16).
//  * 32 bits: v_mfma_f32_16x16x32_bf16 on the codes' values, which bf16 holds
//    exactly (scale included, from 2^-126 on): half the rate, and the sums are
//    binary32 throughout.
//
// Lane l holds 32 bytes of row l % 16; which columns of the 128 those are is
// free, because both operands are loaded alike and one scale covers them all:
// lane group l / 16 takes bytes 16 g .. and 64 + 16 g .. , so that each load of
// a wave covers 64 neighbouring bytes of every row.  The operands are passed in
// exchanged order (B's rows first): a lane then ends up with four neighbouring
// columns of one row of C.
#include <math.h>

#include <atomic>
#include <type_traits>

#include "ws_fp8_common.hpp"

namespace wsg {
namespace {

enum { kDense = 0, kRowGroups = 1, kDepthGroups = 2 };

struct ProductArgs {
  const uint8_t *A, *B, *sa, *sb;
  const void* C0;
  void* C;
  int64_t lda, ldb, ldsa, ldsb, ldc, ldc0;
  int64_t stride_b, stride_sb, stride_c, stride_c0;  // between groups
  int64_t M, N, K;   // K: a multiple of 16
  int32_t b_shift;   // log2 of B's rows that share a scale
  int32_t dtype;     // of C and C0
  float alpha, beta;
  const int32_t* offsets;
  int32_t groups;
  int64_t depth_rows;  // kDepthGroups: rows that the groups cut
  int64_t tiles_m, tiles_n;
  int32_t tile_groups;  // workgroups that take tiles of a tile kernel; those behind them
  int32_t rest_rows;    // take rows M .. rest_end - 1, rest_rows x 16 each (dense products)
  int64_t rest_end;
};

// What one workgroup computes: rows m0 .. m_end - 1 (at most a tile) of its
// product, contracted over K columns of the operands at A, B, sa, sb.
struct Part {
  const uint8_t *A, *B, *sa, *sb;
  int64_t m0, m_end, n0, K, c_at, c0_at;
  bool zero;  // rows of no group: nothing to multiply
};

template <int MODE>
__device__ __forceinline__ bool find_part(const ProductArgs& a, int64_t tm, int64_t tn, int64_t group, int TM, int TN, Part* p) {
  *p = Part{a.A, a.B, a.sa, a.sb, tm * TM, a.M, tn * TN, a.K, 0, 0, false};
  if constexpr (MODE == kRowGroups) {
    const GroupTile gt = find_group_tile(a.offsets, a.groups, a.M, TM, tm);
    if (gt.group < 0) return false;
    p->m0 = gt.lo + gt.index * TM;
    p->m_end = gt.hi;
    p->zero = gt.group >= a.groups;
    if (!p->zero) {
      p->B += gt.group * a.stride_b;
      p->sb += gt.group * a.stride_sb;
    }
  }
  if constexpr (MODE == kDepthGroups) {
    // columns of the groups before this one, each rounded up to 128
    const int lane = threadIdx.x & 63;
    int64_t before = 0, mine = 0;
    for (int first = 0; first <= (int)group; first += 64) {
      const int i = first + lane;
      int64_t n = 0;
      if (i <= (int)group) {
        int64_t lo, hi;
        group_rows(a.offsets, a.groups, a.depth_rows, i, &lo, &hi);
        n = (hi - lo + kBlock - 1) / kBlock;
      }
      if (i == (int)group) mine = n;
      before += i < (int)group ? n : 0;
    }
    for (int d = 32; d; d /= 2) {
      before += __shfl_xor(before, d);
      mine += __shfl_xor(mine, d);
    }
    before = uniform(before);
    mine = uniform(mine);
    const int64_t blocks = a.K / kBlock;
    before = before > blocks ? blocks : before;
    mine = mine > blocks - before ? blocks - before : mine;
    p->A += before * kBlock;
    p->B += before * kBlock;
    p->sa += before * a.ldsa;
    p->sb += before * a.ldsb;
    p->K = mine * kBlock;
    p->c_at = group * a.stride_c;
    p->c0_at = group * a.stride_c0;
  }
  return true;
}

// Up to so many groups, one for each lane of a wave, are put in order of their depths.
// 16384 rows, on average over six draws of the depths, us in the groups' own order and
// in that of their depths: 1024 x 2048 in 16 groups 97.6 and 89.2, in 32 134.8 and
// 133.2, in 64 217 and 212; 512 x 512, where the order costs as much as it saves, 28.3
// and 25.2, 25.9 and 26.1, 29.6 and 30.6.
constexpr int kRanked = 64;

// How many groups are deeper than this lane's, or as deep and before it; -1 for a lane
// without a group.
__device__ __forceinline__ int rank_of_depth(const ProductArgs& a) {
  const int lane = threadIdx.x & 63;
  if (a.groups > kRanked) return 0;
  int depth = -1, rank = 0;
  if (lane < a.groups) {
    int64_t lo, hi;
    group_rows(a.offsets, a.groups, a.depth_rows, lane, &lo, &hi);
    depth = (int)((hi - lo + kBlock - 1) / kBlock);
  }
  for (int i = 0; i < a.groups; ++i) {
    const int other = __builtin_amdgcn_readlane(depth, i);
    rank += other > depth || (other == depth && i < lane);
  }
  return lane < a.groups ? rank : -1;
}

// Four neighbouring columns of row m from n (columns up to N), rounded once.
template <typename T>
__device__ __forceinline__ void store4(const ProductArgs& a, const Part& p, int64_t m, int64_t n, const float* acc) {
  T* c = (T*)a.C + p.c_at + m * a.ldc + n;
  const T* c0 = (const T*)a.C0 + p.c0_at + m * a.ldc0 + n;
  float v[4];
  for (int j = 0; j < 4; ++j) v[j] = a.alpha * acc[j];
  T r[4];
  if (n + 4 <= a.N) {
    if (a.beta != 0.0f) {
      load_n<T, 4>(c0, r);
      for (int j = 0; j < 4; ++j) v[j] = fmaf(a.beta, to_f32(r[j]), v[j]);
    }
    for (int j = 0; j < 4; ++j) r[j] = from_f32<T>(v[j]);
    store_n<T, 4>(c, r);
  } else {
    for (int j = 0; j < 4; ++j)
      if (n + j < a.N) {
        if (a.beta != 0.0f) v[j] = fmaf(a.beta, to_f32(c0[j]), v[j]);
        c[j] = from_f32<T>(v[j]);
      }
  }
}
__device__ __forceinline__ void store_out(const ProductArgs& a, const Part& p, int64_t m, int64_t n, const float* acc) {
  switch (a.dtype) {  // the same for the whole launch
    case WS_OUT_F32: return store4<float>(a, p, m, n, acc);
    case WS_OUT_BF16: return store4<bf16_t>(a, p, m, n, acc);
    default: return store4<f16_t>(a, p, m, n, acc);
  }
}

constexpr uint32_t kOutside = 0x80000000u;  // an offset past every buffer: reads zeros

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const uint8_t* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), (short)0, (int)bytes, 0x00027000);
}
__device__ __forceinline__ i32x4_t load16(__amdgpu_buffer_rsrc_t r, uint32_t at) {
  return __builtin_bit_cast(i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
}
__device__ __forceinline__ i32x8_t join(i32x4_t lo, i32x4_t hi) {
  return i32x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

template <int N, typename F>
__device__ __forceinline__ void static_for(const F& f) {
  if constexpr (N > 0) {
    static_for<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// 2^(byte - 127); 2^-127 is subnormal.
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(max(byte << 23, 1u << 22)); }

// Eight codes (two dwords) times a scale, exactly.
__device__ __forceinline__ bf16x8_t widen(int lo, int hi, float scale) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// acc += A's 16 rows times B's 16 rows, where the sum is, and two wait states after
// what widened the operands: the compiler's own form leaves sums on their way in
// registers that it uses again right behind a product.
__device__ __forceinline__ void multiply_in_place(f32x4_t& acc, const bf16x8_t& fa, const bf16x8_t& fb) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(fb), "v"(fa));
#endif
}

// -- few rows --------------------------------------------------------------------

// A workgroup computes 16 MT rows of 16 columns; its waves share out the blocks
// of the contraction and add up their parts through LDS in a fixed order.
// Operands go from memory straight to registers, U blocks at a time.  For few
// rows: bound by reading B once (1 x 8192 x 8192: 13 to 15 us, 5 TB/s).
// IN_TILE: more than 16 rows inside a tile kernel.
template <int MT, int U, bool WIDE, bool AGPR = false, bool IN_TILE = false>
__device__ __forceinline__ void direct_part(const ProductArgs& a, const Part& p, float* lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int waves = blockDim.x >> 6, r = lane & 15, g = lane >> 4;
  const int rows = (int)min(p.m_end - p.m0, (int64_t)16 * MT), cols = (int)min(a.N - p.n0, (int64_t)16);
  f32x4_t acc[MT];
  for (int i = 0; i < MT; ++i) acc[i] = f32x4_t{0, 0, 0, 0};
  const int blocks = p.zero ? 0 : (int)((p.K + kBlock - 1) / kBlock);
  const __amdgpu_buffer_rsrc_t ra = buffer(p.A + p.m0 * a.lda, (uint32_t)(rows * a.lda));
  const __amdgpu_buffer_rsrc_t rb = buffer(p.B + p.n0 * a.ldb, (uint32_t)(cols * a.ldb));
  const uint8_t* sb = p.sb + ((p.n0 + min(r, cols - 1)) >> a.b_shift);
  for (int b0 = wave; b0 < blocks; b0 += waves * U) {
    i32x4_t vb[U][2], va[U][MT][2];
    int sbv[U], sav[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int b = b0 + u * waves, bs = min(b, blocks - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = b * kBlock + 64 * h + 16 * g;
        const bool in = k < p.K;  // whole chunks: K is a multiple of 16
        vb[u][h] = load16(rb, in ? (uint32_t)(r * a.ldb + k) : kOutside);
        for (int i = 0; i < MT; ++i) va[u][i][h] = load16(ra, in ? (uint32_t)((16 * i + r) * a.lda + k) : kOutside);
      }
      sbv[u] = sb[bs * a.ldsb];
      for (int i = 0; i < MT; ++i) sav[u][i] = p.sa[bs * a.ldsa + p.m0 + min(16 * i + r, rows - 1)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (WIDE) {
        for (int h = 0; h < 2; ++h)
          for (int q = 0; q < 4; q += 2) {
            const bf16x8_t wb = widen(vb[u][h][q], vb[u][h][q + 1], scale_value(sbv[u]));
            for (int i = 0; i < MT; ++i) {
              const bf16x8_t wa = widen(va[u][i][h][q], va[u][i][h][q + 1], scale_value(sav[u][i]));
              if constexpr (IN_TILE) multiply_in_place(acc[i], wa, wb);
              else acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, wa, acc[i], 0, 0, 0);
            }
          }
        continue;
      }
      for (int i = 0; i < MT; ++i)
        acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(join(vb[u][0], vb[u][1]), join(va[u][i][0], va[u][i][1]),
                                                                  acc[i], 0, 0, 0, sbv[u], 0, sav[u][i]);
    }
    // Inside the tile kernels sums stay in one kind of register, and keep the longest
    // wait before anything else reads them, as those of their products in asm do.
#if defined(__HIP_DEVICE_COMPILE__)
    for (int i = 0; i < MT; ++i) {
      if constexpr (AGPR) asm volatile("s_nop 15\n\ts_nop 2" : "+a"(acc[i]));
      else asm volatile("s_nop 15\n\ts_nop 2" : "+v"(acc[i]));
    }
#endif
  }
  // lane: row l % 16 of C's tile, columns 4 (l / 16) ..
  f32x4_t* part = (f32x4_t*)lds;
  for (int i = 0; i < MT; ++i) part[(wave * MT + i) * 64 + lane] = acc[i];
  __syncthreads();
  for (int j = tid; j < 64 * MT; j += blockDim.x) {
    f32x4_t sum = part[j];
    for (int w = 1; w < waves; ++w) sum += part[w * MT * 64 + j];
    const int row = j / 64 * 16 + (j & 15), col = (j & 63) >> 4;
    float v[4] = {sum[0], sum[1], sum[2], sum[3]};
    if (row < rows && 4 * col < cols) store_out(a, p, p.m0 + row, p.n0 + 4 * col, v);
  }
}

template <int MT, int U, int MODE, bool WIDE>
__global__ __launch_bounds__(512) void direct_kernel(ProductArgs a) {  // kDirectThreads
  extern __shared__ float lds[];
  const int64_t tn = blockIdx.x % a.tiles_n, t = blockIdx.x / a.tiles_n;
  Part p;
  if (find_part<MODE>(a, MODE == kDepthGroups ? t % a.tiles_m : t, tn, MODE == kDepthGroups ? t / a.tiles_m : 0, 16 * MT, 16, &p))
    direct_part<MT, U, WIDE>(a, p, lds);
}

// -- tiles -----------------------------------------------------------------------

#define WSG_LDS __attribute__((address_space(3)))

// Byte position, in a row of 128, of 16-byte chunk c of tile row r.  The operand
// read (lane l: row l % 16, chunk l / 16 or four more) is free of bank conflicts
// so; with (r ^ r / 8 % 2) % 8, which suits reads of 32 rows, it took twice as long
// (SQ_LDS_BANK_CONFLICT).  The choice depends on r % 16 only, which is fixed for
// a lane.
__device__ __forceinline__ int chunk_at(int r, int c) { return (c ^ (r & 7)) * 16; }

// A buffer descriptor as four scalars, for asm.
__device__ __forceinline__ i32x4_t raw_buffer(const uint8_t* base, uint32_t bytes) {
  const uint64_t at = (uint64_t)base;
  return i32x4_t{(int)__builtin_amdgcn_readfirstlane((uint32_t)at), (int)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)),
                 (int)__builtin_amdgcn_readfirstlane(bytes), 0x00027000};
}

// 64 lanes' 16 bytes from buffer offsets `at` + k straight to 1 KiB of LDS at
// `to` (zeros where `at` is outside).  As asm, so that the compiler does not wait
// for it before LDS reads of other addresses; whoever reads what it brings waits
// for vmcnt himself.  Nothing else in these kernels uses m0.
__device__ __forceinline__ void load_to_lds(i32x4_t r, uint32_t at, uint32_t k, uint32_t to) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile(
      "s_mov_b32 m0, %3\n\t"
      "s_nop 0\n\t"
      "buffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(at),
      "s"(r), "s"(__builtin_amdgcn_readfirstlane(k)), "s"(__builtin_amdgcn_readfirstlane(to)));
#endif
}

// Waits for this wave's LDS accesses and all but its last YOUNGER loads, then for
// the workgroup.
template <int YOUNGER = 0>
__device__ __forceinline__ void drain_and_meet() {
  static_assert(YOUNGER >= 0 && YOUNGER <= 63, "vmcnt");
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(YOUNGER) : "memory");
#endif
}

template <int WM, int WN, int STAGES>
struct TileShape {
  static constexpr int TM = 32 * WM, TN = 32 * WN, kStage = (TM + TN) * kBlock;
  // One wave a SIMD with sums in accumulation registers, or more with all in the others.
  static constexpr int kWaves = WM * WN > 16 || STAGES * kStage > 80 * 1024 ? 1 : 2;
  static constexpr bool kAgpr = WM * WN > 16;
  // Last rows of a product beside the tiles, more than 16 of them to a workgroup.
  static constexpr bool kDeepRest = STAGES == 2 && kWaves == 2;
  // Rows of products before a block's meeting point.  Few: the loads of the block
  // after next, which keep the address unit busy for half a block of 256 x 256,
  // spread over more products behind it.
  static constexpr int kFirst = WM * WN > 32 ? 3 : WM / 2;
  // Two stages: a thread brings the scales of its rows of the tile block by block;
  // more: those of kDeep blocks at a time lie in LDS.
  static constexpr int kMine = (TM + TN + 255) / 256, kDeep = STAGES == 2 ? 2 : 32;
  // LDS: the stages, the scales, and for every wave 16 rows of what it stores at a
  // time, as many columns as fit
  static constexpr int kScalesAt = STAGES * kStage, kStoreAt = kScalesAt + kDeep * (TM + TN);
  static constexpr int kStoreCols = kWaves == 1 && WN >= 4 ? 64 : 32, kStoreParts = 16 * WN / kStoreCols;
  static constexpr int kPitch = kStoreCols + 4;  // the pitch spreads rows over the banks
  static constexpr int kStoreBytes = 16 * kPitch * 4, kLds = kStoreAt + 4 * kStoreBytes;
  static_assert(kWaves * kLds <= 160 * 1024, "LDS of a CU");
};

// Keeps what reads acc behind the asm statements before, the wait for the last
// products among them.
template <bool AGPR>
__device__ __forceinline__ void settle(f32x4_t& acc) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (AGPR) asm volatile("" : "+a"(acc));
  else asm volatile("" : "+v"(acc));
#endif
}

// Writes a wave's part of a tile, 16 rows at a time by way of its own part of LDS,
// so that a store covers whole stretches of a row.  Where nothing is added, and the
// columns are whole 16-byte pieces, the rows are rounded before LDS and leave in
// such pieces, at addresses that differ by scalars only; else they pass LDS in
// binary32.
// rows, cols: of the tile, inside C.
template <typename T, int WM, int WN, int STAGES>
__device__ __forceinline__ void store_tile(const ProductArgs& a, const Part& p, f32x4_t (&acc)[WM][WN], uint8_t* own, int wm, int wn,
                                           int rows, int cols) {
  typedef TileShape<WM, WN, STAGES> Shape;
  constexpr int kCols = Shape::kStoreCols, kPitch = Shape::kPitch, kTiles = kCols / 16;
  constexpr int N = 16 / sizeof(T), kRow = kCols * (int)sizeof(T) + 16, kPieces = kCols / N, kAtOnce = 64 / kPieces;  // kRow: bytes
  static_assert(16 * kRow <= Shape::kStoreBytes && 64 % kPieces == 0 && 16 % kAtOnce == 0, "16 rows in whole stores");
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const bool plain = a.beta == 0.0f && a.ldc <= (1 << 22) && cols % N == 0;
  const bool whole = rows == Shape::TM && cols == Shape::TN;
  const int rows_left = rows - wm * 16 * WM - lane / kPieces;
  bool in_cols[Shape::kStoreParts];
#pragma unroll
  for (int h = 0; h < Shape::kStoreParts; ++h) in_cols[h] = wn * 16 * WN + h * kCols + lane % kPieces * N < cols;
  const uint32_t ld = (uint32_t)a.ldc * (uint32_t)sizeof(T);  // bytes; used where plain
  uint8_t* const to = (uint8_t*)a.C + uniform((p.c_at + (p.m0 + wm * 16 * WM) * a.ldc + p.n0 + wn * 16 * WN) * (int64_t)sizeof(T));
  const uint32_t mine = lane / kPieces * ld + lane % kPieces * 16;
  const uint8_t* const from = own + lane / kPieces * kRow + lane % kPieces * 16;
#pragma unroll
  for (int i = 0; i < WM; ++i)
#pragma unroll
    for (int h = 0; h < Shape::kStoreParts; ++h) {
#pragma unroll
      for (int j = 0; j < kTiles; ++j) settle<Shape::kAgpr>(acc[i][h * kTiles + j]);
      if (plain) {
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          T t[4];
          for (int k = 0; k < 4; ++k) t[k] = from_f32<T>(a.alpha * acc[i][h * kTiles + j][k]);
          __builtin_memcpy(__builtin_assume_aligned(own + r * kRow + (16 * j + 4 * g) * sizeof(T), 4 * sizeof(T)), t, sizeof(t));
        }
        __builtin_amdgcn_wave_barrier();  // a wave's LDS accesses keep their order
#pragma unroll
        for (int e = 0; e < 16; e += kAtOnce) {
          T t[N];
          __builtin_memcpy(t, __builtin_assume_aligned(from + e * kRow, 16), 16);
          T* c = (T*)(to + (uint64_t)(16 * i + e) * ld + h * kCols * sizeof(T) + mine);
          if (whole) store_n<T, N>(c, t);
          else if (in_cols[h] && 16 * i + e < rows_left) store_n<T, N>(c, t);
        }
      } else {
        float* f = (float*)own;
        const int n0 = wn * 16 * WN + h * kCols;
#pragma unroll
        for (int j = 0; j < kTiles; ++j) *(f32x4_t*)(f + r * kPitch + 16 * j + 4 * g) = acc[i][h * kTiles + j];
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int e = lane; e < 4 * kCols; e += 64) {
          const int row = (wm * WM + i) * 16 + e / (kCols / 4), at = e % (kCols / 4) * 4, col = n0 + at;
          float v[4];
          *(f32x4_t*)v = *(const f32x4_t*)(f + e / (kCols / 4) * kPitch + at);
          if (row < rows && col < cols) store4<T>(a, p, p.m0 + row, p.n0 + col, v);
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
}

// acc += A's 16 rows times B's 16 rows, each operand's scale in byte SA or SB of
// its dword.  As asm with the sum in place: the compiler's own form of it moved
// sums between registers (4 copies and a wait for each of a row's products), and
// what has no side effects does not stay on its side of a barrier.  An operand may
// not come from a VALU instruction less than two wait states before: fragments
// come from LDS, scales by way of settle_scales.
template <bool AGPR, int SA, int SB>
__device__ __forceinline__ void multiply(f32x4_t& acc, const i32x8_t& fa, const i32x8_t& fb, uint32_t sa, uint32_t sb) {
#if defined(__HIP_DEVICE_COMPILE__)
#define WSG_MULTIPLY(c)                                                                            \
  asm volatile(                                                                                    \
      "v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0]" \
      : c(acc)                                                                                     \
      : "v"(fb), "v"(fa), "v"(sb), "v"(sa), "n"(SB & 1), "n"(SA & 1), "n"(SB >> 1), "n"(SA >> 1))
  if constexpr (AGPR) WSG_MULTIPLY("+a");
  else WSG_MULTIPLY("+v");
#undef WSG_MULTIPLY
#endif
}

// The same for 32 of the 128 columns with operands widened to bf16.
template <bool AGPR>
__device__ __forceinline__ void multiply_wide(f32x4_t& acc, const i32x4_t& fa, const i32x4_t& fb) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (AGPR) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(fb), "v"(fa));
  else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(fb), "v"(fa));
#endif
}

// An operand just widened, two wait states before its first product.
__device__ __forceinline__ void settle_wide(i32x4_t& f) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 1" : "+v"(f));
#endif
}

// A quarter of an operand's 128 columns in bf16.
__device__ __forceinline__ i32x4_t widen_part(const i32x8_t& f, int q, float scale) {
  return __builtin_bit_cast(i32x4_t, widen(f[2 * q], f[2 * q + 1], scale));
}
// Byte i of packed scales.
__device__ __forceinline__ float scale_of(const uint32_t* scales, int i) { return scale_value(scales[i / 4] >> i % 4 * 8 & 255u); }

// Rows FROM .. FROM + N - 1 of a block's products in bf16.  Operands are widened a
// quarter at a time between products: A's rows along with the first column of B, a
// column of B, for all of the block, during the one before (FROM = 0), the first
// quarters of the NEXT rows of A during the last.  (All of a column's at once, by
// each half of the rows again, kept the matrix unit waiting: 8192 x 8192 x 8192 in
// 910 us, so 870.)
// between(j, q, i) is called behind every product.
template <bool AGPR, int FROM, int N, int NEXT, int WM, int WN, typename F>
__device__ __forceinline__ void multiply_rows_wide(f32x4_t (&acc)[WM][WN], const i32x8_t (&fa)[WM], const i32x8_t (&fb)[WN],
                                                   i32x4_t (&wa)[WM][4], i32x4_t (&wb)[WN][4], const uint32_t* sa,
                                                   const uint32_t* sb, const F& between) {
  constexpr bool kFresh = FROM == 0;  // B, and the first quarters of A, are still to be widened
  if constexpr (kFresh) {
    wb[0][0] = widen_part(fb[0], 0, scale_of(sb, 0));
#pragma unroll
    for (int i = 0; i < N; ++i) wa[i][0] = widen_part(fa[i], 0, scale_of(sa, i));
#pragma unroll
    for (int i = 0; i < N; ++i) settle_wide(wa[i][0]);
    settle_wide(wb[0][0]);
  }
  __builtin_amdgcn_sched_barrier(0);
  static_for<WN * 4>([&](auto sc) {
    constexpr int j = decltype(sc)::value / 4, q = decltype(sc)::value % 4;
    static_for<N>([&](auto ic) {
      constexpr int i = decltype(ic)::value, row = FROM + i;
      multiply_wide<AGPR>(acc[row][j], wa[row][q], wb[j][q]);
      if constexpr (j == 0 && q < 3) wa[row][q + 1] = widen_part(fa[row], q + 1, scale_of(sa, row));
      if constexpr (kFresh && j == 0 && q < 3 && i == 0) wb[0][q + 1] = widen_part(fb[0], q + 1, scale_of(sb, 0));
      if constexpr (kFresh && i == N / 2 && j + 1 < WN) wb[j + 1][q] = widen_part(fb[j + 1], q, scale_of(sb, j + 1));
      if constexpr (j == WN - 1) {
#pragma unroll
        for (int k = (q * N + i) * NEXT / (4 * N); k < (q * N + i + 1) * NEXT / (4 * N); ++k)
          wa[FROM + N + k][0] = widen_part(fa[FROM + N + k], 0, scale_of(sa, FROM + N + k));
      }
      between(std::integral_constant<int, j>{}, std::integral_constant<int, q>{}, ic);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (j == 0 && q < 3) {
      settle_wide(wa[FROM + N - 1][q + 1]);
      if constexpr (kFresh) settle_wide(wb[0][q + 1]);
    } else if constexpr (kFresh && q == 3 && j + 1 < WN) {
      settle_wide(wb[j + 1][3]);
    }
  });
#pragma unroll
  for (int k = 0; k < NEXT; ++k) settle_wide(wa[FROM + N + k][0]);
}

// Scales just moved, two wait states before their first product.
__device__ __forceinline__ void settle_scales(uint32_t& s) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_nop 1" : "+v"(s));
#endif
}

// A tile of 32 WM x 32 WN by four waves, 2 x 2, of WM x WN matrix instructions
// each.  Blocks of 128 columns are double-buffered in LDS, and a block's products
// come in two halves:
//
//   the first kFirst rows, row by row: the rest of A of block b is read
//   meet: b + 1 has landed everywhere, b has been read everywhere
//   the other rows, column by column: b + 2 is loaded over b; the first rows of A
//   of b + 1 are read, and every column of B of b + 1 once that of b is done
//
// so there is one barrier a block, no wait for memory that had less than a
// block's time, and one set of registers for each operand.  Scales lie in LDS as
// [row % 16][row / 16], so that a lane reads those of all its rows at once and
// the instruction picks a byte.  Small tiles have four stages, b + 4 being loaded
// over b: their blocks are shorter than the way to memory.
// WIDE: results in 32 bits, the same halves (multiply_rows_wide).
//
// A workgroup takes every tile_groups-th of an XCD's tiles.  It starts the loads of its
// next tile before it stores the one it has, in LDS of their own, so that memory
// is written and read at once; the next tile's first meeting waits for both.
//
// Bound: the matrix unit at the clock that its power leaves; 8192 x 8192 x 8192 in
// 370 to 430 us in 16 bits (256 x 256; 3.0 to 2.6 PFLOP/s by the operands' bits), in
// 875 in 32 bits (256 x 128).  Short contractions: the way to the first block and of
// the last sums to memory, 8 us a tile of 256 x 256 where all are written at once
// (8192 x 2 rows for 16 experts of 4096 x 2048: 163 us; without its stores 134).
template <int WM, int WN, int STAGES, int MODE, bool WIDE>
__global__ __launch_bounds__(256, (TileShape<WM, WN, STAGES>::kWaves)) void tile_kernel(ProductArgs a) {
  typedef TileShape<WM, WN, STAGES> Shape;
  constexpr int TM = Shape::TM, TN = Shape::TN, kStage = Shape::kStage, kRows = TM + TN, kFirst = Shape::kFirst, kRest = WM - kFirst;
  extern __shared__ __align__(1024) uint8_t smem[];
  if constexpr (MODE == kDense)
    if (blockIdx.x >= (uint32_t)a.tile_groups) {
      const uint32_t t = blockIdx.x - a.tile_groups, across = (uint32_t)((a.N + 15) / 16);
      const Part p{a.A, a.B, a.sa, a.sb, a.M + (int64_t)(t / across) * a.rest_rows, a.rest_end, t % across * 16, a.K, 0, 0, false};
      if constexpr (Shape::kDeepRest) {
        if (a.rest_rows == 64) return direct_part<4, 2, WIDE, false, true>(a, p, (float*)smem);
        if (a.rest_rows == 32) return direct_part<2, 4, WIDE, false, true>(a, p, (float*)smem);
      }
      return direct_part<1, 4, WIDE, Shape::kWaves == 1>(a, p, (float*)smem);
    }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4, wm = wave >> 1, wn = wave & 1;

  // Tiles: an XCD (workgroups go round them in turn) has a run of them, eight rows
  // of tiles at a time, so that those of one moment share operands in its L2.
  uint32_t tiles_m = (uint32_t)a.tiles_m;
  if (MODE == kRowGroups) tiles_m = (uint32_t)count_group_tiles(a.offsets, a.groups, a.M, TM);
  // Groups of unlike depth are dealt out instead, the deepest first, to the workgroups
  // in turn and back: with runs an XCD had two of 16 groups, and the one with the
  // deepest took twice as long as the others (16 x 1024 x 2048 over 16384 rows: 146 us;
  // dealt out in the groups' order 87 us on average over eight draws of the depths, the
  // deepest first 84; 5 x 1500 x 1500 over 8192 rows 53 and 46).
  const uint32_t tiles_n = (uint32_t)a.tiles_n, plane = tiles_m * tiles_n, tiles = plane * (MODE == kDepthGroups ? a.groups : 1);
  const uint32_t xcd = blockIdx.x % 8, share = tiles / 8, extra = tiles % 8, turns = (a.tile_groups + 7 - xcd) / 8;
  const uint32_t begin = xcd * share + min(xcd, extra), end = MODE == kDepthGroups ? tiles : begin + share + (xcd < extra);
  uint32_t round = 0;
  const auto next_id = [&]() -> uint32_t {
    const uint32_t n = round++;
    if constexpr (MODE == kDepthGroups) return n * a.tile_groups + (n & 1 ? a.tile_groups - 1 - blockIdx.x : blockIdx.x);
    return begin + blockIdx.x / 8 + n * turns;
  };
  uint32_t id = next_id();
  const int rank = MODE == kDepthGroups ? rank_of_depth(a) : 0;

  struct Tile {
    Part p;
    int rows, cols, K, blocks;
    i32x4_t ra, rb;
    const uint8_t* scale_at[Shape::kMine];
  } t;
  // loads: wave w takes the tile's row octets w, w + 4, ..
  const int lr = 8 * wave + (lane >> 3), lc = chunk_at(lr, lane & 7);  // chunk_at is its own inverse
  const uint32_t at_a = (uint32_t)(lr * a.lda + lc), at_b = (uint32_t)(lr * a.ldb + lc);
  const uint32_t step_a = __builtin_amdgcn_readfirstlane((uint32_t)(32 * a.lda)), step_b = __builtin_amdgcn_readfirstlane((uint32_t)(32 * a.ldb));
  const uint32_t lds0 = (uint32_t)(uintptr_t)(WSG_LDS uint8_t*)smem + wave * 1024;
  constexpr int kLoads = (TM + TN) / 32;  // of a wave and block, 1 KiB each
  const auto load = [&](int b, int from, int to) {
    const bool inside = b * kBlock + lc < t.K;  // else zeros: past the last column
    const uint32_t ia = inside ? at_a : kOutside, ib = inside ? at_b : kOutside, lds = lds0 + b % STAGES * kStage;
#pragma unroll
    for (int i = from; i < to; ++i) {
      if (i < TM / 32) load_to_lds(t.ra, ia + i * step_a, b * kBlock, lds + i * 4096);
      else load_to_lds(t.rb, ib + (i - TM / 32) * step_b, b * kBlock, lds + i * 4096);
    }
  };
  // scales of this thread's rows of the tile
  uint8_t* scales = smem + Shape::kScalesAt;
  typedef uint8_t bytes_t[Shape::kMine];
  // where a row's scale lies: [row % 16][row / 16], A's rows first
  const auto scale_place = [](int row) {
    return row < TM ? row % 16 * (2 * WM) + row / 16 : TM + (row - TM) % 16 * (2 * WN) + (row - TM) / 16;
  };
  // Row i of this thread: every thread has one inside the tile, more than one thread
  // the same where there are fewer rows than threads.
  const auto my_row = [&](int i) { return kRows >= 256 ? min(tid + 256 * i, kRows - 1) : tid % kRows; };
  const auto fetch_scales = [&](int b, bytes_t& byte) {
#pragma unroll
    for (int i = 0; i < Shape::kMine; ++i) byte[i] = t.scale_at[i][min(b, t.blocks - 1) * (my_row(i) < TM ? a.ldsa : a.ldsb)];
  };
  const auto keep_scales = [&](int b, const bytes_t& byte) {
#pragma unroll
    for (int i = 0; i < Shape::kMine; ++i) scales[(b & 1) * kRows + scale_place(my_row(i))] = byte[i];
  };
  // scales of kDeep blocks from b, by all threads
  const auto fill_scales = [&](int b) {
    constexpr int kAtOnce = 8;
    static_assert(STAGES == 2 || 256 % kRows == 0, "whole blocks of scales at a time");
    const int row = my_row(0);  // kRows divides 256
    const uint8_t* from = t.scale_at[0];
    const int64_t ld = row < TM ? a.ldsa : a.ldsb;
    for (int k0 = tid / kRows; k0 < Shape::kDeep; k0 += kAtOnce * (256 / kRows)) {
      uint8_t s[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) s[k] = from[min(b + k0 + k * (256 / kRows), t.blocks - 1) * ld];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) scales[(k0 + k * (256 / kRows)) * kRows + scale_place(row)] = s[k];
    }
  };
  bytes_t byte0, byte1, byte;
  // Finds tile `id` and starts on its first two blocks.
  const auto begin_tile = [&]() {
    uint32_t group = 0, at = id;
    if constexpr (MODE == kDepthGroups) {
      group = id / plane;
      at = id % plane;
      if (a.groups <= kRanked) group = __builtin_ctzll(__ballot(rank == (int)group));
    }
    const uint32_t wide = 8 * tiles_n, first = at / wide * 8, high = min(8u, tiles_m - first), in = at % wide;
    find_part<MODE>(a, first + in % high, in / high, group, TM, TN, &t.p);
    t.rows = (int)min(t.p.m_end - t.p.m0, (int64_t)TM);
    t.cols = (int)min(a.N - t.p.n0, (int64_t)TN);
    t.K = t.p.zero ? 0 : (int)t.p.K;
    t.blocks = (t.K + kBlock - 1) / kBlock;
    if (t.blocks == 0) return;
    t.ra = raw_buffer(t.p.A + t.p.m0 * a.lda, (uint32_t)(t.rows * a.lda));
    t.rb = raw_buffer(t.p.B + t.p.n0 * a.ldb, (uint32_t)(t.cols * a.ldb));
#pragma unroll
    for (int i = 0; i < Shape::kMine; ++i) {
      const int row = my_row(i);
      t.scale_at[i] = row < TM ? t.p.sa + t.p.m0 + min(row, t.rows - 1) : t.p.sb + ((t.p.n0 + min(row - TM, t.cols - 1)) >> a.b_shift);
    }
    if constexpr (STAGES == 2) {
      fetch_scales(0, byte0);
      fetch_scales(1, byte1);
      fetch_scales(2, byte);
    }
#pragma unroll
    for (int b = 0; b < STAGES; ++b) load(b, 0, kLoads);
  };

  if (id < end) begin_tile();
  while (id < end) {
    f32x4_t acc[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
      for (int j = 0; j < WN; ++j) acc[i][j] = f32x4_t{0, 0, 0, 0};
    if (t.blocks > 0) {
      const int fa0 = (wm * WM * 16 + r) * kBlock, fb0 = (TM + wn * WN * 16 + r) * kBlock, c0 = chunk_at(r, g), c1 = chunk_at(r, g + 4);
      i32x8_t fa[WM], fb[WN];
      i32x4_t wa[WM][4], wb[WN][4];  // WIDE: operands in bf16
      uint32_t sa[(WM + 3) / 4], sb[(WN + 3) / 4];
      const auto frag = [&](int row, int stage) {
        const uint8_t* f = smem + stage + row;
        return join(*(const i32x4_t*)(f + c0), *(const i32x4_t*)(f + c1));
      };
      const auto read_scales = [&](int b, uint32_t* sa, uint32_t* sb) {
        const uint8_t* s = scales + b % Shape::kDeep * kRows;
        __builtin_memcpy(sa, __builtin_assume_aligned(s + (2 * r + wm) * WM, WM), WM);
        __builtin_memcpy(sb, __builtin_assume_aligned(s + TM + (2 * r + wn) * WN, WN), WN);
      };
      if constexpr (STAGES == 2) {
        keep_scales(0, byte0);
        keep_scales(1, byte1);
      } else {
        fill_scales(0);
      }
      drain_and_meet();
      read_scales(0, sa, sb);
#pragma unroll
      for (int j = 0; j < WN; ++j) fb[j] = frag(fb0 + j * 2048, 0);
#pragma unroll
      for (int i = 0; i < kFirst; ++i) fa[i] = frag(fa0 + i * 2048, 0);
#pragma unroll
      for (int i = 0; i < (WM + 3) / 4; ++i) settle_scales(sa[i]);
#pragma unroll
      for (int j = 0; j < (WN + 3) / 4; ++j) settle_scales(sb[j]);
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): in the loop the compiler then counts LDS reads only
      for (int b = 0; b < t.blocks; ++b) {
        const int here = b % STAGES * kStage, next = (b + 1) % STAGES * kStage;
        if constexpr (WIDE) {
          multiply_rows_wide<Shape::kAgpr, 0, kFirst, kRest>(acc, fa, fb, wa, wb, sa, sb, [&](auto jc, auto qc, auto ic) {
            constexpr int at = (decltype(jc)::value * 4 + decltype(qc)::value) * kFirst + decltype(ic)::value, all = WN * 2 * kFirst;
#pragma unroll
            for (int k = at * kRest / all; k < (at + 1) * kRest / all && at < all; ++k)
              fa[kFirst + k] = frag(fa0 + (kFirst + k) * 2048, here);
          });
        } else {
          static_for<kFirst>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            static_for<WN>([&](auto jc) {
              constexpr int j = decltype(jc)::value, at = i * WN + j, all = (kFirst * WN - 1) / (kFirst > 2 ? 2 : 1);
              multiply<Shape::kAgpr, i % 4, j % 4>(acc[i][j], fa[i], fb[j], sa[i / 4], sb[j / 4]);
#pragma unroll
              for (int k = at * kRest / all; k < (at + 1) * kRest / all && at < all; ++k)
                fa[kFirst + k] = frag(fa0 + (kFirst + k) * 2048, here);
            });
            __builtin_amdgcn_sched_barrier(0);
          });
        }
        drain_and_meet<kLoads * (STAGES - 2)>();
        uint32_t next_sa[(WM + 3) / 4], next_sb[(WN + 3) / 4];
        // What else the block needs is done between its products: the scales first
        // (before the loads, which their wait would wait for), then the loads, one at
        // a time (two hold up the products behind them), and the next operands.
        const auto scales_next = [&]() {
          if constexpr (STAGES == 2) {
            keep_scales(b + 2, byte);
            fetch_scales(b + 3, byte);
          }
          read_scales(b + 1, next_sa, next_sb);
        };
        if constexpr (STAGES > 2)
          if ((b + 1) % Shape::kDeep == 0 && b + 1 < t.blocks) {  // the next blocks' scales; every wave has read the last
            fill_scales(b + 1);
            drain_and_meet();
          }
        if constexpr (WIDE) {
          scales_next();
          __builtin_amdgcn_sched_barrier(0);
          multiply_rows_wide<Shape::kAgpr, kFirst, kRest, 0>(acc, fa, fb, wa, wb, sa, sb, [&](auto jc, auto qc, auto ic) {
            constexpr int j = decltype(jc)::value, q = decltype(qc)::value, i = decltype(ic)::value;
            constexpr int at = (j * 4 + q) * kRest + i, all = WN * 4 * kRest;
            load(b + STAGES, at * kLoads / all, (at + 1) * kLoads / all);
            if constexpr (q == 3 && i == kRest - 1) {
#pragma unroll
              for (int k = j * kFirst / WN; k < (j + 1) * kFirst / WN; ++k) fa[k] = frag(fa0 + k * 2048, next);
            }
            // column j is widened during column j - 1
            if constexpr (q == 0 && i == 0 && j > 0) fb[j] = frag(fb0 + j * 2048, next);
            if constexpr (j == 0 && q == 3 && i == 0) fb[0] = frag(fb0, next);
          });
        } else {
          // loads follow the products of columns kFrom .. kTo - 1
          constexpr int kFrom = WN > 2 ? 1 : 0, kTo = WN > 4 ? WN - 1 : WN, kSlots = (kTo - kFrom) * kRest;
          static_for<WN>([&](auto jc) {
            constexpr int j = decltype(jc)::value;
            static_for<kRest>([&](auto ic) {
              constexpr int i = decltype(ic)::value, row = kFirst + i, at = (j - kFrom) * kRest + i;
              multiply<Shape::kAgpr, row % 4, j % 4>(acc[row][j], fa[row], fb[j], sa[row / 4], sb[j / 4]);
              if constexpr (j == 0 && i == 0) {
                __builtin_amdgcn_sched_barrier(0);
                scales_next();
                __builtin_amdgcn_sched_barrier(0);
              }
              if constexpr (at >= 0 && at < kSlots) load(b + STAGES, at * kLoads / kSlots, (at + 1) * kLoads / kSlots);
              if constexpr (i == 0) {
#pragma unroll
                for (int k = j * kFirst / WN; k < (j + 1) * kFirst / WN; ++k) fa[k] = frag(fa0 + k * 2048, next);
                if constexpr (j > 0) fb[j - 1] = frag(fb0 + (j - 1) * 2048, next);
              }
            });
            __builtin_amdgcn_sched_barrier(0);
          });
          fb[WN - 1] = frag(fb0 + (WN - 1) * 2048, next);
        }
#pragma unroll
        for (int i = 0; i < (WM + 3) / 4; ++i) settle_scales(sa[i] = next_sa[i]);
#pragma unroll
        for (int j = 0; j < (WN + 3) / 4; ++j) settle_scales(sb[j] = next_sb[j]);
      }
      asm volatile("s_nop 15\n\ts_nop 15");  // the last sums, before anything may move them
      drain_and_meet();  // no load of this tile lands, and no wave reads, after this
    }
    const Part p = t.p;
    const int rows = t.rows, cols = t.cols;
    id = next_id();
    if (id < end) begin_tile();
    uint8_t* own = smem + Shape::kStoreAt + wave * Shape::kStoreBytes;
    if constexpr (WIDE) store_tile<float, WM, WN, STAGES>(a, p, acc, own, wm, wn, rows, cols);
    else if (a.dtype == WS_OUT_BF16) store_tile<bf16_t, WM, WN, STAGES>(a, p, acc, own, wm, wn, rows, cols);
    else store_tile<f16_t, WM, WN, STAGES>(a, p, acc, own, wm, wn, rows, cols);
  }
}

// -- host --------------------------------------------------------------------------

// Compute units of the current device, asked for once (256 where it does not say).
int compute_units() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  n = known[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    known[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

// Bytes between rows so that a tile's offsets stay below kOutside.
constexpr int64_t kMaxLd = 1 << 22;

constexpr int kDirectThreads = 512;  // of a workgroup of the direct kernel, at the most
// Tiles of a tile kernel, whose workgroups take any number: their numbers, counted
// two rounds of workgroups past the end, fit 32 bits.
constexpr int64_t kMaxTiles = 1ll << 31;

int64_t tiles_of_rows(int mode, int64_t M, int64_t groups, int rows) {
  return mode == kRowGroups ? group_tiles(M, groups, rows, true) : ceil_div(M, rows);
}
// Tiles of rows x cols that cover a product, or `most` + 1 for more than `most`.
int64_t tiles_of(int mode, int64_t M, int64_t N, int64_t groups, int rows, int cols, int64_t most) {
  const int64_t plane = tiles_of_rows(mode, M, groups, rows) * ceil_div(N, cols);
  if (plane > most) return most + 1;
  const int64_t all = plane * (mode == kDepthGroups ? groups : 1);
  return all > most ? most + 1 : all;
}

template <int MT, int U, int MODE>
ws_status run_direct(ProductArgs a, hipStream_t stream) {
  a.tiles_n = ceil_div(a.N, 16);
  a.tiles_m = tiles_of_rows(MODE, a.M, a.groups, 16 * MT);
  const int64_t most = max_workgroups(kDirectThreads), grid = tiles_of(MODE, a.M, a.N, a.groups, 16 * MT, 16, most);
  if (grid > most) return WS_ERR_INVALID_ARG;
  // Waves that share a contraction: as many as give the card 4096 or one block each.
  int waves = 1;
  while (waves < 8 && grid * waves < 4096 && waves * kBlock < a.K) waves *= 2;
  const auto kernel = a.dtype == WS_OUT_F32 ? &direct_kernel<MT, U, MODE, true> : &direct_kernel<MT, U, MODE, false>;
  return launch("fp8_product", kernel, grid, 64 * waves, waves * MT * 1024, stream, a);
}

template <int WM, int WN, int STAGES, int MODE, bool WIDE>
ws_status run_tiles(ProductArgs a, hipStream_t stream) {
  typedef TileShape<WM, WN, STAGES> Shape;
  constexpr int TM = Shape::TM, TN = Shape::TN;
  a.tiles_n = ceil_div(a.N, TN);
  a.tiles_m = tiles_of_rows(MODE, a.M, a.groups, TM);
  const int64_t tiles = tiles_of(MODE, a.M, a.N, a.groups, TM, TN, kMaxTiles);
  if (tiles > kMaxTiles) return WS_ERR_INVALID_ARG;
  const int64_t most = (int64_t)compute_units() * Shape::kWaves;
  a.tile_groups = (int32_t)(tiles < most ? tiles : most);
  const int64_t rest = a.rest_end > a.M ? ceil_div(a.rest_end - a.M, a.rest_rows) * ceil_div(a.N, 16) : 0;
  const auto kernel = &tile_kernel<WM, WN, STAGES, MODE, WIDE>;
  static std::atomic<uint64_t> allowed;  // devices on which the kernel may use this much LDS
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess && (dev >= 64 || !(allowed.load(std::memory_order_acquire) >> dev & 1))) {
    e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, Shape::kLds);
    if (e == hipSuccess && dev < 64) allowed.fetch_or(1ull << dev, std::memory_order_acq_rel);
  }
  if (e != hipSuccess) return hip_fail("hipFuncSetAttribute", e);
  return launch("fp8_product", kernel, a.tile_groups + rest, 256, Shape::kLds, stream, a);
}

// What a product costs by each kernel, in us (MI355X, 256 CUs; fitted to 23
// products from 64 x 2048 x 2048 to 8192 x 8192 x 8192, most within 15 %).  A CU
// has n tiles: their blocks of 128 columns take `alone` each where it has one,
// n * `shared` otherwise, and every tile `tile` more.
struct TileCost {
  int rows, cols;  // of a tile
  float fixed, alone, shared, tile;
};
//                                  16-bit results                     32-bit results
constexpr TileCost kCost256 =      {256, 256, 4.0f, 1.30f, 1.50f, 7.0f};
constexpr TileCost kCost256Wide =  {256, 128, 4.0f, 1.80f, 1.85f, 4.0f};
constexpr TileCost kCost128[2] =  {{128, 128, 4.0f, 0.60f, 0.57f, 0.5f}, {128, 128, 4.0f, 1.05f, 1.02f, 0.7f}};
constexpr TileCost kCost128Deep =  {128, 128, 4.5f, 0.50f, 0.55f, 2.6f};  // four stages
constexpr TileCost kCost64[2] =   {{64, 64, 3.7f, 0.30f, 0.25f, 0.3f}, {64, 64, 3.7f, 0.50f, 0.37f, 0.3f}};
constexpr TileCost kCost64Deep[2] = {{64, 64, 4.5f, 0.27f, 0.22f, 0.6f}, {64, 64, 4.5f, 0.48f, 0.35f, 0.6f}};

enum Choice { kDirect16, kDirect32, kDirect64, kTile256, kTile128, kTile128Deep, kTile64, kTile64Deep };

// `parts` products of on average rows x N, contracted over K columns each.
struct Work {
  double rows, parts;
  int64_t N, K;
  int size;  // bytes of a result
};

// Bytes of results per us, and a tile's way from its first load to its last store
// where two workgroups of a CU go it in turn: what tiles of few blocks take.
constexpr float kStoreRate = 5.1e6f, kTrip = 1.5f;

float tile_cost(const Work& w, const TileCost& c) {
  // a part's last tile is partly filled: half of one on average, where there are several parts
  const double tiles_m = w.parts > 1 ? w.parts * (w.rows / c.rows + 0.5) : (double)ceil_div((int64_t)w.rows, c.rows);
  const double n = ceil(tiles_m * (double)ceil_div(w.N, c.cols) / compute_units());
  const float blocks = (float)ceil_div(w.K, kBlock);
  if (n <= 1) return c.fixed + blocks * c.alone + c.tile * (float)n;
  const float store = (float)c.rows * c.cols * w.size * compute_units() / kStoreRate;
  return c.fixed + (float)n * fmaxf(blocks * c.shared + c.tile, fmaxf(store, kTrip));
}

// The direct kernel is bound by what its workgroups load, at 11 TB/s from the
// caches, where there are many by starting and ending them (0.7 to 1.2 ns each), and for
// long contractions by the trips that a wave makes.
float direct_cost(const Work& w, int rows) {
  const double tiles_m = w.parts > 1 ? w.parts * (w.rows / rows + 0.5) : (double)ceil_div((int64_t)w.rows, rows);
  const double groups = tiles_m * (double)ceil_div(w.N, 16);
  return (float)(4.0 + groups * (rows + 16.0) * (double)w.K / 11e6 + fmax(groups - 4096.0, 0.0) * (0.55 + 0.01 * rows) / 1e3 +
                 0.03 * (double)w.K / kBlock);
}

// A kernel's tile and the stages of its ring.
ws_fp8_kernel_info kernel_of(Choice c, bool wide) {
  switch (c) {
    case kDirect16: return {16, 16, 0, 0};
    case kDirect32: return {32, 16, 0, 0};
    case kDirect64: return {64, 16, 0, 0};
    case kTile64: return {64, 64, 2, 0};
    case kTile64Deep: return {64, 64, 4, 0};
    case kTile128: return {128, 128, 2, 0};
    case kTile128Deep: return {128, 128, 4, 0};
    default: return {256, wide ? 128 : 256, 2, 0};
  }
}

// The cheapest kernel of those that one launch can run on all of a product's tiles;
// *cost is infinite where there is none.
Choice choose(const Work& w, int mode, int64_t M, int64_t groups, bool wide, float* cost) {
  Choice best = kDirect16;
  *cost = INFINITY;
  const auto consider = [&](Choice c, float t) {
    const ws_fp8_kernel_info k = kernel_of(c, wide);
    const int64_t most = k.stages == 0 ? max_workgroups(kDirectThreads) : kMaxTiles;
    if (t < *cost && tiles_of(mode, M, w.N, groups, k.tile_m, k.tile_n, most) <= most) {
      *cost = t;
      best = c;
    }
  };
  consider(kDirect16, direct_cost(w, 16));
  consider(kDirect32, direct_cost(w, 32));
  consider(kDirect64, direct_cost(w, 64));
  consider(kTile64, tile_cost(w, kCost64[wide]));
  consider(kTile64Deep, tile_cost(w, kCost64Deep[wide]));
  consider(kTile128, tile_cost(w, kCost128[wide]));
  if (!wide) consider(kTile128Deep, tile_cost(w, kCost128Deep));
  consider(kTile256, tile_cost(w, wide ? kCost256Wide : kCost256));
  return best;
}

template <int MODE>
ws_status run_choice(Choice c, const ProductArgs& a, hipStream_t stream) {
  const bool wide = a.dtype == WS_OUT_F32;
  switch (c) {
    case kDirect16: return run_direct<1, 4, MODE>(a, stream);
    case kDirect32: return run_direct<2, 4, MODE>(a, stream);
    case kDirect64: return run_direct<4, 2, MODE>(a, stream);
    case kTile64: return wide ? run_tiles<2, 2, 2, MODE, true>(a, stream) : run_tiles<2, 2, 2, MODE, false>(a, stream);
    case kTile64Deep: return wide ? run_tiles<2, 2, 4, MODE, true>(a, stream) : run_tiles<2, 2, 4, MODE, false>(a, stream);
    case kTile128: return wide ? run_tiles<4, 4, 2, MODE, true>(a, stream) : run_tiles<4, 4, 2, MODE, false>(a, stream);
    case kTile128Deep: return run_tiles<4, 4, 4, MODE, false>(a, stream);
    default: return wide ? run_tiles<8, 4, 2, MODE, true>(a, stream) : run_tiles<8, 8, 2, MODE, false>(a, stream);
  }
}

// One or two parts of a product: the first `split` rows by choice[0], the rest
// by choice[1], `together` in one launch.  No part: no kernel's launch holds it.
struct Plan {
  int count;
  int64_t split;
  Choice choice[2];
  bool together;
};

Plan plan_product(int mode, int64_t M, int64_t N, int64_t K, int64_t groups, bool wide) {
  Work w{(double)M, 1.0, N, K, wide ? 4 : 2};
  if (mode == kRowGroups) {
    w.parts = (double)(groups < M ? groups : M);
    w.rows = (double)M / w.parts;
  }
  if (mode == kDepthGroups) {
    w.parts = (double)groups;
    w.K = ceil_div(ceil_div(K, groups), kBlock) * kBlock;
  }
  float cost;
  Plan plan{1, M, {choose(w, mode, M, groups, wide, &cost), kDirect16}, false};
  if (isinf(cost)) plan.count = 0;
  if (mode == kDense && M > kBlock && M % kBlock != 0) {
    // The last rows by themselves, where they would start tiles of their own that a
    // round has no place for (4104 x 1000 x 4100: 33 x 8 tiles of 128 rows for 256
    // CUs, of which the 8 rows past 4096 fill one row of tiles).
    float main_cost, rest_cost;
    Work top = w, rest = w;
    top.rows = (double)(M / kBlock * kBlock);
    rest.rows = (double)(M % kBlock);
    const Choice cm = choose(top, mode, M / kBlock * kBlock, groups, wide, &main_cost);
    const Choice cr = choose(rest, mode, M % kBlock, groups, wide, &rest_cost);
    if (main_cost + rest_cost < 0.95f * cost) {
      // The last rows in the launch of the tiles, by workgroups of the direct kernel's
      // rows: beside the tiles where a CU has room for two (4216 x 1000 x 4100 in 32
      // bits: 41 us, in a launch of their own 51), else behind them, where they are few
      // (4104 x 1000 x 4100 in bf16: 30.3 and 31.6; but 4160 x 4096 x 4096 in bf16,
      // 16 rows a workgroup: 73, in a launch of their own 66).
      const bool beside = cm == kTile128 || cm == kTile64;
      const ws_fp8_kernel_info last = kernel_of(cr, wide);
      const bool together = cm >= kTile256 && last.stages == 0 && (beside || M % kBlock <= 16) &&
                            ceil_div(M % kBlock, last.tile_m) * ceil_div(N, 16) <= max_workgroups(256) - 2 * compute_units();
      plan = Plan{2, M / kBlock * kBlock, {cm, cr}, together};
    }
  }
  return plan;
}

template <int MODE>
ws_status run_product(const ProductArgs& a, hipStream_t stream) {
  const Plan plan = plan_product(MODE, a.M, a.N, MODE == kDepthGroups ? a.depth_rows : a.K, a.groups, a.dtype == WS_OUT_F32);
  if (plan.count == 0) return WS_ERR_INVALID_ARG;
  if (plan.count == 1) return run_choice<MODE>(plan.choice[0], a, stream);
  ProductArgs m = a, r = a;
  m.M = plan.split;
  r.M = a.M - m.M;
  if (plan.together) {
    m.rest_end = a.M;
    m.rest_rows = kernel_of(plan.choice[1], false).tile_m;
    return run_choice<MODE>(plan.choice[0], m, stream);
  }
  const int size = elem_size(a.dtype);
  r.A += m.M * a.lda;
  r.sa += m.M;
  r.C = (uint8_t*)a.C + m.M * a.ldc * size;
  if (a.C0) r.C0 = (const uint8_t*)a.C0 + m.M * a.ldc0 * size;
  const ws_status s = run_choice<MODE>(plan.choice[0], m, stream);
  return s != WS_OK ? s : run_choice<MODE>(plan.choice[1], r, stream);
}

// Operands of a contraction over K columns; b_batch: B's matrices.
bool operands_fit(const ws_fp8_matrix* A, const ws_fp8_matrix* B, int b_batch) {
  return valid(A) && valid(B) && A->batch <= 1 && A->block_rows == 1 && A->cols == B->cols &&
         (b_batch == 0 ? B->batch <= 1 : B->batch == b_batch) && A->ld <= kMaxLd && B->ld <= kMaxLd;
}
bool result_fits(const ws_matrix* C, const ws_matrix* C0, float alpha, float beta, int64_t M, int64_t N, int batch) {
  const auto fits = [&](const ws_matrix* m) {
    return valid(m) && m->rows == M && m->cols == N && (batch == 0 ? m->batch <= 1 : m->batch == batch);
  };
  if (!(alpha - alpha == 0.0f) || !(beta - beta == 0.0f)) return false;  // finite
  return fits(C) && (beta == 0.0f || (C0 && fits(C0) && C0->dtype == C->dtype));
}

ProductArgs product_args(const ws_fp8_matrix* A, const ws_fp8_matrix* B, float alpha, float beta, const ws_matrix* C0,
                         const ws_matrix* C) {
  ProductArgs a{};
  a.A = (const uint8_t*)A->codes;
  a.B = (const uint8_t*)B->codes;
  a.sa = A->scales;
  a.sb = B->scales;
  a.C = C->data;
  a.lda = A->ld;
  a.ldb = B->ld;
  a.ldsa = A->ld_scales;
  a.ldsb = B->ld_scales;
  a.ldc = C->ld;
  a.M = A->rows;
  a.N = B->rows;
  a.K = ceil_div(A->cols, 16) * 16;
  a.b_shift = B->block_rows == 1 ? 0 : 7;
  a.dtype = C->dtype;
  a.alpha = alpha;
  a.beta = beta;
  a.stride_c = C->stride;
  if (beta != 0.0f) {
    a.C0 = C0->data;
    a.ldc0 = C0->ld;
    a.stride_c0 = C0->stride;
  }
  return a;
}

}  // namespace
}  // namespace wsg

using namespace wsg;

extern "C" {

ws_status ws_fp8_plan(int64_t M, int64_t N, int64_t K, int32_t out_dtype, int32_t groups, int32_t depth,
                      ws_fp8_kernel_info* out, int32_t* count) {
  if (!out || !count || M < 0 || N < 0 || K < 0 || M > kMaxDim || N > kMaxDim || K > kMaxDim || !elem_size(out_dtype) || groups < 0 ||
      groups > (1 << 20) || (groups == 0 && depth != 0))
    return WS_ERR_INVALID_ARG;
  *count = 0;
  if (M == 0 || N == 0) return WS_OK;
  const bool wide = out_dtype == WS_OUT_F32;
  const Plan plan = plan_product(groups == 0 ? kDense : depth ? kDepthGroups : kRowGroups, M, N, K, groups, wide);
  if (plan.count == 0) return WS_ERR_INVALID_ARG;
  for (int i = 0; i < plan.count; ++i) {
    ws_fp8_kernel_info k = kernel_of(plan.choice[i], wide);
    k.rows = i == 0 ? plan.split : M - plan.split;
    k.launch = plan.together ? 0 : i;
    out[i] = k;
  }
  *count = plan.count;
  return WS_OK;
}

ws_status ws_fp8_product(const ws_fp8_matrix* A, const ws_fp8_matrix* B, float alpha, float beta, const ws_matrix* C0,
                         const ws_matrix* C, hipStream_t stream) {
  if (!operands_fit(A, B, 0) || !result_fits(C, C0, alpha, beta, A->rows, B->rows, 0)) return WS_ERR_INVALID_ARG;
  if (A->rows == 0 || B->rows == 0) return WS_OK;
  return run_product<kDense>(product_args(A, B, alpha, beta, C0, C), stream);
}

ws_status ws_fp8_grouped_product(const ws_fp8_matrix* A, const ws_fp8_matrix* B, int32_t groups, const int32_t* offsets,
                                 float alpha, const ws_matrix* C, hipStream_t stream) {
  if (groups < 1 || groups > (1 << 20) || !offsets || (uintptr_t)offsets % 4 || !operands_fit(A, B, groups) ||
      !result_fits(C, nullptr, alpha, 0.0f, A->rows, B->rows, 0))
    return WS_ERR_INVALID_ARG;
  if (A->rows == 0 || B->rows == 0) return WS_OK;
  ProductArgs a = product_args(A, B, alpha, 0.0f, nullptr, C);
  a.offsets = offsets;
  a.groups = groups;
  a.stride_b = B->stride_codes;
  a.stride_sb = B->stride_scales;
  return run_product<kRowGroups>(a, stream);
}

ws_status ws_fp8_grouped_gradient(const ws_fp8_matrix* A, const ws_fp8_matrix* B, int64_t rows, int32_t groups,
                                  const int32_t* offsets, float alpha, float beta, const ws_matrix* C0,
                                  const ws_matrix* C, hipStream_t stream) {
  if (groups < 1 || groups > (1 << 20) || !offsets || (uintptr_t)offsets % 4 || rows < 0 || rows > kMaxDim ||
      !operands_fit(A, B, 0) || B->block_rows != 1 || A->cols != kBlock * ws_fp8_padded_blocks(rows, groups) ||
      !result_fits(C, C0, alpha, beta, A->rows, B->rows, groups))
    return WS_ERR_INVALID_ARG;
  if (A->rows == 0 || B->rows == 0) return WS_OK;
  ProductArgs a = product_args(A, B, alpha, beta, C0, C);
  a.offsets = offsets;
  a.groups = groups;
  a.depth_rows = rows;
  return run_product<kDepthGroups>(a, stream);
}

}  // extern "C"
