// Orthogonalised updates (definitions: ws_orthogonal.h).
//
// X (n x m, n the shorter side of G) and its transpose Y lie in binary16, scaled by
// 2^14 (entries of X stay below 1.3, and those of a large matrix are small), with what
// that leaves of every entry, times 2^11 more, in a third matrix.  A step is three
// launches of one tile kernel, every operand's contraction along its rows:
//
//   S  <- X X^T             off the diagonal, which goes to dA in binary32
//   T  <- b A + c A^2       likewise, dB = a + b A_ii + c (A^2)_ii, with
//                           A^2 = S^2 + (dA_i + dA_j) S + dA_i^2 on the diagonal
//   Y' <- Y T + dB_j Y      and X' its transpose
//
// S and T are symmetric: tiles below their diagonal are computed and written twice.
// Why diagonals are kept apart: once singular values are near 1, A and T are near
// multiples of the identity, and rounding these to binary16 cost most of the error
// (1.0e-3 to 2.3e-3 of the result so, 1e-4 to 1e-3 apart, of values that are alike).
//
// Short sides, and more than five steps (in_two_values): X, Y, S and T are two binary16
// values each, of the same unit, and a product is three; see FINE.
#include <math.h>

#include "ws_orthogonal.hpp"
#include "ws_tile.hpp"

namespace wsg {
namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kUnit = 16384.0f, kPerUnit = 1.0f / kUnit;  // of X, S and T
constexpr float kRest = 2048.0f;                            // of the rest of X, beyond
constexpr int kPad = 128;                                    // sides in the workspace are multiples of it: blocks of 64 columns are even in number

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

enum Kind { kGram, kSquare, kApply, kLast };

// FINE, in what follows: X, Y, S and T are sums of two binary16 values, whose rows lie one
// behind the other, twice as long.
template <bool FINE>
constexpr int kRow = FINE ? 2 : 1;

struct OrthArgs {
  const _Float16 *A, *B;         // operands, `batch` of them
  int64_t stride_a, stride_b;    // elements between them
  int32_t M, N, K;               // multiples of kPad; rows of K elements (FINE: twice)
  int32_t batch, tile_groups, tiles_m, tiles_n;
  uint32_t plane;                // tiles of one matrix
  uint32_t first, count;         // tiles of this launch; quarters: every one of them in four of half its sides
  int32_t quarters;
  _Float16 *to, *mirror;         // S; T; Y' and X'
  int64_t stride_to, stride_mirror;
  const float* d_in;             // kSquare: dA; kApply: dB
  float* d_out;                  // kGram: dA; kSquare: dB
  int64_t stride_d;
  _Float16* rest;                // of Y, where not FINE
  // kLast
  uint16_t* out;
  int64_t ld_out, stride_out;
  int32_t rows, cols, transposed;  // of out; transposed: it is X, not Y
};

template <int WM, int WN, int STAGES, bool FINE = false>
struct OrthShape {
  static constexpr int TM = 32 * WM, TN = 32 * WN, kPart = (TM + TN) * 128, kStage = kRow<FINE> * kPart;
  static constexpr bool kAgpr = WM * WN > 16;
  static constexpr int kWaves = kAgpr || STAGES > 2 ? 1 : (WM * WN > 4 ? 2 : 4) / kRow<FINE>;  // of a SIMD, as workgroups of a CU
  static constexpr int kFirst = WM > 4 ? 3 : WM / 2;
  // a wave's way to memory: 64 (or all its) rows of 32 columns
  static constexpr int kHalves = WM >= 4 ? 2 : 1, kStoreBytes = kHalves * 32 * 32 * 2;
  // Lines of later blocks are asked for ahead by loads that end here, 256 bytes a wave.
  static constexpr bool kAhead = kAgpr;
  static constexpr int kStoreAt = STAGES * kStage, kAheadAt = kStoreAt + 4 * kStoreBytes, kLds = kAheadAt + (kAhead ? 4 * 256 : 0);
  static_assert(kWaves * kLds <= 160 * 1024, "LDS of a CU");
  static_assert((STAGES & (STAGES - 1)) == 0 && (!kAhead || STAGES == 2), "");
};

// One of two descriptors, as scalars.
__device__ __forceinline__ i32x4_t select(bool first, const i32x4_t& a, const i32x4_t& b) {
  i32x4_t r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(first ? a[i] : b[i]);
  return r;
}

// Loads 4 bytes a lane from buffer offsets `at` + k to LDS at `to`, for what that leaves
// in the L2; see load_to_lds.
__device__ __forceinline__ void touch(i32x4_t r, uint32_t at, uint32_t k, uint32_t to) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile(
      "s_mov_b32 m0, %3\n\t"
      "s_nop 0\n\t"
      "buffer_load_dword %0, %1, %2 offen lds" ::"v"(at),
      "s"(r), "s"(__builtin_amdgcn_readfirstlane(k)), "s"(__builtin_amdgcn_readfirstlane(to)));
#endif
}

// acc += A's 16 rows times B's 16 rows over 32 columns; see ws_fp8_product.hip's.
template <bool AGPR>
__device__ __forceinline__ void multiply_f16(f32x4_t& acc, const i32x4_t& fa, const i32x4_t& fb) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (AGPR) asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(fb), "v"(fa));
  else asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+v"(acc) : "v"(fb), "v"(fa));
#endif
}

// Byte position, in a row of 128, of chunk c of row r of B's half of a stage.  B's rows
// are read in an order that gives a lane eight neighbouring columns of the product
// (row_of_b); the position follows that order against bank conflicts.
__device__ __forceinline__ int chunk_of_b(int r, int c) { return (c ^ (r & 3 | (r >> 3 & 1) << 2)) * 16; }
// Row, of 32, that lane r % 16 has of the j-th of two fragments of B: the lanes 4 g ..
// 4 g + 3 of both hold rows 8 g .. 8 g + 7.
__device__ __forceinline__ int row_of_b(int r, int j) { return 8 * (r >> 2) + 4 * j + (r & 3); }

// Writes 32 H x 32 values of a wave, of which lane (r, g) has columns 8 g .. of rows 16 i
// + r, two to a word, turned round by way of its part of LDS: put(column, row, piece)
// takes 8 neighbours of a column.  Pieces of 16 bytes change places within a line, by
// the line's number, against bank conflicts.
template <int H, typename F>
__device__ __forceinline__ void turn_round(const i32x4_t (&v)[2 * H], uint8_t* own, const F& put) {
  constexpr int kPieces = 4 * H;  // of a line
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const auto place = [](int line, int piece) { return (line * kPieces + (piece ^ (line & (kPieces - 1)))) * 16; };
#pragma unroll
  for (int i = 0; i < 2 * H; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // with the neighbouring row's: even lanes take the first column of a word, odd ones the second
      const uint32_t mine = (uint32_t)v[i][k], other = (uint32_t)__builtin_amdgcn_update_dpp(0, v[i][k], 0xb1, 0xf, 0xf, true);  // quad_perm 1 0 3 2
      const uint32_t both = __builtin_amdgcn_perm(other, mine, lane & 1 ? 0x03020706u : 0x05040100u);
      *(uint32_t*)(own + place(8 * g + 2 * k + (lane & 1), 2 * i + r / 8) + (r & 6) * 2) = both;
    }
  __builtin_amdgcn_wave_barrier();  // a wave's LDS accesses keep their order
#pragma unroll
  for (int e = 0; e < 2 * H; ++e) {
    const int line = 64 / kPieces * e + lane / kPieces, at = lane % kPieces;
    put(line, 8 * at, *(const i32x4_t*)(own + place(line, at)));
  }
  __builtin_amdgcn_wave_barrier();
}

// What half a part of a tile's results needs from memory: 32 x 32 values from row m and
// column n, lane (r, g) columns 8 g .. of rows 16 i + r.
template <int KIND>
struct Old {
  f16x8_t value[2], rest[2];  // kSquare: S (its rest where FINE); kApply, kLast: Y
  f32x4_t dn[2];
  float dm[2];
};
template <int KIND, bool FINE>
__device__ __forceinline__ void fetch(const OrthArgs& a, int64_t matrix, int m, int n, Old<KIND>& o) {
  const int lane = threadIdx.x & 63, row = m + (lane & 15), col = n + 8 * (lane >> 4);
  if constexpr (KIND != kGram) {
    const float* d_in = a.d_in + matrix * a.stride_d;
    o.dn[0] = *(const f32x4_t*)(d_in + col);
    o.dn[1] = *(const f32x4_t*)(d_in + col + 4);
    const int64_t at = matrix * a.stride_a + (int64_t)row * (kRow<FINE> * a.K) + col;  // kApply, kLast: N == K
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      o.value[i] = *(const f16x8_t*)(a.A + at + 16 * i * (kRow<FINE> * a.K));
      if constexpr (FINE) o.rest[i] = *(const f16x8_t*)(a.A + at + 16 * i * (2 * a.K) + a.K);
      else if constexpr (KIND != kSquare) o.rest[i] = *(const f16x8_t*)(a.rest + at + 16 * i * a.K);
      if constexpr (KIND == kSquare) o.dm[i] = d_in[row + 16 * i];
    }
  }
}

// What the kind of launch makes of the sums of 32 x 32 results from row m and column n;
// what v leaves goes to `low` (FINE), or, of X, to memory at once.
template <int KIND, bool FINE>
__device__ __forceinline__ void convert(const OrthArgs& a, const f32x4_t* (&acc)[2][2], const Old<KIND>& o, int64_t matrix, int m,
                                        int n, i32x4_t* v, i32x4_t* low) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, col = n + 8 * g;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = m + 16 * i + r;
    float x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float s = (*acc[i][k / 4])[k % 4] * kPerUnit;
      if constexpr (KIND == kGram) {
        x[k] = s;
      } else if constexpr (KIND == kSquare) {  // in units of kUnit
        float own = (float)o.value[i][k];
        if constexpr (FINE) own += (float)o.rest[i][k];
        const float square = fmaf(o.dm[i] + o.dn[k / 4][k % 4], own, s);
        x[k] = fmaf(kC, square, kB * own);
      } else {
        x[k] = fmaf(o.dn[k / 4][k % 4], fmaf((float)o.rest[i][k], FINE ? 1.0f : 1.0f / kRest, (float)o.value[i][k]), s);
      }
    }
    if constexpr (KIND == kGram || KIND == kSquare) {
      if (m + 32 > n && n + 32 > m) {  // the diagonal is near
        float* d_out = a.d_out + matrix * a.stride_d;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (row == col + k) {
            if constexpr (KIND == kGram) {
              d_out[row] = x[k] * kPerUnit;
            } else {  // S is zero there
              d_out[row] = fmaf(kC, fmaf(o.dm[i], o.dm[i], (*acc[i][k / 4])[k % 4] * (kPerUnit * kPerUnit)), fmaf(kB, o.dm[i], kA));
            }
            x[k] = 0.0f;
          }
      }
    }
    if constexpr (KIND == kLast) {
      bf16_t t[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) t[k] = from_f32<bf16_t>(x[k] * kPerUnit);
      __builtin_memcpy(&v[i], t, 16);
    } else {
      f16x8_t t;
#pragma unroll
      for (int k = 0; k < 8; ++k) t[k] = (_Float16)x[k];
      v[i] = __builtin_bit_cast(i32x4_t, t);
      if constexpr (FINE) {
        f16x8_t left;
#pragma unroll
        for (int k = 0; k < 8; ++k) left[k] = (_Float16)(x[k] - (float)t[k]);
        low[i] = __builtin_bit_cast(i32x4_t, left);
      } else if constexpr (KIND == kApply) {
        f16x8_t left;
#pragma unroll
        for (int k = 0; k < 8; ++k) left[k] = (_Float16)((x[k] - (float)t[k]) * kRest);
        *(f16x8_t*)(a.rest + matrix * a.stride_a + (int64_t)row * a.N + col) = left;
      }
    }
  }
}

// Writes 32 H x 32 converted results of a wave from row m and column n where they belong.
template <int KIND, int H, bool FINE>
__device__ __forceinline__ void write_part(const OrthArgs& a, const i32x4_t (&v)[2 * H], const i32x4_t (&low)[2 * H], int64_t matrix,
                                           int m, int n, bool twice, uint8_t* own) {
  const int lane = threadIdx.x & 63, r = lane & 15, col = n + 8 * (lane >> 4);
  if constexpr (KIND == kLast) {
    uint16_t* out = a.out + matrix * a.stride_out;
    const auto put = [&](int row, int col, i32x4_t piece) {
      if (row >= a.rows) return;
      uint16_t* to = out + (int64_t)row * a.ld_out + col;
      if (col + 8 <= a.cols) {
        store_n<bf16_t, 8>((bf16_t*)to, (const bf16_t*)&piece);
      } else {
        for (int e = 0; e < 8; ++e)
          if (col + e < a.cols) to[e] = ((const uint16_t*)&piece)[e];
      }
    };
    if (a.transposed) {
      turn_round<H>(v, own, [&](int line, int at, i32x4_t piece) { put(n + line, m + at, piece); });
    } else {
#pragma unroll
      for (int i = 0; i < 2 * H; ++i) put(m + 16 * i + r, col, v[i]);
    }
  } else {
    constexpr int R = kRow<FINE>;
    _Float16* to = a.to + matrix * a.stride_to + (int64_t)(m + r) * (R * a.N) + col;
#pragma unroll
    for (int i = 0; i < 2 * H; ++i) {
      *(i32x4_t*)(to + 16 * i * (int64_t)(R * a.N)) = v[i];
      if constexpr (FINE) *(i32x4_t*)(to + 16 * i * (int64_t)(R * a.N) + a.N) = low[i];
    }
    if (twice) {
      _Float16* mirror = a.mirror + matrix * a.stride_mirror;
      turn_round<H>(v, own, [&](int line, int at, i32x4_t piece) { *(i32x4_t*)(mirror + (int64_t)(n + line) * (R * a.M) + m + at) = piece; });
      if constexpr (FINE)
        turn_round<H>(low, own, [&](int line, int at, i32x4_t piece) { *(i32x4_t*)(mirror + (int64_t)(n + line) * (R * a.M) + a.M + m + at) = piece; });
    }
  }
}

// A tile of 32 WM x 32 WN by four waves, 2 x 2.  Blocks of 64 columns lie in a ring of
// STAGES in LDS, and a block's products come in two halves, as in ws_fp8_product.hip:
//
//   the first kFirst rows, row by row: the rest of A of block b is read
//   meet: b + 1 has landed everywhere, b has been read everywhere
//   the other rows, column by column: b + STAGES is loaded over b; the first rows of A
//   of b + 1 are read, and every column of B of b + 1 once that of b is done
//
// Loads go on into a workgroup's next tile, whose first blocks are there when the tile it
// has is written (a tile has two blocks or more; with more stages a workgroup has one).
// Long rings are for few tiles, one a CU, whose blocks are shorter than the way to memory.
// FINE: a stage has the rests of A and B too, for three products: A's rests by B, A by
// B's rests, A by B; what both rests would give is below 2^-22 of the last.  (As three times
// the contraction instead, one product a block: 128 x 4096 341 us, 4 x 188 x 1358 227.)
template <int WM, int WN, int STAGES, int KIND, bool FINE>
__device__ __forceinline__ void orth_step(const OrthArgs& a) {
  typedef OrthShape<WM, WN, STAGES, FINE> Shape;
  constexpr int TM = Shape::TM, TN = Shape::TN, kStage = Shape::kStage, kFirst = Shape::kFirst, kRows = WM - kFirst;
  constexpr int kProducts = FINE ? 6 : 2;  // of two fragments and a block
  constexpr bool kSymmetric = KIND == kGram || KIND == kSquare;
  static_assert(!kSymmetric || TM == TN, "tiles of the lower triangle");
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 15, g = lane >> 4, wm = wave >> 1, wn = wave & 1;
  // an XCD (workgroups go round them in turn) has a run of the tiles
  const uint32_t tiles = a.count, xcd = blockIdx.x % 8, share = tiles / 8, extra = tiles % 8;
  const uint32_t turns = (a.tile_groups + 7 - xcd) / 8, end = xcd * share + min(xcd, extra) + share + (xcd < extra);
  uint32_t id = xcd * share + min(xcd, extra) + blockIdx.x / 8;

  const uint32_t ld = (uint32_t)a.K * (2 * kRow<FINE>);  // bytes between rows of both operands
  const int lr = 8 * wave + (lane >> 3);  // chunk_at and chunk_of_b are their own inverses
  const uint32_t at_a = (uint32_t)lr * ld + chunk_at(lr, lane & 7), at_b = (uint32_t)lr * ld + chunk_of_b(lr, lane & 7), step = 32 * ld;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(WSG_LDS uint8_t*)smem + wave * 1024;
  const int blocks = a.K / 64;  // even: every tile's first one lies in stage 0 where there are two, or where a workgroup has one tile
  constexpr int kHalf = (TM + TN) / 32, kLoads = kRow<FINE> * kHalf;  // of a wave and block, 1 KiB each
  struct Tile {
    int64_t matrix;
    int m0, n0;
    i32x4_t ra, rb;
    uint32_t ahead_a, ahead_b;  // rows of the tile that this workgroup asks for ahead
  } t, later;
  // Where tile `id` lies; past the last one: nowhere, which reads zeros.
  const auto find_tile = [&](Tile& t, uint32_t id) {
    const uint32_t tile = a.first + (a.quarters ? id / 4 : id), matrix = tile / a.plane, in = tile % a.plane;
    uint32_t tm, tn;
    if constexpr (kSymmetric) {  // row after row of the lower triangle
      tm = (uint32_t)((sqrtf(8.0f * (float)in + 1.0f) - 1.0f) * 0.5f);
      while (tm * (tm + 1) / 2 > in) --tm;
      while ((tm + 1) * (tm + 2) / 2 <= in) ++tm;
      tn = in - tm * (tm + 1) / 2;
    } else {  // eight rows of tiles at a time
      const uint32_t wide = 8 * a.tiles_n, first = in / wide * 8, high = min(8u, a.tiles_m - first);
      tm = first + in % wide % high;
      tn = in % wide / high;
    }
    if (a.quarters) {
      tm = 2 * tm + id % 4 / 2;
      tn = 2 * tn + id % 2;
    }
    // past the last tile, and a quarter beside the matrix or above its diagonal: nothing
    const bool there = id < end && (int)tm * TM < a.M && (int)tn * TN < a.N && (!kSymmetric || tn <= tm);
    t.matrix = there ? matrix : 0;
    t.m0 = __builtin_amdgcn_readfirstlane(there ? (int)tm * TM : a.M);
    t.n0 = __builtin_amdgcn_readfirstlane(there ? (int)tn * TN : a.N);
    t.ra = raw_buffer((const uint8_t*)(a.A + t.matrix * a.stride_a + (int64_t)t.m0 * (kRow<FINE> * a.K)), (uint32_t)min(a.M - t.m0, TM) * ld);
    t.rb = raw_buffer((const uint8_t*)(a.B + t.matrix * a.stride_b + (int64_t)t.n0 * (kRow<FINE> * a.K)), (uint32_t)min(a.N - t.n0, TN) * ld);
    t.ahead_a = tn % 4 * 64;
    t.ahead_b = tm % 8 * 32;
  };
  // Loads `from` .. `to` of a block, which may be one of the next tile's first.
  const auto load = [&](int b, int from, int to) {
    const bool here = b < blocks;
    const int k = (here ? b : b - blocks) * 128;
    const uint32_t lds = lds0 + (b & (STAGES - 1)) * kStage;
    const i32x4_t ra = select(here, t.ra, later.ra), rb = select(here, t.rb, later.rb);
#pragma unroll
    for (int l = from; l < to; ++l) {
      const int i = l % kHalf, at = l / kHalf * ((int)ld / 2) + k;  // rests: the second half of a row
      if (i < TM / 32) load_to_lds(ra, at_a + i * step, at, lds + l * 4096);
      else load_to_lds(rb, at_b + (i - TM / 32) * step, at, lds + l * 4096);
    }
  };
  // Asks for lines of a block, so that they are in the L2 when they are loaded: 32 rows
  // a wave of those that the tiles beside this one share, waves 0 and 1 of A, 2 of B.
  const auto ask_ahead = [&](int b) {
    const bool here = b < blocks;
    const int k = (here ? b : b - blocks) * 128;
    const uint32_t row = wave < 2 ? (here ? t.ahead_a : later.ahead_a) + 32 * wave + lane : (here ? t.ahead_b : later.ahead_b) + lane;
    const i32x4_t ra = select(here, t.ra, later.ra), rb = select(here, t.rb, later.rb);
    touch(select(wave < 2, ra, rb), lane < 32 && wave < 3 && b < 2 * blocks ? row * ld : kOutside, k,
          (uint32_t)(uintptr_t)(WSG_LDS uint8_t*)smem + Shape::kAheadAt + wave * 256);
  };

  if (id >= end) return;
  find_tile(t, id);
  if constexpr (STAGES > 2) find_tile(later, id + turns);  // more stages than blocks
  for (int b = 0; b < STAGES; ++b) load(b, 0, kLoads);
  drain_and_meet<kLoads * (STAGES - 1)>();
  for (; id < end; id += turns) {
    find_tile(later, id + turns);
    // The first meeting leaves a load under way as the others do: not one of block 1's.
    if constexpr (Shape::kAhead) ask_ahead(3);
    f32x4_t acc[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
      for (int j = 0; j < WN; ++j) acc[i][j] = f32x4_t{0, 0, 0, 0};
    const int fa0 = (wm * WM * 16 + r) * 128, a0 = fa0 + chunk_at(r, g), a1 = fa0 + chunk_at(r, g + 4);
    const int fb0 = (TM + wn * WN * 16 + row_of_b(r, 0)) * 128, b0 = fb0 + chunk_of_b(row_of_b(r, 0), g), b1 = fb0 + chunk_of_b(row_of_b(r, 0), g + 4);
    i32x4_t fa[WM][2 * kRow<FINE>], fb[WN][2 * kRow<FINE>];  // two of the values, two of their rests
    const auto frag_a = [&](int i, int stage) {
#pragma unroll
      for (int p = 0; p < kRow<FINE>; ++p) {
        fa[i][2 * p] = *(const i32x4_t*)(smem + stage + p * Shape::kPart + a0 + i * 2048);
        fa[i][2 * p + 1] = *(const i32x4_t*)(smem + stage + p * Shape::kPart + a1 + i * 2048);
      }
    };
    const auto frag_b = [&](int j, int stage) {
#pragma unroll
      for (int p = 0; p < kRow<FINE>; ++p) {
        fb[j][2 * p] = *(const i32x4_t*)(smem + stage + p * Shape::kPart + b0 + j / 2 * 4096 + j % 2 * 512);
        fb[j][2 * p + 1] = *(const i32x4_t*)(smem + stage + p * Shape::kPart + b1 + j / 2 * 4096 + j % 2 * 512);
      }
    };
    // product q of a block: rests by values, values by rests, values by values
    const auto of_a = [](int q) { return kProducts - q > 4 ? q + 2 : q % 2; };
    const auto of_b = [](int q) { return FINE && q / 2 == 1 ? q % 2 + 2 : q % 2; };
#pragma unroll
    for (int j = 0; j < WN; ++j) frag_b(j, 0);
#pragma unroll
    for (int i = 0; i < kFirst; ++i) frag_a(i, 0);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): in the loop the compiler then counts LDS reads only
    for (int b = 0; b < blocks; ++b) {
      const int here = (b & (STAGES - 1)) * kStage, next = ((b + 1) & (STAGES - 1)) * kStage;
      static_for<kFirst>([&](auto ic) {
        constexpr int i = decltype(ic)::value;
        static_for<kProducts * WN>([&](auto jc) {
          constexpr int q = decltype(jc)::value / WN, j = decltype(jc)::value % WN, n = i * kProducts * WN + decltype(jc)::value;
          constexpr int all = kFirst * kProducts / 2 * WN;  // slots: the first half of these products
          multiply_f16<Shape::kAgpr>(acc[i][j], fa[i][of_a(q)], fb[j][of_b(q)]);
          if constexpr (n < all) {
#pragma unroll
            for (int k = n * kRows / all; k < (n + 1) * kRows / all; ++k) frag_a(kFirst + k, here);
          }
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      drain_and_meet<Shape::kAhead ? 1 : kLoads * (STAGES - 2)>();  // all but the lines asked for, or the later blocks
      static_for<WN>([&](auto jc) {
        constexpr int j = decltype(jc)::value;
        static_for<kProducts * kRows>([&](auto ic) {
          constexpr int q = decltype(ic)::value / kRows, i = kFirst + decltype(ic)::value % kRows;
          constexpr int n = j * kProducts * kRows + decltype(ic)::value, all = kProducts * kRows * (WN > 2 ? WN - 1 : WN);
          multiply_f16<Shape::kAgpr>(acc[i][j], fa[i][of_a(q)], fb[j][of_b(q)]);
          if constexpr (n < all) load(b + STAGES, n * kLoads / all, (n + 1) * kLoads / all);
          if constexpr (decltype(ic)::value == 0) {
#pragma unroll
            for (int k = j * kFirst / WN; k < (j + 1) * kFirst / WN; ++k) frag_a(k, next);
            if constexpr (j > 0) frag_b(j - 1, next);
          }
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      frag_b(WN - 1, next);
      if constexpr (Shape::kAhead) ask_ahead(b + 4);
    }
    asm volatile("s_nop 15\n\ts_nop 15");  // the last sums, before anything may move them
    const int64_t matrix = t.matrix;
    const int m0 = t.m0, n0 = t.n0;
    t = later;
    uint8_t* own = smem + Shape::kStoreAt + wave * Shape::kStoreBytes;
    // parts of 32 kHalves x 32; what the next half of one needs is fetched before a half is converted
    constexpr int kHalves = Shape::kHalves, kParts = WM / (2 * kHalves) * (WN / 2);
    const auto place = [&](int p, int* m, int* n) {
      *m = m0 + (wm * WM + p / (WN / 2) * (2 * kHalves)) * 16;
      *n = n0 + (wn * WN + p % (WN / 2) * 2) * 16;
      return *m < a.M && *n < a.N;  // sides are multiples of kPad
    };
    Old<KIND> old[2];
    i32x4_t v[2 * kHalves], low[2 * kHalves];
    int m, n;
    if (place(0, &m, &n)) fetch<KIND, FINE>(a, matrix, m, n, old[0]);
    static_for<kHalves * kParts>([&](auto hc) {
      constexpr int h = decltype(hc)::value, p = h / kHalves;
      if constexpr (h + 1 < kHalves * kParts)
        if (place((h + 1) / kHalves, &m, &n)) fetch<KIND, FINE>(a, matrix, m + (h + 1) % kHalves * 32, n, old[(h + 1) % 2]);
      const f32x4_t* part[2][2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          f32x4_t& s = acc[p / (WN / 2) * (2 * kHalves) + h % kHalves * 2 + i][p % (WN / 2) * 2 + j];
          settle<Shape::kAgpr>(s);
          part[i][j] = &s;
        }
      if (place(p, &m, &n)) {
        convert<KIND, FINE>(a, part, old[h % 2], matrix, m + h % kHalves * 32, n, v + h % kHalves * 2, low + h % kHalves * 2);
        if constexpr (h % kHalves == kHalves - 1) write_part<KIND, kHalves, FINE>(a, v, low, matrix, m, n, !kSymmetric || m0 != n0, own);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  }
}

template <int WM, int WN, int STAGES, int KIND>
__global__ __launch_bounds__(256, (OrthShape<WM, WN, STAGES>::kWaves)) void orth_step_kernel(OrthArgs a) {
  orth_step<WM, WN, STAGES, KIND, false>(a);
}
template <int WM, int WN, int STAGES, int KIND>
__global__ __launch_bounds__(256, (OrthShape<WM, WN, STAGES, true>::kWaves)) void orth_fine_kernel(OrthArgs a) {
  orth_step<WM, WN, STAGES, KIND, true>(a);
}

// -- the start -------------------------------------------------------------------

struct OrthStartArgs {
  const void* G;
  int64_t rows, cols, ld, stride;
  double* sums;
  int32_t parts, transposed;  // transposed: Y is G^T, X is G
  _Float16 *X, *Y, *rest;     // rest: where not FINE
  int64_t n, m;               // padded sides
};

constexpr int kSumThreads = 256, kMostParts = 256;

__device__ __forceinline__ double sum_of_wave(double x) {
  for (int d = 32; d; d /= 2) x += __shfl_xor(x, d);
  return x;
}

// The sum of squares of a part of a matrix, in binary64: it neither overflows nor loses
// small gradients.
template <typename T>
__global__ __launch_bounds__(kSumThreads) void orth_sum_kernel(OrthStartArgs a) {
  __shared__ double part[kSumThreads / 64];
  const int64_t matrix = blockIdx.x / a.parts, p = blockIdx.x % a.parts;
  const T* G = (const T*)a.G + matrix * a.stride;
  double sum = 0.0;
  const int64_t chunks = (a.cols + 7) / 8, all = chunks * a.rows;
  for (int64_t i = p * kSumThreads + threadIdx.x; i < all; i += (int64_t)a.parts * kSumThreads) {
    const int64_t c = i % chunks * 8;
    const T* row = G + i / chunks * a.ld;
    float v[8];
    if (c + 8 <= a.cols) {
      T t[8];
      if constexpr (sizeof(T) == 4) {
        load_n<T, 4>(row + c, t);
        load_n<T, 4>(row + c + 4, t + 4);
      } else {
        load_n<T, 8>(row + c, t);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = to_f32(t[k]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = c + k < a.cols ? to_f32(row[c + k]) : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) sum = fma((double)v[k], (double)v[k], sum);
  }
  sum = sum_of_wave(sum);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kSumThreads / 64; ++w) sum += part[w];
    a.sums[blockIdx.x] = sum;
  }
}

// 64 x 64 values of G, normalised, to X, Y and what they leave; zeros around.
template <typename T, bool FINE>
__global__ __launch_bounds__(256) void orth_start_kernel(OrthStartArgs a) {
  __shared__ float tile[64][65];
  const int64_t rows = a.transposed ? a.n : a.m, cols = a.transposed ? a.m : a.n;  // padded sides of G
  const int64_t across = cols / 64, plane = rows / 64 * across, matrix = blockIdx.x / plane, in = blockIdx.x % plane;
  const int64_t r0 = in / across * 64, c0 = in % across * 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T* G = (const T*)a.G + matrix * a.stride;
  float v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {  // in flight before the sums are
    const int64_t r = r0 + 4 * i + wave, c = c0 + lane;
    v[i] = r < a.rows && c < a.cols ? to_f32(G[r * a.ld + c]) : 0.0f;
  }
  double sum = 0.0;  // every wave by itself, in the same order
#pragma unroll
  for (int i = 0; i < kMostParts; i += 64) sum += lane + i < a.parts ? a.sums[matrix * a.parts + lane + i] : 0.0;
  sum = sum_of_wave(sum);
  const double by = sum == 0.0 ? 0.0 : sum > 1.7e308 || sum != sum ? (double)NAN : (double)kUnit / sqrt(sum);
#pragma unroll
  for (int i = 0; i < 16; ++i) tile[4 * i + wave][lane] = (float)((double)v[i] * by);
  __syncthreads();
  constexpr int R = kRow<FINE>;
  constexpr float unit = FINE ? 1.0f : kRest;  // of rests
  _Float16 *X = a.X + matrix * a.n * a.m * R, *Y = a.Y + matrix * a.n * a.m * R;
  // as G lies: Y (with its rest) where G is tall, else X
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = 32 * i + tid / 8, c = tid % 8 * 8;
    _Float16 hi[8], lo[8], thi[8], tlo[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float x = tile[row][c + k], y = tile[c + k][row];
      hi[k] = (_Float16)x;
      lo[k] = (_Float16)((x - (float)hi[k]) * unit);
      thi[k] = (_Float16)y;
      tlo[k] = (_Float16)((y - (float)thi[k]) * unit);
    }
    const int64_t straight = (r0 + row) * cols * R + c0 + c, turned = (c0 + row) * rows * R + r0 + c;
    _Float16 *s = a.transposed ? X : Y, *t = a.transposed ? Y : X;
    *(i32x4_t*)(s + straight) = *(const i32x4_t*)hi;
    *(i32x4_t*)(t + turned) = *(const i32x4_t*)thi;
    if constexpr (FINE) {
      *(i32x4_t*)(s + straight + cols) = *(const i32x4_t*)lo;
      *(i32x4_t*)(t + turned + rows) = *(const i32x4_t*)tlo;
    } else {
      _Float16* rest = a.rest + matrix * a.n * a.m;
      *(i32x4_t*)(rest + (a.transposed ? turned : straight)) = *(const i32x4_t*)(a.transposed ? tlo : lo);
    }
  }
}

// -- host ---------------------------------------------------------------------

struct Layout {
  int64_t n, m;  // padded sides
  int64_t sums, X, Y0, Y1, rest, S, T, dA, dB, all;
};

Layout layout(int64_t rows, int64_t cols, int64_t batch, bool fine) {
  Layout l{};
  const int64_t size = fine ? 4 : 2;  // of a value
  l.n = ceil_div(rows < cols ? rows : cols, kPad) * kPad;
  l.m = ceil_div(rows < cols ? cols : rows, kPad) * kPad;
  const auto take = [&](int64_t bytes) {
    const int64_t at = l.all;
    l.all += ceil_div(bytes, 256) * 256;
    return at;
  };
  l.sums = take(batch * kMostParts * 8);
  l.X = take(batch * l.n * l.m * size);
  l.Y0 = take(batch * l.n * l.m * size);
  l.Y1 = take(batch * l.n * l.m * size);
  l.rest = take(fine ? 0 : batch * l.n * l.m * 2);
  l.S = take(batch * l.n * l.n * size);
  l.T = take(batch * l.n * l.n * size);
  l.dA = take(batch * l.n * 4);
  l.dB = take(batch * l.n * 4);
  return l;
}

// Sides, and what the launches hold: workgroups for 64 x 64 of the padded matrices, and
// kMostParts of each.
bool orth_sizes(int64_t rows, int64_t cols, int64_t batch) {
  if (rows < 0 || cols < 0 || batch < 0 || rows > WS_ORTHOGONAL_SIDE || cols > WS_ORTHOGONAL_SIDE) return false;
  return rows == 0 || cols == 0 ||
         (batch <= max_workgroups(256) / kMostParts && 4 * ceil_div(rows, kPad) * ceil_div(cols, kPad) * batch <= max_workgroups(256));
}

template <bool FINE>
auto start_kernel(int32_t dtype) {
  return dtype == WS_OUT_F32 ? &orth_start_kernel<float, FINE> : dtype == WS_OUT_BF16 ? &orth_start_kernel<bf16_t, FINE> : &orth_start_kernel<f16_t, FINE>;
}

// Where operands of one binary16 value would cost more than the rounding to bf16, 1.7e-3 in
// norm.  Products T X leave the rest of X out: where a part of the directions stands out,
// that is noise in the others.  The largest error after five steps of operands of one value that a
// replay over many spectra found (a quarter to half of the singular values 1, the others
// 1/1000): 4.3e-3 for 128 rows, 3.0e-3 for 256, 2.3e-3 for 400, 1.95e-3 for 512, 1.7e-3 for 640 and more; after
// twenty 2e-2.  Of two: 2e-5 after five steps, 1e-4 after twenty.  us of two and of one,
// five steps: 200 x 700 125 and 102, 128 x 4096 203 and 146, 384 x 384 121 and 101,
// 512 x 4096 253 and 190, 1000 x 2500 315 and 203, 16 of 1024 x 2048 2540 and 1230.
constexpr int64_t kFineSide = 384;
constexpr int32_t kCoarseSteps = 5;
bool in_two_values(int64_t rows, int64_t cols, int32_t steps) { return (rows < cols ? rows : cols) <= kFineSide || steps > kCoarseSteps; }

// Launches tiles of 32 WM x 32 WN.
template <int WM, int WN, int STAGES, int KIND, bool FINE = false>
ws_status launch_tiles(OrthArgs a, hipStream_t stream) {
  typedef OrthShape<WM, WN, STAGES, FINE> Shape;
  if (a.quarters) a.count *= 4;
  const uint32_t most = (uint32_t)compute_units() * Shape::kWaves;
  a.tile_groups = (int32_t)(a.count < most ? a.count : most);
  const auto kernel = [] {
    if constexpr (FINE) return &orth_fine_kernel<WM, WN, STAGES, KIND>;
    else return &orth_step_kernel<WM, WN, STAGES, KIND>;
  }();
  static std::atomic<uint64_t> allowed;
  const ws_status s = allow_lds((const void*)kernel, Shape::kLds, allowed);
  if (s != WS_OK) return s;
  return launch("orthogonalize", kernel, a.tile_groups, 256, Shape::kLds, stream, a);
}

// Tiles of 256 x 256 where they fill the card.  What their last round leaves of half the
// card or less runs in quarters, in a launch of its own (16 x 2048 x 4096: X X^T 300 us,
// so 340; A^2 190, so 212).  Fewer: 128 x 128, two workgroups a CU, or with a long ring
// where there is one a CU (1024 x 1024: 147 us for five steps, with two stages 252); 64 x 64
// where even these would leave CUs without work (1024 columns of 2560: X X^T 13 us, in
// 128 x 128 31), and for short contractions (4 x 188 x 1358: 125 us, in 128 x 128 142;
// 2500 x 1000 the other way round, 214 and 208).
// FINE, whose blocks have three times the products: 128 x 128 from four rounds on (16 of
// 384 x 4096: 966 us, in 64 x 64 1001; below, 100 of 250 x 300 472 and 361), else 64 x 64,
// with a long ring where there is one a CU (128 x 4096 203, with two stages 253).
template <int KIND, bool FINE>
ws_status run_tiles(OrthArgs a, hipStream_t stream) {
  constexpr bool kSymmetric = KIND == kGram || KIND == kSquare;
  const auto cut = [&](int side) {
    a.tiles_m = (int32_t)ceil_div(a.M, side);
    a.tiles_n = (int32_t)ceil_div(a.N, side);
    a.plane = kSymmetric ? a.tiles_m * (a.tiles_m + 1) / 2 : a.tiles_m * a.tiles_n;
    a.first = 0;
    a.count = a.plane * (uint32_t)a.batch;
    a.quarters = 0;
  };
  const uint32_t cus = (uint32_t)compute_units();
  if constexpr (FINE) {
    cut(128);
    if (a.count > 4 * cus) return launch_tiles<4, 4, 2, KIND, true>(a, stream);
    cut(64);
    if (a.count > cus) return launch_tiles<2, 2, 2, KIND, true>(a, stream);
    return launch_tiles<2, 2, 4, KIND, true>(a, stream);
  } else {
    cut(256);
    if (a.count < cus) {
      cut(128);
      if (a.count > cus) return launch_tiles<4, 4, 2, KIND>(a, stream);
      if (4 * a.count > cus && a.K > 512) return launch_tiles<4, 4, 4, KIND>(a, stream);
      cut(64);
      if (a.count > cus) return launch_tiles<2, 2, 2, KIND>(a, stream);
      return launch_tiles<2, 2, 8, KIND>(a, stream);
    }
    const uint32_t rest = a.count % cus <= cus / 2 ? a.count % cus : 0;
    a.count -= rest;
    const ws_status s = launch_tiles<8, 8, 2, KIND>(a, stream);
    if (s != WS_OK || rest == 0) return s;
    a.first = a.count;
    a.count = rest;
    a.quarters = 1;
    return launch_tiles<4, 4, 2, KIND>(a, stream);
  }
}

template <bool FINE>
ws_status run_steps(const OrthArgs& gram, const OrthArgs& square, OrthArgs apply, _Float16* Y0, _Float16* Y1, int steps, hipStream_t stream) {
  ws_status s = WS_OK;
  for (int i = 0; i < steps && s == WS_OK; ++i) {
    s = run_tiles<kGram, FINE>(gram, stream);
    if (s == WS_OK) s = run_tiles<kSquare, FINE>(square, stream);
    apply.A = i & 1 ? Y1 : Y0;
    apply.to = i & 1 ? Y0 : Y1;
    if (s == WS_OK) s = i + 1 < steps ? run_tiles<kApply, FINE>(apply, stream) : run_tiles<kLast, FINE>(apply, stream);
  }
  return s;
}

}  // namespace
}  // namespace wsg

using namespace wsg;

extern "C" {

int64_t ws_orthogonal_workspace(int64_t rows, int64_t cols, int32_t batch) {
  if (!orth_sizes(rows, cols, batch)) return -1;
  if (rows == 0 || cols == 0 || batch == 0) return 0;
  // which of them runs depends on the steps
  const int64_t tiles = layout(rows, cols, batch, true).all;
  const int64_t few = (rows < cols ? rows : cols) > kFewRows ? 0 : few_workspace(rows, cols, batch);
  return few > tiles ? few : tiles;
}

ws_status ws_orthogonalize(const ws_matrix* G, int32_t steps, const ws_matrix* out, void* workspace, int64_t workspace_bytes,
                           hipStream_t stream) {
  if (!valid(G, true) || !valid(out, true) || G->rows != out->rows || G->cols != out->cols || G->batch != out->batch ||
      out->dtype != WS_OUT_BF16 || steps < 1 || steps > WS_ORTHOGONAL_STEPS)
    return WS_ERR_INVALID_ARG;
  const int64_t need = ws_orthogonal_workspace(G->rows, G->cols, G->batch);
  if (need < 0 || workspace_bytes < need || (need > 0 && (!workspace || (uintptr_t)workspace % 256))) return WS_ERR_INVALID_ARG;
  if (need == 0) return WS_OK;
  if (by_gram_matrix(G->rows, G->cols, steps)) return orthogonalize_few(G, steps, out, workspace, stream);
  const bool fine = in_two_values(G->rows, G->cols, steps);
  const int64_t row = fine ? 2 : 1;
  const Layout l = layout(G->rows, G->cols, G->batch, fine);
  uint8_t* w = (uint8_t*)workspace;
  OrthStartArgs s{};
  s.G = G->data;
  s.rows = G->rows;
  s.cols = G->cols;
  s.ld = G->ld;
  s.stride = G->stride;
  s.sums = (double*)(w + l.sums);
  s.transposed = G->rows <= G->cols;
  s.X = (_Float16*)(w + l.X);
  s.Y = (_Float16*)(w + l.Y0);
  s.rest = (_Float16*)(w + l.rest);
  s.n = l.n;
  s.m = l.m;
  const int64_t parts = ceil_div(G->rows * G->cols, 8 * kSumThreads * 4);
  s.parts = (int32_t)(parts < kMostParts ? parts : kMostParts);
  const int64_t grid = l.n / 64 * (l.m / 64) * G->batch;
  ws_status st = launch("orthogonalize", G->dtype == WS_OUT_F32 ? &orth_sum_kernel<float> : G->dtype == WS_OUT_BF16 ? &orth_sum_kernel<bf16_t>
                                                                                                                   : &orth_sum_kernel<f16_t>,
                        (int64_t)s.parts * G->batch, kSumThreads, 0, stream, s);
  if (st == WS_OK)
    st = launch("orthogonalize", fine ? start_kernel<true>(G->dtype) : start_kernel<false>(G->dtype), grid, 256, 0, stream, s);
  OrthArgs gram{}, square{}, apply{};
  gram.batch = square.batch = apply.batch = G->batch;
  gram.A = gram.B = (const _Float16*)(w + l.X);
  gram.stride_a = gram.stride_b = l.n * l.m * row;
  gram.M = gram.N = (int32_t)l.n;
  gram.K = (int32_t)l.m;
  gram.to = gram.mirror = (_Float16*)(w + l.S);
  gram.stride_to = gram.stride_mirror = l.n * l.n * row;
  gram.d_out = (float*)(w + l.dA);
  gram.stride_d = square.stride_d = apply.stride_d = l.n;
  square.A = square.B = (const _Float16*)(w + l.S);
  square.stride_a = square.stride_b = l.n * l.n * row;
  square.M = square.N = square.K = (int32_t)l.n;
  square.to = square.mirror = (_Float16*)(w + l.T);
  square.stride_to = square.stride_mirror = l.n * l.n * row;
  square.d_in = (const float*)(w + l.dA);
  square.d_out = (float*)(w + l.dB);
  apply.B = (const _Float16*)(w + l.T);
  apply.stride_a = apply.stride_to = apply.stride_mirror = l.n * l.m * row;
  apply.stride_b = l.n * l.n * row;
  apply.M = (int32_t)l.m;
  apply.N = apply.K = (int32_t)l.n;
  apply.mirror = (_Float16*)(w + l.X);
  apply.d_in = (const float*)(w + l.dB);
  apply.rest = (_Float16*)(w + l.rest);
  apply.out = (uint16_t*)out->data;
  apply.ld_out = out->ld;
  apply.stride_out = out->stride;
  apply.rows = (int32_t)out->rows;
  apply.cols = (int32_t)out->cols;
  apply.transposed = s.transposed;
  if (st != WS_OK) return st;
  _Float16 *Y0 = (_Float16*)(w + l.Y0), *Y1 = (_Float16*)(w + l.Y1);
  return fine ? run_steps<true>(gram, square, apply, Y0, Y1, steps, stream) : run_steps<false>(gram, square, apply, Y0, Y1, steps, stream);
}

}  // extern "C"
