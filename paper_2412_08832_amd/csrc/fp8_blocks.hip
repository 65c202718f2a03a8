// fp8_blocks.hip -- e4m3 codes with a scale for each block of 128, and their products.
//
// A block of 128 values y has amax = max |y| (NaN ignored unless all are NaN), scale =
// amax / 448 and codes e4m3(y * (448 / amax)), the quotients correctly rounded in fp32
// and 448 / amax taken as 0 where it is not finite: y ~ code * scale, as for the
// library's per-row codes.  The product of row codes A (m x k) and B (n x k) is
//
//   out[i][j] = sum_b sa[i][b] * sb[j][b] * sum_{k in block b} A[i][k] * B[j][k],
//
// where sb has one row per row of B or one per 128 of them.  The outer sum is an fp32 fma
// per block, and the result is rounded once.  The inner sum is made by the matrix cores:
//   - 16-bit outputs: one MFMA 16x16x128 on the codes.  Its products are exact, but its
//     adder keeps about 17 bits below the largest of the products it adds: measured on
//     N(0, 1) operands 1.3e-5 of the result, a twentieth of fp16's rounding and a hundredth
//     of bf16's.  (The older MFMA 16x16x32 for FP8 measures the same.)
//   - 32-bit outputs: the codes widened to bf16, exactly, and four MFMA 16x16x32 for bf16,
//     which add in full fp32 (1e-8 for 128 products) at half the rate.

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "hadacore.h"
#include "internal.h"

namespace hadacore {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef int i8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));

constexpr int kWave = 64;
constexpr int kBlock = 128;

// ---- groups of rows --------------------------------------------------------------
//
// `ends` holds the end of each group among `rows` rows, in order: group g is rows
// [ends[g - 1], ends[g]), group 0 starts at 0.  Ends are clamped to [0, rows], so that
// a wrong one gives wrong rows but no access out of bounds.

struct Piece {
  int group;   // which group (groups: the rows after the last end); -1: there is no such piece
  int low;     // first row of the piece
  int high;    // end of its group
};

__device__ __forceinline__ int clamp_end(int e, int rows) {
  return e < 0 ? 0 : e > rows ? rows : e;
}

// Piece `id` of the groups cut into pieces of `unit` rows: group 0's first, then group
// 1's, ...  With `rest` the rows after the last end are one more group.  Called by
// whole waves; 64 groups at a time by a prefix sum over the lanes.
__device__ __forceinline__ Piece find_piece(const int32_t *ends, int groups, int rows, int unit,
                                            int id, bool rest) {
  const int lane = threadIdx.x & (kWave - 1);
  int base = 0;
  const int all = groups + (rest ? 1 : 0);
  for (int g0 = 0; g0 < all; g0 += kWave) {
    const int g = g0 + lane;
    int low = 0, high = 0;
    if (g < all) {
      low = g > 0 ? clamp_end(ends[g - 1], rows) : 0;
      high = g < groups ? clamp_end(ends[g], rows) : rows;
    }
    const int count = high > low ? high - low : 0;
    const int pieces = (count + unit - 1) / unit;
    int sum = pieces;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const int other = __shfl_up(sum, d);
      if (lane >= d) sum += other;
    }
    const uint64_t hit = __ballot(pieces > 0 && id >= base + sum - pieces && id < base + sum);
    if (hit != 0) {
      const int at = __builtin_ctzll(hit);
      const int first = base + __builtin_amdgcn_readlane(sum - pieces, at);
      const int lo = __builtin_amdgcn_readlane(low, at);
      return {g0 + at, lo + (id - first) * unit, __builtin_amdgcn_readlane(high, at)};
    }
    base += __builtin_amdgcn_readlane(sum, kWave - 1);
  }
  return {-1, 0, 0};
}

// The blocks of 128 rows before group g, and in it, with every group padded to whole
// blocks.  Called by whole waves.
__device__ __forceinline__ void group_blocks(const int32_t *ends, int groups, int rows, int g,
                                             int &before, int &count) {
  const int lane = threadIdx.x & (kWave - 1);
  int sum = 0, own = 0;
  for (int i = lane; i <= g && i < groups; i += kWave) {
    const int low = i > 0 ? clamp_end(ends[i - 1], rows) : 0;
    const int high = clamp_end(ends[i], rows);
    const int b = high > low ? (high - low + kBlock - 1) / kBlock : 0;
    if (i < g)
      sum += b;
    else
      own = b;
  }
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) {
    sum += __shfl_xor(sum, d);
    own += __shfl_xor(own, d);
  }
  before = __builtin_amdgcn_readfirstlane(sum);
  count = __builtin_amdgcn_readfirstlane(own);
}

// ---- quantizers ------------------------------------------------------------------

template <int DT>
__device__ __forceinline__ float widen(uint32_t h) {
  if constexpr (DT == HADACORE_FP16) {
    return (float)__builtin_bit_cast(_Float16, (uint16_t)h);
  } else {
    return __builtin_bit_cast(float, h << 16);
  }
}

// 8 values of a row from `p` on, of which the first `valid` exist (the others are 0).
// Rows may start at any 2-byte address; the hardware takes 16-byte loads from there.
template <int DT>
__device__ __forceinline__ void load8(const uint16_t *p, int valid, float (&v)[8]) {
  typedef u4 u4_any __attribute__((aligned(2)));
  if (valid >= 8) {
    const u4 r = *reinterpret_cast<const u4_any *>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = widen<DT>(r[j] & 0xFFFFu);
      v[2 * j + 1] = widen<DT>(r[j] >> 16);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < valid ? widen<DT>(p[j]) : 0.0f;
  }
}

// Maximum that ignores NaN (fmaxf returns the other operand).
__device__ __forceinline__ float abs_max(const float (&v)[8]) {
  float a = fabsf(v[0]);
#pragma unroll
  for (int j = 1; j < 8; ++j) a = fmaxf(a, fabsf(v[j]));
  return a;
}

__device__ __forceinline__ float inverse_scale(float amax) {
  const float inv = 448.0f / amax;
  return inv < __builtin_inff() ? inv : 0.0f;  // Inf and NaN: 0
}

// 4 codes, round to nearest even.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

__device__ __forceinline__ u2 codes8(const float (&v)[8], float mul) {
  return u2{codes4(v[0] * mul, v[1] * mul, v[2] * mul, v[3] * mul),
            codes4(v[4] * mul, v[5] * mul, v[6] * mul, v[7] * mul)};
}

__device__ __forceinline__ void store_codes8(uint8_t *p, u2 c, int valid) {
  if (valid >= 8) {
    *reinterpret_cast<u2 *>(p) = c;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < valid) p[j] = (uint8_t)(c[j / 4] >> (8 * (j % 4)));
  }
}

// Rows rotated by 2^L <= 64 values: 16 lanes hold a block of 128, 8 consecutive values
// each, so the stages on index bits 0-2 are in registers and those on bits 3-5 between
// lanes.  HBM-bound: one 16-byte load and one 8-byte store per lane.
template <int DT, int L>
__global__ __launch_bounds__(256) void short_rotation_kernel(
    const uint16_t *in, int64_t in_stride, uint8_t *codes, int64_t codes_stride, float *scales,
    int64_t scales_stride, int64_t m, int k, int blocks, float scale) {
  const int sub = threadIdx.x & 15;
  const int64_t total = m * blocks, step = (int64_t)gridDim.x * 16;
  // every lane of a wave takes part in the exchanges, so the bound is the wave's
  for (int64_t i0 = (int64_t)blockIdx.x * 16 + (threadIdx.x / kWave) * 4; i0 < total; i0 += step) {
    const int64_t i = i0 + ((threadIdx.x >> 4) & 3);
    const int64_t row = i < total ? i / blocks : 0;
    const int block = i < total ? (int)(i - row * blocks) : 0;
    const int col = block * kBlock + sub * 8;
    const int valid = i < total ? k - col : 0;
    float v[8];
    load8<DT>(in + row * in_stride + col, valid, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= scale;
#pragma unroll
    for (int b = 0; b < 3; ++b) {
      if (b >= L) break;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if ((j & (1 << b)) == 0) {
          const float x = v[j], y = v[j | (1 << b)];
          v[j] = x + y;
          v[j | (1 << b)] = x - y;
        }
      }
    }
#pragma unroll
    for (int b = 3; b < 6; ++b) {
      if (b >= L) break;
      const int bit = 1 << (b - 3);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float other = __shfl_xor(v[j], bit);
        v[j] = (sub & bit) != 0 ? other - v[j] : v[j] + other;
      }
    }
    float a = abs_max(v);
#pragma unroll
    for (int d = 1; d < 16; d *= 2) a = fmaxf(a, __shfl_xor(a, d));
    if (valid > 0) {
      store_codes8(codes + row * codes_stride + col, codes8(v, inverse_scale(a)), valid);
      if (sub == 0) scales[row * scales_stride + block] = a / 448.0f;
    }
  }
}

template <int DT>
hipError_t short_rotations(const uint16_t *in, int64_t in_stride, uint8_t *codes,
                           int64_t codes_stride, float *scales, int64_t scales_stride, int64_t m,
                           int k, int L, float scale, hipStream_t stream) {
  const int blocks = (k + kBlock - 1) / kBlock;
  const int64_t groups = (m * blocks + 15) / 16;
  const dim3 grid((uint32_t)(groups < (1 << 20) ? groups : (1 << 20)));
  const auto go = [&](auto l) {
    hipLaunchKernelGGL((short_rotation_kernel<DT, decltype(l)::value>), grid, dim3(256), 0, stream,
                       in, in_stride, codes, codes_stride, scales, scales_stride, m, k, blocks,
                       scale);
    return hipGetLastError();
  };
  switch (L) {
    case 0: return go(std::integral_constant<int, 0>{});
    case 1: return go(std::integral_constant<int, 1>{});
    case 2: return go(std::integral_constant<int, 2>{});
    case 3: return go(std::integral_constant<int, 3>{});
    case 4: return go(std::integral_constant<int, 4>{});
    case 5: return go(std::integral_constant<int, 5>{});
    case 6: return go(std::integral_constant<int, 6>{});
    default: return hipErrorInvalidValue;
  }
}

// Tiles of 128 x 128 (columns = false: one scale per tile, codes as the input lies and,
// where asked, transposed) or the columns of 128 rows (columns = true: one scale per
// column and 128 rows, transposed codes only).  A workgroup takes one tile: thread t
// holds the 8 x 8 square of rows 8 * (t / 16) and columns 8 * (t % 16), whose codes it
// transposes in registers; the transposed tile goes through LDS so that its rows leave
// as whole 128-byte lines.  HBM-bound.
struct TileArgs {
  const uint16_t *in;
  int64_t in_stride, in_batch;
  uint8_t *codes;
  int64_t codes_stride, codes_batch;
  uint8_t *codes_t;
  int64_t codes_t_stride, codes_t_batch;
  float *scales;
  int64_t scales_stride, scales_batch;
  const int32_t *ends;  // columns: groups of rows, or null for one group of all
  int groups;
  int m, k;
};

// Byte j of four words, as the word of their transposed square.
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d,
                                           uint32_t (&t)[4]) {
  const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u);  // a0 b0 a1 b1
  const uint32_t ab2 = __builtin_amdgcn_perm(b, a, 0x07030602u);  // a2 b2 a3 b3
  const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u);
  const uint32_t cd2 = __builtin_amdgcn_perm(d, c, 0x07030602u);
  t[0] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
  t[1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
  t[2] = __builtin_amdgcn_perm(cd2, ab2, 0x05040100u);
  t[3] = __builtin_amdgcn_perm(cd2, ab2, 0x07060302u);
}

template <int DT, bool COLUMNS>
__global__ __launch_bounds__(256) void tile_kernel(TileArgs p) {
  // transposed codes: row c of 128 bytes, its 8-byte words at (word ^ (c / 8)): the 16
  // threads that write one word of 16 rows then use different banks
  __shared__ __align__(16) u2 turned[kBlock * 16];
  __shared__ float maxima[4][kBlock];
  const int t = threadIdx.x, wave = t / kWave;
  const int rg = t >> 4, cg = t & 15;
  const int col0 = blockIdx.x * kBlock;
  const int out_block = blockIdx.y;  // block of rows of the output (a padded one for columns)
  int row0 = out_block * kBlock, row_end = p.m;
  if constexpr (COLUMNS) {
    if (p.ends != nullptr) {
      const Piece piece = find_piece(p.ends, p.groups, p.m, kBlock, out_block, false);
      row0 = piece.low;
      row_end = piece.group < 0 ? 0 : piece.high;
    }
  }
  const uint16_t *in = p.in + blockIdx.z * p.in_batch;
  const int col = col0 + cg * 8;
  float v[8][8];
  const int rows = row_end - row0;  // <= 0: a block past the last group, all zero
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = rg * 8 + i;
    load8<DT>(in + (int64_t)(row0 + r) * p.in_stride + col, r < rows ? p.k - col : 0, v[i]);
  }
  float mul[8];
  if constexpr (COLUMNS) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float a = fabsf(v[0][j]);
#pragma unroll
      for (int i = 1; i < 8; ++i) a = fmaxf(a, fabsf(v[i][j]));
      a = fmaxf(a, __shfl_xor(a, 16));
      a = fmaxf(a, __shfl_xor(a, 32));
      if ((t & 48) == 0) maxima[wave][cg * 8 + j] = a;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = cg * 8 + j;
      const float a = fmaxf(fmaxf(maxima[0][c], maxima[1][c]), fmaxf(maxima[2][c], maxima[3][c]));
      mul[j] = inverse_scale(a);
      if (rg == 0 && col + j < p.k)
        p.scales[(int64_t)(col + j) * p.scales_stride + out_block] = a / 448.0f;
    }
  } else {
    float a = abs_max(v[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) a = fmaxf(a, abs_max(v[i]));
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) a = fmaxf(a, __shfl_xor(a, d));
    if ((t & 63) == 0) maxima[wave][0] = a;
    __syncthreads();
    a = fmaxf(fmaxf(maxima[0][0], maxima[1][0]), fmaxf(maxima[2][0], maxima[3][0]));
    const float inv = inverse_scale(a);
#pragma unroll
    for (int j = 0; j < 8; ++j) mul[j] = inv;
    if (t == 0)
      p.scales[blockIdx.z * p.scales_batch + out_block * p.scales_stride + blockIdx.x] = a / 448.0f;
  }
  uint32_t words[8][2];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      words[i][h] = codes4(v[i][4 * h] * mul[4 * h], v[i][4 * h + 1] * mul[4 * h + 1],
                           v[i][4 * h + 2] * mul[4 * h + 2], v[i][4 * h + 3] * mul[4 * h + 3]);
    if constexpr (!COLUMNS) {
      const int r = rg * 8 + i;
      if (r < rows)
        store_codes8(p.codes + blockIdx.z * p.codes_batch + (int64_t)(row0 + r) * p.codes_stride +
                         col,
                     u2{words[i][0], words[i][1]}, p.k - col);
    }
  }
  if (!COLUMNS && p.codes_t == nullptr) return;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t low[4], high[4];
    transpose4(words[0][h], words[1][h], words[2][h], words[3][h], low);
    transpose4(words[4][h], words[5][h], words[6][h], words[7][h], high);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = cg * 8 + h * 4 + j;
      turned[c * 16 + (rg ^ cg)] = u2{low[j], high[j]};
    }
  }
  __syncthreads();
  // transposed rows are padded to whole blocks for columns, and end at m for tiles
  const int left = COLUMNS ? kBlock : rows;
  uint8_t *out = p.codes_t + blockIdx.z * p.codes_t_batch + (int64_t)out_block * kBlock;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = i * 16 + rg;  // 16 threads write the 128 bytes of one transposed row
    if (col0 + c < p.k)
      store_codes8(out + (int64_t)(col0 + c) * p.codes_t_stride + cg * 8,
                   turned[c * 16 + (cg ^ (c >> 3))], left - cg * 8);
  }
}

// ---- products ------------------------------------------------------------------

constexpr int kTiles = 0;     // all rows of A with one B
constexpr int kGroups = 1;    // groups of rows of A, each with its own B
constexpr int kGradient = 2;  // groups of blocks of k, each with its own output

struct ProductArgs {
  const uint8_t *a;
  int64_t a_pitch;
  const float *sa;
  int64_t sa_pitch;
  const uint8_t *b;
  int64_t b_pitch, b_batch;
  const float *sb;
  int64_t sb_pitch, sb_batch;
  void *out;
  int64_t out_pitch, out_batch;
  const int32_t *ends;
  int groups;
  int m, n, k;
  int tiles_m, tiles_n;  // the grid (kGradient: of each group)
  int kind, out_type;
};

// 16 bytes of LDS per lane at `lds` + 16 * lane from base + offset, asynchronously.
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t base, void *lds, int offset,
                                            int uniform_offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(
      base, (__attribute__((address_space(3))) void *)lds, 16, offset, uniform_offset, 0, 0);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t uniform_rsrc(const void *base) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  const uint64_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b);
  const uint64_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>((hi << 32) | lo), (short)0,
                                           -1, 0x00020000);
}

// The first `valid` of 16 bytes.
__device__ __forceinline__ u4 first_bytes(u4 v, int valid) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int n = valid - 4 * j;
    v[j] = n >= 4 ? v[j] : n <= 0 ? 0u : v[j] & ((1u << (8 * n)) - 1u);
  }
  return v;
}

template <int OUT>
__device__ __forceinline__ void store_out(void *out, int64_t at, float v) {
  if constexpr (OUT == HADACORE_FP32) {
    static_cast<float *>(out)[at] = v;
  } else if constexpr (OUT == HADACORE_FP16) {
    static_cast<_Float16 *>(out)[at] = (_Float16)v;
  } else {
    static_cast<__bf16 *>(out)[at] = (__bf16)v;
  }
}

template <int OUT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (OUT == HADACORE_FP16) {
    return __builtin_bit_cast(uint32_t, h2{(_Float16)a, (_Float16)b});
  } else {
    return __builtin_bit_cast(uint32_t, bf2{(__bf16)a, (__bf16)b});
  }
}

// 16 consecutive outputs of a row, of which the first `valid` exist.
template <int OUT>
__device__ __forceinline__ void store_row16(void *out, int64_t at, const float (&v)[16], int valid,
                                            bool aligned) {
  if (valid >= 16 && aligned) {
    if constexpr (OUT == HADACORE_FP32) {
      f4 *p = reinterpret_cast<f4 *>(static_cast<float *>(out) + at);
#pragma unroll
      for (int q = 0; q < 4; ++q) p[q] = f4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    } else {
      u4 *p = reinterpret_cast<u4 *>(static_cast<uint16_t *>(out) + at);
#pragma unroll
      for (int q = 0; q < 2; ++q)
        p[q] = u4{pack2<OUT>(v[8 * q], v[8 * q + 1]), pack2<OUT>(v[8 * q + 2], v[8 * q + 3]),
                  pack2<OUT>(v[8 * q + 4], v[8 * q + 5]), pack2<OUT>(v[8 * q + 6], v[8 * q + 7])};
    }
  } else {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (j < valid) store_out<OUT>(out, at + j, v[j]);
  }
}

// An operand of one lane: 32 codes of a row, or the same widened to bf16, 8 for each of
// four MFMAs.
template <bool FULL>
struct Operand {
  i8v codes;
  __device__ __forceinline__ void set(i8v c) { codes = c; }
  __device__ __forceinline__ static f4 product(const Operand &x, const Operand &y) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x.codes, y.codes, f4{0, 0, 0, 0}, 0, 0,
                                                            0, 0, 0, 0);
  }
};

template <>
struct Operand<true> {
  bf8 values[4];
  __device__ __forceinline__ void set(i8v c) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bf2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * s + h], 1.0f, false);
        const bf2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[2 * s + h], 1.0f, true);
        values[s][4 * h] = lo[0];
        values[s][4 * h + 1] = lo[1];
        values[s][4 * h + 2] = hi[0];
        values[s][4 * h + 3] = hi[1];
      }
    }
  }
  __device__ __forceinline__ static f4 product(const Operand &x, const Operand &y) {
    f4 r = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < 4; ++s)
      r = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.values[s], y.values[s], r, 0, 0, 0);
    return r;
  }
};

// A tile of BM x BN outputs by WM x WN waves, from LDS tiles of 128 bytes of k that are
// loaded one step ahead.
//
// B is the MFMA's first operand and A its second, so a lane's four results are four
// columns n of one row m: its A scale is one value, and its stores are along the row.
// Lane l of an MFMA holds 32 bytes of row l & 15 of either operand: the 16-byte chunks
// g and g + 4, g = l >> 4, of the 128 (any order of k will do that both share).  The rows
// of B are laid out in LDS so that row 16 j + i of 64 is column 16 (i / 4) + 4 j + i % 4 of
// the tile: lane group g then holds columns 16 g .. 16 g + 15 over its four MFMAs.
//
// LDS rows are 128 bytes; chunk c of row r lies at c ^ ((r >> 1) & 7), which the loads
// obey by choosing their global chunk, since LDS addresses of a load run with the lane.
template <int BM, int BN, int WM, int WN, bool BROWS, bool FULL>
__global__ __launch_bounds__(WM *WN *kWave) void product_kernel(ProductArgs p) {
  constexpr int kThreads = WM * WN * kWave;
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16;  // MFMA tiles of a wave
  static_assert(TN % 4 == 0 && (BN / WN) <= kBlock, "a wave's columns are in one block of B");
  constexpr int kLoadsA = BM * 8 / kThreads, kLoadsB = BN * 8 / kThreads;
  constexpr int SB = BROWS ? BN : BN / kBlock > 0 ? BN / kBlock : 1;
  __shared__ __align__(16) uint8_t tile_a[2][BM * kBlock];
  __shared__ __align__(16) uint8_t tile_b[2][BN * kBlock];
  __shared__ __align__(16) float scale_a[2][BM];
  __shared__ __align__(16) float scale_b[2][SB];

  const int t = threadIdx.x, lane = t & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(t / kWave);
  const int wm = wave / WN, wn = wave % WN;
  const int g = lane >> 4, li = lane & 15;

  // which tile
  int tile = blockIdx.x, m0, n0, m_end = p.m, kb0 = 0, kb1 = (p.k + kBlock - 1) / kBlock;
  const uint8_t *b = p.b;
  const float *sb = p.sb;
  int64_t out_at = 0;
  n0 = (tile % p.tiles_n) * BN;
  tile /= p.tiles_n;
  if (p.kind == kGroups) {
    const Piece piece = find_piece(p.ends, p.groups, p.m, BM, tile, true);
    if (piece.group < 0) return;
    m0 = piece.low;
    m_end = piece.high;
    if (m0 < 0 || m0 >= m_end) return;
    if (piece.group == p.groups) {
      kb1 = 0;  // rows after the last group: zeros
    } else {
      b += piece.group * p.b_batch;
      sb += piece.group * p.sb_batch;
    }
  } else {
    m0 = (tile % p.tiles_m) * BM;
    if (p.kind == kGradient) {
      const int group = tile / p.tiles_m;
      out_at = group * p.out_batch;
      if (p.ends != nullptr) {
        int before, count;
        group_blocks(p.ends, p.groups, p.k, group, before, count);
        kb0 = before < kb1 ? before : kb1;
        kb1 = before + count < kb1 ? before + count : kb1;
      }
    }
  }
  const __amdgpu_buffer_rsrc_t ra = uniform_rsrc(p.a + (int64_t)m0 * p.a_pitch);
  const __amdgpu_buffer_rsrc_t rb = uniform_rsrc(b + (int64_t)n0 * p.b_pitch);

  // the rows past the end repeat the last one; their results are not stored
  int off_a[kLoadsA], off_b[kLoadsB];
#pragma unroll
  for (int i = 0; i < kLoadsA; ++i) {
    const int s = i * kThreads + t, r = s >> 3;
    const int row = r < m_end - m0 ? r : m_end - m0 - 1;
    off_a[i] = row * (int)p.a_pitch + (((s & 7) ^ ((r >> 1) & 7)) << 4);
  }
#pragma unroll
  for (int i = 0; i < kLoadsB; ++i) {
    const int s = i * kThreads + t, r = s >> 3;
    const int c = (r & ~63) + 16 * ((r & 15) >> 2) + 4 * ((r >> 4) & 3) + (r & 3);
    const int row = c < p.n - n0 ? c : p.n - n0 - 1;
    off_b[i] = row * (int)p.b_pitch + (((s & 7) ^ ((r >> 1) & 7)) << 4);
  }
  const int tail = p.k & (kBlock - 1);
  const int kb_tail = tail != 0 ? p.k / kBlock : -1;
  // thread t brings the A scale of row t and the B scale of column (or block) t
  const int srow = t < m_end - m0 ? t : m_end - m0 - 1;
  const float *sa_at = p.sa + (int64_t)(m0 + srow) * p.sa_pitch;
  const int scol = BROWS ? (n0 + t < p.n ? n0 + t : p.n - 1)
                         : (n0 / kBlock + t <= (p.n - 1) / kBlock ? n0 / kBlock + t
                                                                  : (p.n - 1) / kBlock);
  const float *sb_at = sb + (int64_t)scol * p.sb_pitch;
  float next_sa = 0.0f, next_sb = 0.0f;

  const auto load = [&](int kb) {
    uint8_t *la = tile_a[kb & 1], *lb = tile_b[kb & 1];
    if (kb != kb_tail) {
#pragma unroll
      for (int i = 0; i < kLoadsA; ++i)
        load_to_lds(ra, la + (i * kThreads + wave * kWave) * 16, off_a[i], kb * kBlock);
#pragma unroll
      for (int i = 0; i < kLoadsB; ++i)
        load_to_lds(rb, lb + (i * kThreads + wave * kWave) * 16, off_b[i], kb * kBlock);
    } else {
      // the last, partial block of k: codes past it are 0
#pragma unroll
      for (int i = 0; i < kLoadsA; ++i) {
        const int s = i * kThreads + t, valid = tail - (((s & 7) ^ ((s >> 4) & 7)) << 4);
        u4 v = {0, 0, 0, 0};
        if (valid > 0)
          v = first_bytes(__builtin_amdgcn_raw_buffer_load_b128(ra, off_a[i], kb * kBlock, 0),
                          valid);
        *reinterpret_cast<u4 *>(la + s * 16) = v;
      }
#pragma unroll
      for (int i = 0; i < kLoadsB; ++i) {
        const int s = i * kThreads + t, valid = tail - (((s & 7) ^ ((s >> 4) & 7)) << 4);
        u4 v = {0, 0, 0, 0};
        if (valid > 0)
          v = first_bytes(__builtin_amdgcn_raw_buffer_load_b128(rb, off_b[i], kb * kBlock, 0),
                          valid);
        *reinterpret_cast<u4 *>(lb + s * 16) = v;
      }
    }
    if (t < BM) next_sa = sa_at[kb];
    if (t < SB) next_sb = sb_at[kb];
  };

  f4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f4{0, 0, 0, 0};

  const int key = (li >> 1) & 7;
  const int chunk0 = ((g ^ key) << 4), chunk1 = (((g + 4) ^ key) << 4);
  const auto fragment = [&](const uint8_t *tile_rows) {
    const uint8_t *row = tile_rows + li * kBlock;
    const u4 lo = *reinterpret_cast<const u4 *>(row + chunk0);
    const u4 hi = *reinterpret_cast<const u4 *>(row + chunk1);
    return i8v{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3],
               (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };

  if (kb0 < kb1) load(kb0);
  for (int kb = kb0; kb < kb1; ++kb) {
    // this step's tiles and scales have come; the barrier also ends the last step's reads
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (t < BM) scale_a[kb & 1][t] = next_sa;
    if (t < SB) scale_b[kb & 1][t] = next_sb;
    __syncthreads();
    if (kb + 1 < kb1) load(kb + 1);
    const uint8_t *la = tile_a[kb & 1] + wm * (BM / WM) * kBlock;
    const uint8_t *lb = tile_b[kb & 1] + wn * (BN / WN) * kBlock;
    Operand<FULL> fb[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j].set(fragment(lb + j * 16 * kBlock));
    f4 col[TN];
    float uniform_b = 0.0f;
    if constexpr (BROWS) {
#pragma unroll
      for (int j = 0; j < TN; ++j)
        col[j] = *reinterpret_cast<const f4 *>(
            &scale_b[kb & 1][wn * (BN / WN) + (j & ~3) * 16 + 16 * g + 4 * (j & 3)]);
    } else {
      uniform_b = scale_b[kb & 1][wn * (BN / WN) / kBlock];
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      Operand<FULL> fa;
      fa.set(fragment(la + i * 16 * kBlock));
      float s = scale_a[kb & 1][wm * (BM / WM) + i * 16 + li];
      if constexpr (!BROWS) s *= uniform_b;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const f4 r = Operand<FULL>::product(fb[j], fa);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          acc[i][j][q] = __builtin_fmaf(r[q], BROWS ? s * col[j][q] : s, acc[i][j][q]);
      }
    }
  }

  const int wide = FULL ? 4 : 2;
  const bool aligned =
      ((reinterpret_cast<uintptr_t>(p.out) | (uintptr_t)((p.out_pitch | out_at) * wide)) & 15) == 0;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int row = m0 + wm * (BM / WM) + i * 16 + li;
    if (row >= m_end) continue;
#pragma unroll
    for (int j = 0; j < TN; j += 4) {
      const int column = n0 + wn * (BN / WN) + j * 16 + 16 * g;
      float v[16];
#pragma unroll
      for (int q = 0; q < 16; ++q) v[q] = acc[i][j + q / 4][q % 4];
      const int64_t at = out_at + (int64_t)row * p.out_pitch + column;
      if constexpr (FULL)
        store_row16<HADACORE_FP32>(p.out, at, v, p.n - column, aligned);
      else if (p.out_type == HADACORE_FP16)
        store_row16<HADACORE_FP16>(p.out, at, v, p.n - column, aligned);
      else
        store_row16<HADACORE_BF16>(p.out, at, v, p.n - column, aligned);
    }
  }
}

template <int BM, int BN, int WM, int WN>
hipError_t launch_product(ProductArgs p, bool b_rows, hipStream_t stream) {
  p.tiles_n = (p.n + BN - 1) / BN;
  p.tiles_m = (p.m + BM - 1) / BM;
  int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  // ragged groups: each has at most one tile that is not full, the rows after them too
  if (p.kind == kGroups)
    tiles = ((int64_t)(p.m / BM) + (p.groups + 1 < p.m ? p.groups + 1 : p.m)) * p.tiles_n;
  if (p.kind == kGradient) tiles *= p.groups;
  if (tiles * (WM * WN * kWave) >= (int64_t(1) << 32)) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)tiles), block(WM * WN * kWave);
  const auto go = [&](auto rows, auto full) {
    hipLaunchKernelGGL(
        (product_kernel<BM, BN, WM, WN, decltype(rows)::value, decltype(full)::value>), grid,
        block, 0, stream, p);
    return hipGetLastError();
  };
  if (p.out_type == HADACORE_FP32)
    return b_rows ? go(std::true_type{}, std::true_type{}) : go(std::false_type{}, std::true_type{});
  return b_rows ? go(std::true_type{}, std::false_type{}) : go(std::false_type{}, std::false_type{});
}

hipError_t launch_product(const ProductArgs &p, bool b_rows, hipStream_t stream) {
  return launch_product<128, 128, 2, 2>(p, b_rows, stream);
}

// ---- arguments -------------------------------------------------------------------

// Rows of codes: offsets inside a tile of 256 rows stay below 2^31 bytes.
constexpr int64_t kMaxCodePitch = int64_t(1) << 22;
constexpr int64_t kMaxPitch = int64_t(1) << 26;
constexpr int64_t kMaxBytes = int64_t(1) << 42;

bool aligned_to(const void *p, uintptr_t bytes) {
  return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
}

bool is_output_type(hadacore_dtype t) {
  return t == HADACORE_FP16 || t == HADACORE_BF16 || t == HADACORE_FP32;
}

int64_t blocks_of(int64_t k) { return (k + kBlock - 1) / kBlock; }

// A batch of matrices as a byte range: `batch` of them `step` elements apart.
Span batch_span(const void *p, int64_t batch, int64_t step, int64_t rows, int64_t pitch,
                int64_t width, int64_t size) {
  Span s = span(p, rows, pitch, width, size);
  if (batch > 1 && s.hi > s.lo) s.hi += (uintptr_t)((batch - 1) * step * size);
  return s;
}

// Codes and scales of `batch` matrices: everything but the device pointers' contents.
hadacore_status check_codes(const void *codes, int64_t pitch, int64_t step, const float *scales,
                            int64_t scales_pitch, int64_t scales_step, int64_t batch, int64_t rows,
                            int64_t k, int64_t scale_rows) {
  if (pitch < k || pitch % 16 != 0 || pitch > kMaxCodePitch || scales_pitch < blocks_of(k) ||
      scales_pitch > kMaxCodePitch)
    return HADACORE_ERROR_INVALID_STRIDE;
  if (batch > 1 && (step % 16 != 0 || step < 0 || scales_step < 0))
    return HADACORE_ERROR_INVALID_STRIDE;
  if (rows * batch == 0 || k == 0) return HADACORE_SUCCESS;
  if (batch > 1 && (step > kMaxBytes / batch || scales_step > kMaxBytes / batch))
    return HADACORE_ERROR_TOO_LARGE;
  if (pitch > kMaxBytes / rows || scales_pitch > kMaxBytes / scale_rows)
    return HADACORE_ERROR_TOO_LARGE;
  if (codes == nullptr || scales == nullptr) return HADACORE_ERROR_INVALID_VALUE;
  if (!aligned_to(codes, 16) || !aligned_to(scales, 4)) return HADACORE_ERROR_MISALIGNED;
  return HADACORE_SUCCESS;
}

constexpr int64_t kMaxDim = int64_t(1) << 30;

// The checks that the three products share; `scale_rows` is that of B.
hadacore_status check_product(const ProductArgs &p, int64_t m, int64_t n, int64_t k,
                              int64_t groups, int64_t scale_rows) {
  const bool batch_b = p.kind == kGroups, batch_out = p.kind == kGradient;
  if (!is_output_type(p.out_type)) return HADACORE_ERROR_INVALID_DTYPE;
  const int size = p.out_type == HADACORE_FP32 ? 4 : 2;
  hadacore_status st = check_codes(p.a, p.a_pitch, 0, p.sa, p.sa_pitch, 0, 1, m, k, m);
  if (st != HADACORE_SUCCESS) return st;
  st = check_codes(p.b, p.b_pitch, p.b_batch, p.sb, p.sb_pitch, p.sb_batch, batch_b ? groups : 1, n,
                   k, scale_rows);
  if (st != HADACORE_SUCCESS) return st;
  if (p.out_pitch < n || p.out_pitch > kMaxPitch || (batch_out && groups > 1 && p.out_batch < 0))
    return HADACORE_ERROR_INVALID_STRIDE;
  if (m == 0 || n == 0 || (batch_out && groups == 0)) return HADACORE_SUCCESS;
  if (p.out_pitch > kMaxBytes / m || (batch_out && p.out_batch > kMaxBytes / groups))
    return HADACORE_ERROR_TOO_LARGE;
  if (p.out == nullptr) return HADACORE_ERROR_INVALID_VALUE;
  if (!aligned_to(p.out, size)) return HADACORE_ERROR_MISALIGNED;
  const Span out = batch_span(p.out, batch_out ? groups : 1, p.out_batch, m, p.out_pitch, n, size);
  const int64_t batch = batch_b ? groups : 1;
  if (spans_overlap(out, span(p.a, m, p.a_pitch, k, 1)) ||
      spans_overlap(out, span(p.sa, m, p.sa_pitch, blocks_of(k), 4)) ||
      spans_overlap(out, batch_span(p.b, batch, p.b_batch, n, p.b_pitch, k, 1)) ||
      spans_overlap(out,
                    batch_span(p.sb, batch, p.sb_batch, scale_rows, p.sb_pitch, blocks_of(k), 4)) ||
      (p.ends != nullptr && spans_overlap(out, span(p.ends, 1, groups, groups, 4))))
    return HADACORE_ERROR_OVERLAP;
  return HADACORE_SUCCESS;
}

hadacore_status check_ends(const int32_t *ends, int64_t groups) {
  if (groups > 0 && ends == nullptr) return HADACORE_ERROR_INVALID_VALUE;
  return aligned_to(ends, 4) ? HADACORE_SUCCESS : HADACORE_ERROR_MISALIGNED;
}

hadacore_status run_product(const ProductArgs &p, bool b_rows, void *stream) {
  const hadacore_status dev = check_device();
  if (dev != HADACORE_SUCCESS) return dev;
  const hipError_t e = launch_product(p, b_rows, static_cast<hipStream_t>(stream));
  return e == hipSuccess               ? HADACORE_SUCCESS
         : e == hipErrorInvalidValue ? HADACORE_ERROR_TOO_LARGE
                                     : HADACORE_ERROR_LAUNCH;
}

hadacore_status run_tiles(const TileArgs &p, bool columns, int64_t row_blocks, int64_t batch,
                          hadacore_dtype dtype, void *stream) {
  const int64_t col_blocks = blocks_of(p.k);
  if (row_blocks > 65535 || batch > 65535) return HADACORE_ERROR_TOO_LARGE;
  if (row_blocks * col_blocks * batch * 256 >= (int64_t(1) << 32)) return HADACORE_ERROR_TOO_LARGE;
  const hadacore_status dev = check_device();
  if (dev != HADACORE_SUCCESS) return dev;
  const dim3 grid((uint32_t)col_blocks, (uint32_t)row_blocks, (uint32_t)batch);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == HADACORE_FP16) {
    if (columns)
      hipLaunchKernelGGL((tile_kernel<HADACORE_FP16, true>), grid, dim3(256), 0, s, p);
    else
      hipLaunchKernelGGL((tile_kernel<HADACORE_FP16, false>), grid, dim3(256), 0, s, p);
  } else {
    if (columns)
      hipLaunchKernelGGL((tile_kernel<HADACORE_BF16, true>), grid, dim3(256), 0, s, p);
    else
      hipLaunchKernelGGL((tile_kernel<HADACORE_BF16, false>), grid, dim3(256), 0, s, p);
  }
  return hipGetLastError() == hipSuccess ? HADACORE_SUCCESS : HADACORE_ERROR_LAUNCH;
}

}  // namespace

hipError_t launch_short_rotations(const uint16_t *in, int64_t in_stride, uint8_t *codes,
                                  int64_t codes_stride, float *scales, int64_t scales_stride,
                                  int64_t m, int k, int L, hadacore_dtype dtype, float scale,
                                  hipStream_t stream) {
  return dtype == HADACORE_FP16
             ? short_rotations<HADACORE_FP16>(in, in_stride, codes, codes_stride, scales,
                                              scales_stride, m, k, L, scale, stream)
             : short_rotations<HADACORE_BF16>(in, in_stride, codes, codes_stride, scales,
                                              scales_stride, m, k, L, scale, stream);
}

}  // namespace hadacore

using namespace hadacore;

extern "C" int64_t hadacore_padded_tokens(int64_t tokens, int64_t groups) {
  if (tokens < 0 || groups < 0) return 0;
  return (tokens + (kBlock - 1) * (groups < tokens ? groups : tokens)) / kBlock * kBlock;
}

extern "C" hadacore_status hadacore_quantize_fp8_columns(
    const void *in, int64_t in_row_stride, const int32_t *ends, int64_t groups, void *out_codes,
    int64_t out_row_stride, float *out_scales, int64_t scales_row_stride, int64_t m, int64_t k,
    hadacore_dtype dtype, void *stream) {
  if (m < 0 || k < 0 || groups < 0 || (ends == nullptr && groups != 1))
    return HADACORE_ERROR_INVALID_VALUE;
  if (dtype != HADACORE_FP16 && dtype != HADACORE_BF16) return HADACORE_ERROR_INVALID_DTYPE;
  if (m >= kMaxDim || k >= kMaxDim || groups >= kMaxDim) return HADACORE_ERROR_TOO_LARGE;
  const int64_t places = hadacore_padded_tokens(m, groups), blocks = places / kBlock;
  if (in_row_stride < k || in_row_stride > kMaxPitch || out_row_stride < places ||
      out_row_stride % 16 != 0 || out_row_stride > kMaxCodePitch || scales_row_stride < blocks ||
      scales_row_stride > kMaxCodePitch)
    return HADACORE_ERROR_INVALID_STRIDE;
  if (k == 0 || places == 0) return HADACORE_SUCCESS;
  if (in == nullptr || out_codes == nullptr || out_scales == nullptr)
    return HADACORE_ERROR_INVALID_VALUE;
  if (!aligned_to(in, 2) || !aligned_to(out_codes, 16) || !aligned_to(out_scales, 4) ||
      !aligned_to(ends, 4))
    return HADACORE_ERROR_MISALIGNED;
  if (in_row_stride > kMaxBytes / m || out_row_stride > kMaxBytes / k)
    return HADACORE_ERROR_TOO_LARGE;
  const Span si = span(in, m, in_row_stride, k, 2), sc = span(out_codes, k, out_row_stride, places, 1),
             ss = span(out_scales, k, scales_row_stride, blocks, 4),
             se = span(ends, ends != nullptr, groups, groups, 4);
  if (spans_overlap(si, sc) || spans_overlap(si, ss) || spans_overlap(sc, ss) ||
      spans_overlap(se, sc) || spans_overlap(se, ss))
    return HADACORE_ERROR_OVERLAP;
  TileArgs p{};
  p.in = static_cast<const uint16_t *>(in);
  p.in_stride = in_row_stride;
  p.codes_t = static_cast<uint8_t *>(out_codes);
  p.codes_t_stride = out_row_stride;
  p.scales = out_scales;
  p.scales_stride = scales_row_stride;
  p.ends = ends;
  p.groups = (int)groups;
  p.m = (int)m;
  p.k = (int)k;
  return run_tiles(p, true, blocks, 1, dtype, stream);
}

extern "C" hadacore_status hadacore_quantize_fp8_tiles(
    const void *in, int64_t in_row_stride, int64_t in_batch_stride, void *out_codes,
    int64_t out_row_stride, int64_t out_batch_stride, void *out_codes_t, int64_t out_t_row_stride,
    int64_t out_t_batch_stride, float *out_scales, int64_t scales_row_stride,
    int64_t scales_batch_stride, int64_t batch, int64_t m, int64_t k, hadacore_dtype dtype,
    void *stream) {
  if (m < 0 || k < 0 || batch < 0) return HADACORE_ERROR_INVALID_VALUE;
  if (dtype != HADACORE_FP16 && dtype != HADACORE_BF16) return HADACORE_ERROR_INVALID_DTYPE;
  if (m >= kMaxDim || k >= kMaxDim || batch >= kMaxDim) return HADACORE_ERROR_TOO_LARGE;
  const bool turned = out_codes_t != nullptr;
  if (in_row_stride < k || in_row_stride > kMaxPitch || out_row_stride < k ||
      out_row_stride % 16 != 0 || out_row_stride > kMaxCodePitch ||
      scales_row_stride < blocks_of(k) || scales_row_stride > kMaxCodePitch ||
      (turned && (out_t_row_stride < m || out_t_row_stride % 16 != 0 ||
                  out_t_row_stride > kMaxCodePitch)))
    return HADACORE_ERROR_INVALID_STRIDE;
  if (batch > 1 && (in_batch_stride < 0 || out_batch_stride < (m - 1) * out_row_stride + k ||
                    out_batch_stride % 16 != 0 ||
                    scales_batch_stride < (blocks_of(m) - 1) * scales_row_stride + blocks_of(k) ||
                    (turned && (out_t_batch_stride < (k - 1) * out_t_row_stride + m ||
                                out_t_batch_stride % 16 != 0))))
    return HADACORE_ERROR_INVALID_STRIDE;
  if (m == 0 || k == 0 || batch == 0) return HADACORE_SUCCESS;
  if (in == nullptr || out_codes == nullptr || out_scales == nullptr)
    return HADACORE_ERROR_INVALID_VALUE;
  if (!aligned_to(in, 2) || !aligned_to(out_codes, 16) || !aligned_to(out_codes_t, 16) ||
      !aligned_to(out_scales, 4))
    return HADACORE_ERROR_MISALIGNED;
  if (in_row_stride > kMaxBytes / m || out_row_stride > kMaxBytes / m ||
      (turned && out_t_row_stride > kMaxBytes / k) ||
      (batch > 1 && (in_batch_stride > kMaxBytes / batch || out_batch_stride > kMaxBytes / batch ||
                     scales_batch_stride > kMaxBytes / batch ||
                     (turned && out_t_batch_stride > kMaxBytes / batch))))
    return HADACORE_ERROR_TOO_LARGE;
  const Span si = batch_span(in, batch, in_batch_stride, m, in_row_stride, k, 2),
             sc = batch_span(out_codes, batch, out_batch_stride, m, out_row_stride, k, 1),
             st = batch_span(out_codes_t, turned ? batch : 0, out_t_batch_stride, turned ? k : 0,
                             out_t_row_stride, m, 1),
             ss = batch_span(out_scales, batch, scales_batch_stride, blocks_of(m),
                             scales_row_stride, blocks_of(k), 4);
  if (spans_overlap(si, sc) || spans_overlap(si, ss) || spans_overlap(sc, ss) ||
      (turned && (spans_overlap(si, st) || spans_overlap(sc, st) || spans_overlap(ss, st))))
    return HADACORE_ERROR_OVERLAP;
  TileArgs p{};
  p.in = static_cast<const uint16_t *>(in);
  p.in_stride = in_row_stride;
  p.in_batch = in_batch_stride;
  p.codes = static_cast<uint8_t *>(out_codes);
  p.codes_stride = out_row_stride;
  p.codes_batch = out_batch_stride;
  p.codes_t = static_cast<uint8_t *>(out_codes_t);
  p.codes_t_stride = out_t_row_stride;
  p.codes_t_batch = out_t_batch_stride;
  p.scales = out_scales;
  p.scales_stride = scales_row_stride;
  p.scales_batch = scales_batch_stride;
  p.m = (int)m;
  p.k = (int)k;
  return run_tiles(p, false, blocks_of(m), batch, dtype, stream);
}

extern "C" hadacore_status hadacore_matmul_fp8(
    const void *a, int64_t a_row_stride, const float *a_scales, int64_t a_scales_row_stride,
    const void *b, int64_t b_row_stride, const float *b_scales, int64_t b_scales_row_stride,
    int32_t b_scale_rows, void *out, int64_t out_row_stride, hadacore_dtype out_dtype, int64_t m,
    int64_t n, int64_t k, void *stream) {
  if (m < 0 || n < 0 || k < 0 || (b_scale_rows != 1 && b_scale_rows != kBlock))
    return HADACORE_ERROR_INVALID_VALUE;
  if (m >= kMaxDim || n >= kMaxDim || k >= kMaxDim) return HADACORE_ERROR_TOO_LARGE;
  ProductArgs p{};
  p.a = static_cast<const uint8_t *>(a);
  p.a_pitch = a_row_stride;
  p.sa = a_scales;
  p.sa_pitch = a_scales_row_stride;
  p.b = static_cast<const uint8_t *>(b);
  p.b_pitch = b_row_stride;
  p.sb = b_scales;
  p.sb_pitch = b_scales_row_stride;
  p.out = out;
  p.out_pitch = out_row_stride;
  p.m = (int)m;
  p.n = (int)n;
  p.k = (int)k;
  p.groups = 1;
  p.kind = kTiles;
  p.out_type = out_dtype;
  const hadacore_status st =
      check_product(p, m, n, k, 1, b_scale_rows == 1 ? n : blocks_of(n));
  if (st != HADACORE_SUCCESS || m == 0 || n == 0) return st;
  return run_product(p, b_scale_rows == 1, stream);
}

extern "C" hadacore_status hadacore_matmul_fp8_grouped(
    const void *a, int64_t a_row_stride, const float *a_scales, int64_t a_scales_row_stride,
    const void *b, int64_t b_row_stride, int64_t b_batch_stride, const float *b_scales,
    int64_t b_scales_row_stride, int64_t b_scales_batch_stride, const int32_t *ends,
    int64_t groups, void *out, int64_t out_row_stride, hadacore_dtype out_dtype, int64_t m,
    int64_t n, int64_t k, void *stream) {
  if (m < 0 || n < 0 || k < 0 || groups < 0) return HADACORE_ERROR_INVALID_VALUE;
  if (m >= kMaxDim || n >= kMaxDim || k >= kMaxDim || groups >= kMaxDim)
    return HADACORE_ERROR_TOO_LARGE;
  hadacore_status st = check_ends(ends, groups);
  if (st != HADACORE_SUCCESS) return st;
  ProductArgs p{};
  p.a = static_cast<const uint8_t *>(a);
  p.a_pitch = a_row_stride;
  p.sa = a_scales;
  p.sa_pitch = a_scales_row_stride;
  p.b = static_cast<const uint8_t *>(b);
  p.b_pitch = b_row_stride;
  p.b_batch = b_batch_stride;
  p.sb = b_scales;
  p.sb_pitch = b_scales_row_stride;
  p.sb_batch = b_scales_batch_stride;
  p.ends = ends;
  p.out = out;
  p.out_pitch = out_row_stride;
  p.m = (int)m;
  p.n = (int)n;
  p.k = (int)k;
  p.groups = (int)groups;
  p.kind = kGroups;
  p.out_type = out_dtype;
  st = check_product(p, m, n, k, groups, blocks_of(n));
  if (st != HADACORE_SUCCESS || m == 0 || n == 0) return st;
  return run_product(p, false, stream);
}

extern "C" hadacore_status hadacore_weight_gradient_fp8_grouped(
    const void *a, int64_t a_row_stride, const float *a_scales, int64_t a_scales_row_stride,
    const void *b, int64_t b_row_stride, const float *b_scales, int64_t b_scales_row_stride,
    const int32_t *ends, int64_t groups, void *out, int64_t out_row_stride,
    int64_t out_batch_stride, hadacore_dtype out_dtype, int64_t places, int64_t n, int64_t k,
    void *stream) {
  if (places < 0 || n < 0 || k < 0 || groups < 0 || (ends == nullptr && groups != 1))
    return HADACORE_ERROR_INVALID_VALUE;
  if (places % kBlock != 0) return HADACORE_ERROR_INVALID_SIZE;
  if (places >= kMaxDim || n >= kMaxDim || k >= kMaxDim || groups >= kMaxDim)
    return HADACORE_ERROR_TOO_LARGE;
  if (!aligned_to(ends, 4)) return HADACORE_ERROR_MISALIGNED;
  ProductArgs p{};
  p.a = static_cast<const uint8_t *>(a);
  p.a_pitch = a_row_stride;
  p.sa = a_scales;
  p.sa_pitch = a_scales_row_stride;
  p.b = static_cast<const uint8_t *>(b);
  p.b_pitch = b_row_stride;
  p.sb = b_scales;
  p.sb_pitch = b_scales_row_stride;
  p.ends = ends;
  p.out = out;
  p.out_pitch = out_row_stride;
  p.out_batch = out_batch_stride;
  p.m = (int)n;
  p.n = (int)k;
  p.k = (int)places;
  p.groups = (int)groups;
  p.kind = kGradient;
  p.out_type = out_dtype;
  if (groups > 1 && out_batch_stride < (n - 1) * out_row_stride + k)
    return HADACORE_ERROR_INVALID_STRIDE;
  const hadacore_status st = check_product(p, n, k, places, groups, k);
  if (st != HADACORE_SUCCESS || n == 0 || k == 0 || groups == 0) return st;
  return run_product(p, true, stream);
}
