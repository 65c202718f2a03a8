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
//     of bf16's.  (The older MFMA 16x16x32 for FP8 measures the same.)  At most a sum is
//     128 * 2^-16 = 2^-9 of that largest product off, which shows where large products cancel.
//   - 32-bit outputs: the codes widened to bf16, exactly, and four MFMA 16x16x32 for bf16,
//     which add in full fp32 (1e-8 for 128 products) at half the rate.

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

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

// Sum over the lanes up to this one, of the whole wave (row shifts, then row broadcasts).
__device__ __forceinline__ int prefix_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);  // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);  // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);  // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);  // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // row_bcast:31
  return x;
}

// Piece `id` of the groups cut into pieces of `unit` rows: group 0's first, then group
// 1's, ...  With `rest` the rows after the last end are one more group.  Called by
// whole waves; 64 groups at a time by a prefix sum over the lanes.
__device__ __forceinline__ Piece find_piece(const int32_t *ends, int groups, int rows, int unit,
                                            int id, bool rest) {
  const int lane = threadIdx.x & (kWave - 1);
  int base = 0, start = 0;  // pieces and rows before these 64 groups
  const int all = groups + (rest ? 1 : 0);
  for (int g0 = 0; g0 < all; g0 += kWave) {
    const int g = g0 + lane;
    const int high = g < groups ? clamp_end(ends[g], rows) : rows;
    // wave_shr:1, the first lane's from the groups before
    const int low = __builtin_amdgcn_update_dpp(start, high, 0x138, 0xF, 0xF, false);
    const int pieces = g < all && high > low ? (high - low + unit - 1) / unit : 0;
    const int sum = prefix_sum(pieces);
    const uint64_t hit = __ballot(pieces > 0 && id >= base + sum - pieces && id < base + sum);
    if (hit != 0) {
      const int at = __builtin_ctzll(hit);
      const int first = base + __builtin_amdgcn_readlane(sum - pieces, at);
      const int lo = __builtin_amdgcn_readlane(low, at);
      return {g0 + at, lo + (id - first) * unit, __builtin_amdgcn_readlane(high, at)};
    }
    base += __builtin_amdgcn_readlane(sum, kWave - 1);
    start = __builtin_amdgcn_readlane(high, kWave - 1);
  }
  return {-1, 0, 0};
}

// How many pieces there are.
__device__ __forceinline__ int count_pieces(const int32_t *ends, int groups, int rows, int unit,
                                            bool rest) {
  const int lane = threadIdx.x & (kWave - 1);
  int count = 0, start = 0;
  const int all = groups + (rest ? 1 : 0);
  for (int g0 = 0; g0 < all; g0 += kWave) {
    const int g = g0 + lane;
    const int high = g < groups ? clamp_end(ends[g], rows) : rows;
    const int low = __builtin_amdgcn_update_dpp(start, high, 0x138, 0xF, 0xF, false);
    const int pieces = g < all && high > low ? (high - low + unit - 1) / unit : 0;
    count += __builtin_amdgcn_readlane(prefix_sum(pieces), kWave - 1);
    start = __builtin_amdgcn_readlane(high, kWave - 1);
  }
  return count;
}

// The blocks of 128 rows before group `group`, and in it, with every group padded to whole
// blocks.  Called by whole waves.
__device__ __forceinline__ void group_blocks(const int32_t *ends, int groups, int rows, int group,
                                             int &before, int &count) {
  const int lane = threadIdx.x & (kWave - 1);
  int base = 0, start = 0;  // blocks and rows before these 64 groups
  for (int g0 = 0; g0 < groups; g0 += kWave) {
    const int g = g0 + lane;
    const int high = g < groups ? clamp_end(ends[g], rows) : rows;
    const int low = __builtin_amdgcn_update_dpp(start, high, 0x138, 0xF, 0xF, false);
    const int blocks = g < groups && high > low ? (high - low + kBlock - 1) / kBlock : 0;
    const int sum = prefix_sum(blocks);
    if (group < g0 + kWave) {
      before = base + __builtin_amdgcn_readlane(sum - blocks, group - g0);
      count = __builtin_amdgcn_readlane(blocks, group - g0);
      return;
    }
    base += __builtin_amdgcn_readlane(sum, kWave - 1);
    start = __builtin_amdgcn_readlane(high, kWave - 1);
  }
  before = base;
  count = 0;
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

// 8 values of a row, widened.
template <int DT>
__device__ __forceinline__ void widen8(u4 raw, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = widen<DT>(raw[j] & 0xFFFFu);
    v[2 * j + 1] = widen<DT>(raw[j] >> 16);
  }
}

// Cache policy of a quantizer by its size.  Which one is fastest depends on whether the input
// lies in the last-level cache (256 MB), which a call cannot know; us, plain / kStreamOut /
// kStreamIn, on inputs in the cache and not:
//   columns of 2048 x 4096        8.1 /  7.4 /  7.3     7.9 /  7.2 /  7.1
//              8320 x 4096       22.4 / 22.3 / 24.9    21.2 / 23.4 / 21.8
//             16384 x 4096       36.7 / 36.6 / 40.3    44.0 / 43.3 / 38.1
//   tiles of   2048 x 4096        9.4 /  7.6 /  8.7     9.2 /  8.4 /  8.6   (both orders)
//              8320 x 4096       26.2 / 26.8 / 27.7    25.4 / 28.0 / 24.9
//          4 x 4096 x 4096       45.3 / 45.2 / 46.5    48.7 / 50.1 / 43.0
//   rows of    2048 x 4096        7.0 /  6.5 /  7.0     7.1 /  7.0 /  6.7   (not rotated)
//              8320 x 4096       23.2 / 22.7 / 21.0    19.7 / 19.8 / 19.1
//             16384 x 4096       37.1 / 37.6 / 39.0    37.2 / 36.2 / 35.4
// From 2^22 elements codes of whole lines are stored with SC1 | NT, which an input in the
// cache gains from.  Inputs of more than 64 MiB (2^25 elements) are taken not to be there:
// they are streamed in, with SC1 stores, which gains up to a seventh if so and costs up to an
// eighth if not.  Below 2^22 the three are alike, and the next product reads the codes from the
// L2: plain.  So are codes that are not whole lines (8192 rows of 8191: 40 us, streamed 60),
// and rows off 16 bytes, whose loads share lines, are not streamed in.
constexpr int kPlain = 0, kStreamOut = 1, kStreamIn = 2;

int quantizer_policy(int64_t elements, const void *in, int64_t in_stride, const void *codes,
                     int64_t pitch, int64_t width) {
  if (elements < (1 << 22) || (reinterpret_cast<uintptr_t>(codes) & 127) != 0 ||
      (pitch | width) % 128 != 0)
    return kPlain;
  const bool aligned = (reinterpret_cast<uintptr_t>(in) & 15) == 0 && in_stride % 8 == 0;
  return elements > (1 << 25) && aligned ? kStreamIn : kStreamOut;
}

// 8 values from `p` on.  Rows may start at any 2-byte address; the hardware takes 16-byte
// loads from there.
template <int POLICY>
__device__ __forceinline__ u4 load8(const uint16_t *p) {
  typedef u4 u4_any __attribute__((aligned(2)));
  if constexpr (POLICY == kStreamIn) {
    return __builtin_nontemporal_load(reinterpret_cast<const u4_any *>(p));
  } else {
    return *reinterpret_cast<const u4_any *>(p);
  }
}

// The first `valid` < 8 of them, and zeros.
__device__ __forceinline__ u4 load_some(const uint16_t *p, int valid) {
  u4 raw = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 7; ++j)
    if (j < valid) raw[j / 2] |= (uint32_t)p[j] << (16 * (j % 2));
  return raw;
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

template <int POLICY>
__device__ __forceinline__ void store_codes8(uint8_t *p, u2 c, int valid) {
  if (valid >= 8) {
    if constexpr (POLICY == kStreamIn)
      asm volatile("global_store_dwordx2 %0, %1, off sc1" ::"v"(p), "v"(c) : "memory");
    else if constexpr (POLICY == kStreamOut)
      asm volatile("global_store_dwordx2 %0, %1, off sc1 nt" ::"v"(p), "v"(c) : "memory");
    else
      *reinterpret_cast<u2 *>(p) = c;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < valid) p[j] = (uint8_t)(c[j / 4] >> (8 * (j % 4)));
  }
}

// The value of lane ^ BIT, by permutations inside rows of 16 lanes (xor 4: row_half_mirror,
// which is xor 7, and quad_perm xor 3).
template <int BIT>
__device__ __forceinline__ float lane_xor(float v) {
  const auto dpp = [](int x, auto ctrl) {
    return __builtin_amdgcn_mov_dpp(x, decltype(ctrl)::value, 0xF, 0xF, true);
  };
  const int x = __builtin_bit_cast(int, v);
  if constexpr (BIT == 1)
    return __builtin_bit_cast(float, dpp(x, std::integral_constant<int, 0xB1>{}));
  else if constexpr (BIT == 2)
    return __builtin_bit_cast(float, dpp(x, std::integral_constant<int, 0x4E>{}));
  else
    return __builtin_bit_cast(float, dpp(dpp(x, std::integral_constant<int, 0x141>{}),
                                         std::integral_constant<int, 0x1B>{}));
}

// Maximum over 16 lanes: xor 1 and 2, then the mirrors of 8 and 16 lanes, whose halves
// hold one value each by then.
__device__ __forceinline__ float max16(float a) {
  a = fmaxf(a, lane_xor<1>(a));
  a = fmaxf(a, lane_xor<2>(a));
  a = fmaxf(a, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, a), 0x141,
                                                                  0xF, 0xF, true)));
  return fmaxf(a, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, a),
                                                                     0x140, 0xF, 0xF, true)));
}

template <int BIT>
__device__ __forceinline__ void lane_butterflies(float (&v)[8], int lane) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float other = lane_xor<BIT>(v[j]);
    v[j] = (lane & BIT) != 0 ? other - v[j] : v[j] + other;
  }
}

// Blocks of a group of lanes: 8192 rows of 8192 take 34.2 us with two (5.9 TB/s), 40.2
// with one, 34.9 with four.
constexpr int kTurns = 2;

// Rows rotated by 2^L <= 64 values: 16 lanes hold a block of 128, 8 consecutive values
// each, so the stages on index bits 0-2 are in registers and those on bits 3-5 between
// lanes.  HBM-bound; a group of lanes takes kTurns blocks, whose loads go out together.
// 8192 bf16 rows of 8192 without rotation: 34 us, 5.9 TB/s.
template <int DT, int L, int POLICY>
__global__ __launch_bounds__(256) void short_rotation_kernel(
    const uint16_t *in, int64_t in_stride, uint8_t *codes, int64_t codes_stride, float *scales,
    int64_t scales_stride, int64_t m, int k, int blocks, float scale) {
  const int sub = threadIdx.x & 15;
  const int64_t total = m * blocks, step = (int64_t)gridDim.x * 16 * kTurns;
  // every lane of a wave takes part in the exchanges, so the bound is the workgroup's; the
  // division is in 32 bits where it can be
  for (int64_t i0 = (int64_t)blockIdx.x * 16 * kTurns; i0 < total; i0 += step) {
    u4 raw[kTurns];
    int64_t row[kTurns];
    int block[kTurns], valid[kTurns];
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
      const int64_t i = i0 + u * 16 + (threadIdx.x >> 4);
      row[u] = i >= total         ? 0
               : total >> 32 == 0 ? (int64_t)((uint32_t)i / (uint32_t)blocks)
                                  : i / blocks;
      block[u] = i < total ? (int)(i - row[u] * blocks) : 0;
      valid[u] = i < total ? k - block[u] * kBlock - sub * 8 : 0;
    }
    bool some = false;
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
      some |= valid[u] < 8;
      const uint16_t *from = in + row[u] * in_stride;
      raw[u] = u4{0, 0, 0, 0};
      if (valid[u] >= 8) raw[u] = load8<POLICY>(from + block[u] * kBlock + sub * 8);
    }
    if (some) {
#pragma unroll
      for (int u = 0; u < kTurns; ++u)
        if (valid[u] < 8)
          raw[u] = load_some(in + row[u] * in_stride + block[u] * kBlock + sub * 8, valid[u]);
    }
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
      float v[8];
      widen8<DT>(raw[u], v);
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
      if constexpr (L > 3) lane_butterflies<1>(v, sub);
      if constexpr (L > 4) lane_butterflies<2>(v, sub);
      if constexpr (L > 5) lane_butterflies<4>(v, sub);
      const float a = max16(abs_max(v));
      if (valid[u] > 0) {
        store_codes8<POLICY>(codes + row[u] * codes_stride + block[u] * kBlock + sub * 8,
                             codes8(v, inverse_scale(a)), valid[u]);
        if (sub == 0) scales[row[u] * scales_stride + block[u]] = a / 448.0f;
      }
    }
  }
}

template <int DT>
hipError_t short_rotations(const uint16_t *in, int64_t in_stride, uint8_t *codes,
                           int64_t codes_stride, float *scales, int64_t scales_stride, int64_t m,
                           int k, int L, float scale, hipStream_t stream) {
  const int blocks = (k + kBlock - 1) / kBlock;
  const int64_t groups = (m * blocks + 16 * kTurns - 1) / (16 * kTurns);
  const dim3 grid((uint32_t)(groups < (1 << 20) ? groups : (1 << 20)));
  const auto with = [&](auto l, auto policy) {
    hipLaunchKernelGGL((short_rotation_kernel<DT, decltype(l)::value, decltype(policy)::value>), grid,
                       dim3(256), 0, stream, in, in_stride, codes, codes_stride, scales,
                       scales_stride, m, k, blocks, scale);
    return hipGetLastError();
  };
  const int policy = quantizer_policy(m * k, in, in_stride, codes, codes_stride, k);
  const auto go = [&](auto l) {
    return policy == kStreamIn    ? with(l, std::integral_constant<int, kStreamIn>{})
           : policy == kStreamOut ? with(l, std::integral_constant<int, kStreamOut>{})
                                  : with(l, std::integral_constant<int, kPlain>{});
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
// as whole 128-byte lines.  HBM-bound: 8 bf16 weights of 2048 x 4096 to both orders 42 us,
// 6.4 TB/s; 8191 rows of 4096 in 8 groups to columns 18.6 us, 5.7 TB/s.  All of a thread's
// loads go out before anything uses one; before they did, 52 and 26 us.
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

template <int DT, bool COLUMNS, int POLICY>
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
    if (p.ends != nullptr || p.groups == 0) {
      const Piece piece = find_piece(p.ends, p.groups, p.m, kBlock, out_block, false);
      row0 = piece.low;
      row_end = piece.group < 0 ? 0 : piece.high;
    }
  }
  const uint16_t *in = p.in + blockIdx.z * p.in_batch;
  const int col = col0 + cg * 8;
  float v[8][8];
  const int rows = row_end - row0;  // <= 0: a block past the last group, all zero
  {
    // all loads before the first use; rows past the end repeat the last one, as zeros
    u4 raw[8];
    if (p.k - col >= 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = rg * 8 + i, last = rows > 0 ? rows - 1 : 0;
        raw[i] = load8<POLICY>(in + (int64_t)(row0 + (r < last ? r : last)) * p.in_stride + col);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        raw[i] = rg * 8 + i < rows
                     ? load_some(in + (int64_t)(row0 + rg * 8 + i) * p.in_stride + col, p.k - col)
                     : u4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (rg * 8 + i >= rows) raw[i] = u4{0, 0, 0, 0};
      widen8<DT>(raw[i], v[i]);
    }
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
    if (t < kBlock) {
      const float a = fmaxf(fmaxf(maxima[0][t], maxima[1][t]), fmaxf(maxima[2][t], maxima[3][t]));
      maxima[0][t] = inverse_scale(a);
      if (col0 + t < p.k)
        p.scales[(int64_t)(col0 + t) * p.scales_stride + out_block] = a / 448.0f;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) mul[j] = maxima[0][cg * 8 + j];
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
        store_codes8<POLICY>(p.codes + blockIdx.z * p.codes_batch + (int64_t)(row0 + r) * p.codes_stride +
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
      store_codes8<POLICY>(out + (int64_t)(col0 + c) * p.codes_t_stride + cg * 8,
                   turned[c * 16 + (cg ^ (c >> 3))], left - cg * 8);
  }
}

// ---- products ------------------------------------------------------------------

constexpr int kDense = 0;     // all rows of A with one B
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
  int tiles_m, tiles_n;  // the tiles (kGradient: of each group; kGroups: at most)
  uint32_t tiles;        // in all
  bool nt_out;           // outputs with the streaming cache policy
  int kind, out_type;
};

// Asynchronous loads into LDS: lane l's 16 bytes from base + offset + uniform_offset go to
// `lds` + 16 l.  In asm, because the compiler waits for all outstanding loads of this kind
// before any LDS read, which would undo the loading ahead: the kernel waits itself
// (wait_stages) before the barrier that publishes the data.  The instruction writes no
// register; the wait state is the one that it needs after a write of M0 (which no other
// instruction of these kernels uses, and which may not be named as clobbered).
// NT: with the streaming cache policy, for data that nobody reads again.
template <bool NT = false>
__device__ __forceinline__ void load_to_lds(u4 base, uint32_t lds, int offset, int uniform_offset) {
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds"
                 :
                 : "s"(lds), "v"(offset), "s"(base), "s"(uniform_offset)
                 : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(lds), "v"(offset), "s"(base), "s"(uniform_offset)
                 : "memory");
}

// The same for one 4-byte word of each lane's own address.
__device__ __forceinline__ void load_word_to_lds(const float *from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :
               : "s"(lds), "v"(from)
               : "memory");
}

// Waits until at most the loads of `ahead` later stages of `LOADS` loads are in flight,
// `ahead` being at most MOST.
template <int MOST, int LOADS>
__device__ __forceinline__ void wait_stages(int ahead) {
  if constexpr (MOST > 0) {
    if (ahead < MOST) {
      wait_stages<MOST - 1, LOADS>(ahead);
      return;
    }
  }
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(MOST * LOADS) : "memory");
}

__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

// A buffer over everything from `base`, which is the same in every lane: the range check
// is off, the rows that a kernel reads are clamped instead.
__device__ __forceinline__ u4 buffer_words(const void *base) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  return u4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b),
            (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) & 0xFFFFu, 0xFFFFFFFFu,
            0x00020000u};
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

// 16 bytes of consecutive outputs of a row, of which the first `valid` exist, in one store
// (rows may start at any value's address; the hardware takes 16-byte stores there) or, at the
// end of a row, value by value.  `nt`: with the streaming cache policy.
template <int OUT, int N>
__device__ __forceinline__ void store_row(void *out, int64_t at, const float (&v)[N], int valid,
                                          bool nt) {
  typedef u4 u4_any __attribute__((aligned(2)));
  if (valid >= N) {
    u4 bits;
    if constexpr (OUT == HADACORE_FP32)
      bits = __builtin_bit_cast(u4, f4{v[0], v[1], v[2], v[3]});
    else
      bits = u4{pack2<OUT>(v[0], v[1]), pack2<OUT>(v[2], v[3]), pack2<OUT>(v[4], v[5]),
                pack2<OUT>(v[6], v[7])};
    char *to = static_cast<char *>(out) + at * (OUT == HADACORE_FP32 ? 4 : 2);
    // In asm, since the compiler would make one ordinary store of the two branches; with the
    // wait state that a store of more than 8 bytes needs before its data may be overwritten,
    // which the compiler does not see to here.
    if (nt)
      asm volatile("global_store_dwordx4 %0, %1, off sc1 nt\n\ts_nop 1" ::"v"(to), "v"(bits)
                   : "memory");
    else
      *reinterpret_cast<u4_any *>(to) = bits;
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
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
  __device__ __forceinline__ static f4 part(int s, const Operand &x, const Operand &y, f4 r) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.values[s], y.values[s], r, 0, 0, 0);
  }
  __device__ __forceinline__ static f4 product(const Operand &x, const Operand &y) {
    f4 r = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < 4; ++s) r = part(s, x, y, r);
    return r;
  }
};

// Which tile a workgroup takes.  Workgroups go to the 8 XCDs in turn, each with an L2 of
// its own: of 256 that run together (one to a CU), each XCD takes 32 consecutive tiles, and
// tiles are numbered in bands of kBand rows, down the band first, so that 32 tiles read
// 4 strips of A and 8 of B.  (On a part of a card the numbering is as complete, only the strips
// are shared less.)
struct TileAt {
  int matrix, m, n;
};

__device__ __forceinline__ TileAt tile_at(uint32_t id, uint32_t total, int tiles_m, int tiles_n) {
  constexpr uint32_t kXcds = 8, kTogether = 256;
  constexpr int kBand = 4;
  const uint32_t first = id & ~(kTogether - 1);
  const uint32_t count = total - first < kTogether ? total - first : kTogether;
  const uint32_t xcd = id & (kXcds - 1), turn = (id - first) / kXcds;
  const uint32_t each = count / kXcds, more = count % kXcds;
  const uint32_t tile = first + xcd * each + (xcd < more ? xcd : more) + turn;
  const uint32_t per = (uint32_t)tiles_m * (uint32_t)tiles_n;
  const int matrix = (int)(tile / per), rest = (int)(tile % per);
  const int band = rest / (kBand * tiles_n), in_band = rest % (kBand * tiles_n);
  const int high = tiles_m - band * kBand < kBand ? tiles_m - band * kBand : kBand;
  return {matrix, band * kBand + in_band % high, in_band / high};
}

// Which of 32 columns row i of the j-th of two MFMAs is (a lane holds rows 4 g .. 4 g + 3).
template <bool FULL>
__device__ __forceinline__ int tile_column(int j, int i) {
  return FULL ? 16 * j + i : 8 * (i >> 2) + 4 * j + (i & 3);
}

// The whole tiles' kernel: BM x BN outputs by WM x WN waves, in steps of a block of k.
//
// The rows of A and B and their scales go through D stages of LDS, loaded D - 1 steps
// ahead; one barrier a step.  All loads are of the kind that goes to LDS, the same number
// in every wave, so that a wait counts stages.
//
// B is the MFMA's first operand and A its second, so a lane's four results are four
// columns n of one row m: its A scale is one value, and its stores are along the row.
// Lane l of an MFMA holds 32 bytes of row l & 15 of either operand: the 16-byte chunks
// g and g + 4, g = l >> 4, of the 128 (any order of k will do that both share).  The rows
// of B are laid out in LDS so that a lane's results make 16-byte stores and the stores of
// its four lane groups 64 bytes of a row: in 32 bits the j-th MFMA's rows are its columns,
// in 16 bits two MFMAs' results are joined (tile_column).
//
// LDS rows are 128 bytes; chunk c of row r lies at c ^ ((r >> 1) & 7), which the loads
// obey by choosing their global chunk, since LDS addresses of a load run with the lane.
//
// Both operands go through LDS: a step of 256 x 256 reads 1536 cycles of it and writes 512,
// as many as its MFMAs take, so the two bound it together, at the clock that the card's
// power leaves (1.83 GHz of 2.4).  Loading B to registers in the MFMA's order touches 64
// lines an instruction and was 3 times slower, weights laid out for it beforehand reached
// 2.14 PFLOP/s, MFMAs of 32 x 32 x 64 spilled (2.2).  Measured: 16384 x 4096 x 4096 with tile
// scales to bf16 230 us, 2.39 PFLOP/s; 4001 tokens' gradient of 4096 x 4096, scales of both
// rows, 73 us, 1.85 PFLOP/s (a scale of B costs 8 VALU operations a product more); to 32
// bits, 8 gradients of 2048 x 4096 from 8191 tokens, 179-197 us, 0.70-0.77 PFLOP/s (half the MFMA rate,
// the widening, and a 256 MiB store).
// A tile's rows and columns, where its outputs start, and its blocks of k.
struct Tile {
  int m0, n0, m_end, kb0, kb1;
  int64_t out_at;
  const uint8_t *b;
  const float *sb;
};

// The tiles of a workgroup: first + blockIdx.x, + gridDim.x, ... below `end`, of `total`
// tiles of bm x bn; or, with `parts`, the quarters of the tiles from `first` on, the first
// quarters of all before the second ones.
struct Tiles {
  int bm, bn, tiles_m;
  uint32_t total, first, end, parts, id;

  __device__ __forceinline__ bool next(const ProductArgs &p, Tile &to) {
    for (; id < end; id += gridDim.x) {
      const uint32_t part = parts ? id / parts : 0;
      const TileAt at = tile_at(first + (parts ? id % parts : id), total, tiles_m, p.tiles_n);
      to = {at.m * bm, at.n * bn, p.m, 0, (p.k + kBlock - 1) / kBlock, 0, p.b, p.sb};
      if (p.kind == kGroups) {
        const Piece piece = find_piece(p.ends, p.groups, p.m, bm, at.m, true);
        to.m0 = piece.low;
        to.m_end = piece.high;
        if (piece.group < 0 || to.m0 < 0) continue;
        if (piece.group == p.groups) {
          to.kb1 = 0;  // rows after the last group: zeros
        } else {
          to.b += piece.group * p.b_batch;
          to.sb += piece.group * p.sb_batch;
        }
      } else if (p.kind == kGradient) {
        to.out_at = at.matrix * p.out_batch;
        if (p.ends != nullptr) {
          int before, count;
          group_blocks(p.ends, p.groups, p.k, at.matrix, before, count);
          to.kb0 = before < to.kb1 ? before : to.kb1;
          to.kb1 = before + count < to.kb1 ? before + count : to.kb1;
        }
      }
      to.m0 += (int)(part >> 1) * (bm / 2);
      to.n0 += (int)(part & 1) * (bn / 2);
      if (to.m0 >= to.m_end || to.n0 >= p.n) continue;
      id += gridDim.x;
      return true;
    }
    return false;
  }
};

template <int BM, int BN, int WM, int WN, int D, int KS, bool BROWS>
struct Shape {
  static constexpr int kThreads = WM * WN * kWave;  // of one share of k
  // scales of A's rows, then of B's columns or blocks of columns
  static constexpr int SB = BROWS ? BN : BN / kBlock > 0 ? BN / kBlock : 1;
  static constexpr int kScales = (BM + SB + kThreads - 1) / kThreads;
  static constexpr int kStageBytes = (BM + BN) * kBlock;
  static constexpr int kTileBytes = KS * D * kStageBytes, kScaleFloats = KS * D * kScales * kThreads;
};

// Sums the tiles of `which`, through `tiles` and `scale_memory` of LDS.
template <int BM, int BN, int WM, int WN, int D, int KS, bool LOOP, bool BROWS, bool FULL>
__device__ __forceinline__ void sum_tiles(const ProductArgs &p, uint8_t *tiles, float *scale_memory,
                                          Tiles which) {
  using S = Shape<BM, BN, WM, WN, D, KS, BROWS>;
  constexpr int kThreads = S::kThreads, kScales = S::kScales;
  constexpr int TM = BM / WM / 16, TN = BN / WN / 16;  // MFMA tiles of a wave
  static_assert(TN % 2 == 0 && kBlock % (BN / WN) == 0, "a wave's columns are in one block of B");
  constexpr int kLoadsA = BM * 8 / kThreads, kLoadsB = BN * 8 / kThreads;
  constexpr int kTiles = kLoadsA + kLoadsB;  // loads of 16 bytes a thread
  constexpr int kLoads = kTiles + kScales;
  static_assert(kLoads * (D - 2) < 64, "loads in flight that one wait can count");
  constexpr int kStageBytes = S::kStageBytes;
  static_assert(!LOOP || (D == 2 && KS == 1), "a loop over tiles loads one block ahead");

  const int share = KS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
  const int t = threadIdx.x - share * kThreads, lane = t & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(t / kWave);
  const int wm = wave / WN, wn = wave % WN;
  uint8_t *const ring = tiles + share * D * kStageBytes;
  float (*const scales)[kScales * kThreads] =
      reinterpret_cast<float (*)[kScales * kThreads]>(scale_memory + share * D * kScales * kThreads);
  const int g = lane >> 4, li = lane & 15;

  const int tail = p.k & (kBlock - 1), kb_tail = tail != 0 ? p.k / kBlock : -1;

  // The next tile that has something to sum, into `tile`; those that have not get zeros.
  Tile tile;
  const auto take = [&] {
    while (which.next(p, tile)) {
      if (tile.kb0 < tile.kb1) return true;
      for (int e = threadIdx.x; e < BM * BN; e += KS * kThreads) {
        const int row = tile.m0 + e / BN, column = tile.n0 + e % BN;
        const int64_t to = tile.out_at + (int64_t)row * p.out_pitch + column;
        if (row < tile.m_end && column < p.n) {
          if constexpr (FULL)
            static_cast<float *>(p.out)[to] = 0.0f;
          else
            static_cast<uint16_t *>(p.out)[to] = 0;
        }
      }
    }
    return false;
  };

  // Where the loads of `tile` come from.
  u4 ra, rb;
  int off[kTiles];
  const float *scale_at[kScales];
  const auto aim = [&] {
    // the rows past the end repeat the last one; their results are not stored
    const int rows = tile.m_end - tile.m0, columns = p.n - tile.n0;
    ra = buffer_words(p.a + (int64_t)tile.m0 * p.a_pitch);
    rb = buffer_words(tile.b + (int64_t)tile.n0 * p.b_pitch);
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const int s = (i < kLoadsA ? i : i - kLoadsA) * kThreads + t, r = s >> 3;
      const int c = (r & ~31) + tile_column<FULL>((r >> 4) & 1, r & 15);
      const int row = i < kLoadsA ? (r < rows ? r : rows - 1) : (c < columns ? c : columns - 1);
      off[i] = row * (int)(i < kLoadsA ? p.a_pitch : p.b_pitch) + (((s & 7) ^ ((s >> 4) & 7)) << 4);
    }
    // the threads past the scales bring the last one again
#pragma unroll
    for (int i = 0; i < kScales; ++i) {
      const int r = i * kThreads + t, last = BROWS ? p.n - 1 : (p.n - 1) / kBlock;
      const int c = (BROWS ? tile.n0 : tile.n0 / kBlock) + r - BM;
      scale_at[i] = r < BM ? p.sa + (int64_t)(tile.m0 + (r < rows ? r : rows - 1)) * p.sa_pitch
                           : tile.sb + (int64_t)(c < last ? c : last) * p.sb_pitch;
    }
  };

  // One of a thread's kLoads loads of block kb.  In the last, partial block (TAIL) chunks
  // wholly past k may lie past the matrix: the row's first one is loaded instead, so the
  // block's offset is the lane's there.
  const auto load_piece = [&](int kb, int stage, int i, auto is_tail) {
    if (i >= kTiles) {
      load_word_to_lds(scale_at[i - kTiles] + kb,
                       lds_address(&scales[stage][(i - kTiles) * kThreads + wave * kWave]));
      return;
    }
    int from = off[i], at = kb * kBlock;
    if constexpr (decltype(is_tail)::value) {
      const int s = (i < kLoadsA ? i : i - kLoadsA) * kThreads + t;
      const int c = ((s & 7) ^ ((s >> 4) & 7)) << 4;
      from = c < tail ? from + at : from - c;
      at = 0;
    }
    // A's rows and then B's
    load_to_lds(i < kLoadsA ? ra : rb,
                lds_address(ring + stage * kStageBytes) + (i * kThreads + wave * kWave) * 16, from, at);
  };

  f4 acc[TM][TN];
  const int key = (li >> 1) & 7;
  const int chunk0 = li * kBlock + ((g ^ key) << 4), chunk1 = li * kBlock + (((g + 4) ^ key) << 4);
  const auto fragment = [&](const uint8_t *tile_rows, auto is_tail) {
    u4 lo = *reinterpret_cast<const u4 *>(tile_rows + chunk0);
    u4 hi = *reinterpret_cast<const u4 *>(tile_rows + chunk1);
    if constexpr (decltype(is_tail)::value) {
      lo = first_bytes(lo, tail - g * 16);
      hi = first_bytes(hi, tail - g * 16 - 64);
    }
    return i8v{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3],
               (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };

  using No = std::false_type;
  using Yes = std::true_type;
  // the stores of a whole tile: one of 16 bytes for each kStore results
  constexpr int kStore = FULL ? 4 : 8, kStores = TM * TN * 4 / kStore;
  static_assert(kStores < 64, "stores in flight that one wait can count");
  // One step: the products of the block in `stage`, of which `ahead` more are on their way,
  // and in between the loads of block `load_kb` (LOAD: 0 none, 1 a whole block, 2 the tail)
  // into the stage that the last step has read.  Issuing them all first would hold up the wave, which takes its turn at the
  // address unit, 16 cycles a load; the first half of the step leaves them time to arrive.
  // `storing`: kStores stores went out after this block's loads, and need not have ended.
  const auto step = [&](int stage, int ahead, int load_kb, auto what, auto is_tail,
                        bool storing = false) {
    constexpr int LOAD = decltype(what)::value;
    // this block has come; the barrier also ends the last step's reads
    if (LOOP && storing)
      wait_stages<1, kStores>(1);
    else
      wait_stages<D - 2, kLoads>(ahead);
    __syncthreads();
    const uint8_t *la = ring + stage * kStageBytes + wm * (BM / WM) * kBlock;
    const uint8_t *lb = ring + stage * kStageBytes + (BM + wn * (BN / WN)) * kBlock;
    const int into = stage == 0 ? D - 1 : stage - 1;
    f4 col[TN];
    float uniform_b = 0.0f, s[TM];
    const auto load_scales = [&] {
      if constexpr (BROWS) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
          col[j] = *reinterpret_cast<const f4 *>(
              &scales[stage][BM + wn * (BN / WN) + (j & ~1) * 16 + tile_column<FULL>(j & 1, 4 * g)]);
      } else {
        uniform_b = scales[stage][BM + wn * (BN / WN) / kBlock];
      }
#pragma unroll
      for (int i = 0; i < TM; ++i) s[i] = scales[stage][wm * (BM / WM) + i * 16 + li];
    };
    const auto scale = [&](int i, int j, const f4 &r) {
      if (!BROWS && j == 0) s[i] *= uniform_b;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        acc[i][j][q] = __builtin_fmaf(r[q], BROWS ? s[i] * col[j][q] : s[i], acc[i][j][q]);
      // keeps the sums here: the compiler would move them past the next barrier
      asm volatile("" : "+v"(acc[i][j]));
    };
    // spreads the loads over the first half of TM * TN products
    const auto load_slot = [&](int c) {
      if constexpr (LOAD != 0) {
        constexpr int kOver = TM * TN / 2;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
          if (i * kOver / kLoads == c)
            load_piece(load_kb, into, i, std::bool_constant<LOAD == 2>{});
      }
    };
    // Scaling a product waits for its MFMA, so it is done later, between the next ones, and
    // the operand of the next row of products is read during this one's.  The barriers of
    // the scheduler keep that order, which the compiler would undo.
    Operand<FULL> fa[2], fb[TN];
    if constexpr (FULL) {
      // a row of products at once, as TN chains of four MFMAs that do not wait for each
      // other; the next row's codes are widened when they have come
      i8v raw = fragment(la, is_tail);
      i8v raw_b[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) raw_b[j] = fragment(lb + j * 16 * kBlock, is_tail);
      load_scales();
      fa[0].set(raw);
#pragma unroll
      for (int j = 0; j < TN; ++j) fb[j].set(raw_b[j]);
      f4 r[2][TN];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        if (i + 1 < TM) raw = fragment(la + (i + 1) * 16 * kBlock, is_tail);
#pragma unroll
        for (int part = 0; part < 4; ++part) {
#pragma unroll
          for (int j = 0; j < TN; ++j)
            r[i & 1][j] = Operand<FULL>::part(part, fb[j], fa[i & 1],
                                              part == 0 ? f4{0, 0, 0, 0} : r[i & 1][j]);
#pragma unroll
          for (int j = part * TN / 4; j < (part + 1) * TN / 4; ++j) {
            if (i > 0) scale(i - 1, j, r[(i - 1) & 1][j]);
            load_slot(i * TN + j);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (i + 1 < TM) fa[(i + 1) & 1].set(raw);
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) scale(TM - 1, j, r[(TM - 1) & 1][j]);
    } else {
      constexpr int kAhead = 3;
      f4 r[kAhead + 1];
      fa[0].set(fragment(la, is_tail));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        fb[j].set(fragment(lb + j * 16 * kBlock, is_tail));
        __builtin_amdgcn_sched_barrier(0);
      }
      load_scales();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int c = 0; c < TM * TN + kAhead; ++c) {
        if (c < TM * TN) {
          const int i = c / TN, j = c % TN;
          if (j == 0 && i + 1 < TM)
            fa[(i + 1) & 1].set(fragment(la + (i + 1) * 16 * kBlock, is_tail));
          r[c % (kAhead + 1)] = Operand<FULL>::product(fb[j], fa[i & 1]);
        }
        if (c >= kAhead)
          scale((c - kAhead) / TN, (c - kAhead) % TN, r[(c - kAhead) % (kAhead + 1)]);
        load_slot(c);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  // Whether the tile was whole is returned.
  const auto store = [&](const Tile &of) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int row = of.m0 + wm * (BM / WM) + i * 16 + li;
      if (row >= of.m_end) continue;
#pragma unroll
      for (int j = 0; j < TN; j += kStore / 4) {
        const int column = of.n0 + wn * (BN / WN) + (j & ~1) * 16 + tile_column<FULL>(j & 1, 4 * g);
        float v[kStore];
#pragma unroll
        for (int q = 0; q < kStore; ++q) v[q] = acc[i][j + q / 4][q % 4];
        const int64_t to = of.out_at + (int64_t)row * p.out_pitch + column;
        if constexpr (FULL)
          store_row<HADACORE_FP32>(p.out, to, v, p.n - column, p.nt_out);
        else if (p.out_type == HADACORE_FP16)
          store_row<HADACORE_FP16>(p.out, to, v, p.n - column, p.nt_out);
        else
          store_row<HADACORE_BF16>(p.out, to, v, p.n - column, p.nt_out);
      }
    }
    return of.m_end - of.m0 >= BM && p.n - of.n0 >= BN;
  };
  const auto clear = [&] {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = f4{0, 0, 0, 0};
  };
  const auto load_first = [&](int kb, int stage) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if (kb == kb_tail)
        load_piece(kb, stage, i, Yes{});
      else
        load_piece(kb, stage, i, No{});
    }
  };
  using None = std::integral_constant<int, 0>;
  using Whole = std::integral_constant<int, 1>;
  using Partial = std::integral_constant<int, 2>;
  const auto after = [](int stage) { return stage == D - 1 ? 0 : stage + 1; };

  if (!take()) return;
  aim();
  if constexpr (LOOP) {
    // The workgroup goes through tiles: the last step of one loads the first block of the
    // next, whose loads are under way while this one's results are stored.
    load_first(tile.kb0, 0);
    bool more = true, storing = false;
    for (int stage = 0; more;) {
      const Tile now = tile;
      clear();
      for (int kb = now.kb0; kb < now.kb1; ++kb, stage = after(stage)) {
        int next = kb + 1;
        if (next == now.kb1) {
          more = take();
          if (more) aim();
          // after the last tile its last block once more, which nobody reads
          next = more ? tile.kb0 : kb;
        }
        step(stage, 0, next, Whole{}, No{}, storing);
        storing = false;
      }
      storing = store(now);
    }
    wait_stages<0, 0>(0);
  } else {
    // One tile to a workgroup.  This share of the blocks of k, and the steps that all take:
    const int steps = (tile.kb1 - tile.kb0 + KS - 1) / KS;
    const int kb0 = tile.kb0 + share * steps < tile.kb1 ? tile.kb0 + share * steps : tile.kb1;
    const int kb1 = kb0 + steps < tile.kb1 ? kb0 + steps : tile.kb1;
    clear();
    if (kb0 < kb1) {
#pragma unroll
      for (int d = 0; d < D - 1; ++d)
        if (kb0 + d < kb1) load_first(kb0 + d, d);
      const int whole = kb1 - 1 == kb_tail ? kb1 - 1 : kb1;  // end of the whole blocks
      int kb = kb0, stage = 0;
      for (; kb + D - 1 < whole; ++kb, stage = after(stage))
        step(stage, kb1 - 1 - kb, kb + D - 1, Whole{}, No{});
      if (kb + D - 1 < kb1) {
        step(stage, kb1 - 1 - kb, kb + D - 1, Partial{}, No{});
        ++kb;
        stage = after(stage);
      }
      for (; kb < whole; ++kb, stage = after(stage)) step(stage, kb1 - 1 - kb, 0, None{}, No{});
      if (kb < kb1) step(stage, 0, 0, None{}, Yes{});
    }
    if constexpr (KS > 1) {
      // the other shares' barriers, then the sums of the shares, added in their order
      for (int i = kb1 - kb0; i < steps; ++i) __syncthreads();
      static_assert((KS - 1) * BM * BN * 4 <= S::kTileBytes, "the sums fit the stages");
      f4 *sums = reinterpret_cast<f4 *>(tiles);
      __syncthreads();
      if (share > 0) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j)
            sums[(((share - 1) * TM + i) * TN + j) * kThreads + t] = acc[i][j];
      }
      __syncthreads();
      if (share > 0) return;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int q = 0; q < KS - 1; ++q) acc[i][j] += sums[((q * TM + i) * TN + j) * kThreads + t];
    }
    store(tile);
  }
}

// One tile to a workgroup, or (LOOP) as many workgroups as run together, each going through
// tiles.  SPLIT: the tiles of the last turn, if they would leave half of the workgroups or
// more without one, are cut into quarters: a turn of quarters with k = 4096 takes 21 us
// where one of whole tiles takes 60 (16384 tokens over 16 experts of 2048 x 4096: 180 us
// instead of 189).
template <int BM, int BN, int WM, int WN, int D, int KS, bool LOOP, bool SPLIT, bool BROWS, bool FULL>
__global__ __launch_bounds__(KS *WM *WN *kWave) void product_kernel(ProductArgs p) {
  using S = Shape<BM, BN, WM, WN, D, KS, BROWS>;
  // quarters have twice the stages in the same LDS
  using Q = Shape<BM / 2, BN / 2, WM, WN, 2 * D, KS, BROWS>;
  static_assert(!SPLIT || Q::kTileBytes <= S::kTileBytes, "quarters fit");
  __shared__ __align__(16) uint8_t tiles[S::kTileBytes];
  __shared__ __align__(16) float scales[SPLIT ? Q::kScaleFloats : S::kScaleFloats];
  Tiles which{BM, BN, p.tiles_m, p.tiles, 0, p.tiles, 0, blockIdx.x};
  if constexpr (LOOP && SPLIT) {
    if (p.kind == kGroups) {
      // ragged groups: the tiles that there are, not those that there may be (p.tiles_m), which
      // ends that go down can pass by any number, up to a count that does not fit
      const uint32_t count = (uint32_t)count_pieces(p.ends, p.groups, p.m, BM, true);
      which.tiles_m = count < (uint32_t)p.tiles_m ? (int)count : p.tiles_m;
      which.total = (uint32_t)which.tiles_m * (uint32_t)p.tiles_n;
    }
    const uint32_t rest = which.total % gridDim.x;
    const bool split = rest <= gridDim.x / 2;
    which.end = split ? which.total - rest : which.total;
    sum_tiles<BM, BN, WM, WN, D, KS, LOOP, BROWS, FULL>(p, tiles, scales, which);
    if (!split) return;
    for (uint32_t id = blockIdx.x; id < 4 * rest; id += gridDim.x) {
      __syncthreads();
      sum_tiles<BM / 2, BN / 2, WM, WN, 2 * D, KS, false, BROWS, FULL>(
          p, tiles, scales, Tiles{BM, BN, which.tiles_m, which.total, which.end, id + 1, rest, id});
    }
  } else {
    sum_tiles<BM, BN, WM, WN, D, KS, LOOP, BROWS, FULL>(p, tiles, scales, which);
  }
}

// Few rows of A: the product is a reading of B at HBM speed.  A workgroup takes 16 MT rows
// of A and 16 RB rows of B; its W waves share the blocks of k, each summing its own, and
// add their sums in LDS in the order of the waves.  Every wave streams its blocks through
// D stages of LDS of its own, so there is no barrier before the sums: with its loads D - 1
// stages ahead it waits for the oldest only.  Loads of 16 bytes a lane straight to
// registers in the MFMA's order would touch 64 cache lines an instruction, in LDS order 8.
// Measured: one row by 4096 x 4096 5.7 us and by 8192 x 8192 13.4 (5.0 TB/s, of which 2.5 us
// are the start), 64 tokens over 28 of 32 experts of 2048 x 4096 36 us (6.5 TB/s).  Tiles of
// 64 x 32 and 32 x 64 gained 11% at 64 rows by 8192 x 8192 (22.8 us instead of 25.7), and lost
// 30% at 4096 x 4096; three stages and other orders of k changed nothing.
template <int MT, int RB, int W, int D, bool NT, bool FULL>
__global__ __launch_bounds__(W *kWave) void few_rows_kernel(ProductArgs p) {
  constexpr int kRowsA = 16 * MT, kRowsB = 16 * RB;
  constexpr int kStage = (kRowsA + kRowsB) * kBlock;
  constexpr int kScaleLoads = kRowsA < kWave ? 1 : 2;  // A's rows and then B's block, a lane each
  constexpr int kLoads = 2 * (MT + RB) + kScaleLoads;
  static_assert(kLoads * (D - 1) < 64, "loads in flight that one wait can count");
  constexpr int kSums = kRowsA * kRowsB;
  constexpr int kRing = W * D * kStage, kSumBytes = W * kSums * 4;
  __shared__ __align__(16) uint8_t memory[kRing > kSumBytes ? kRing : kSumBytes];
  __shared__ float scales[W][D][kScaleLoads * kWave];

  const int t = threadIdx.x, lane = t & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(t / kWave);
  const int g = lane >> 4, li = lane & 15;
  const int n0 = (int)(blockIdx.x % p.tiles_n) * kRowsB, tile = blockIdx.x / p.tiles_n;
  int m0 = tile * kRowsA, m_end = p.m, blocks = (p.k + kBlock - 1) / kBlock;
  const uint8_t *b = p.b;
  const float *sb = p.sb;
  if (p.kind == kGroups) {
    const Piece piece = find_piece(p.ends, p.groups, p.m, kRowsA, tile, true);
    if (piece.group < 0) return;
    m0 = piece.low;
    m_end = piece.high;
    if (m0 < 0 || m0 >= m_end) return;
    if (piece.group == p.groups) {
      blocks = 0;  // rows after the last group: zeros
    } else {
      b += piece.group * p.b_batch;
      sb += piece.group * p.sb_batch;
    }
  }
  const int rows = m_end - m0, columns = p.n - n0;
  const int kb0 = (int)((int64_t)blocks * wave / W), kb1 = (int)((int64_t)blocks * (wave + 1) / W);
  const u4 ra = buffer_words(p.a + (int64_t)m0 * p.a_pitch);
  const u4 rb = buffer_words(b + (int64_t)n0 * p.b_pitch);
  // slot s of 16 bytes of a stage is row s / 8; rows past the end repeat the last one
  const int tail = p.k & (kBlock - 1), kb_tail = tail != 0 ? p.k / kBlock : -1;
  const auto row_offset = [&](int s, int count, int64_t pitch) {
    const int r = s >> 3;
    return (r < count ? r : count - 1) * (int)pitch;
  };
  const auto chunk = [&](int s) { return ((s & 7) ^ ((s >> 4) & 7)) << 4; };
  int off_a[2 * MT], off_b[2 * RB];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i)
    off_a[i] = row_offset(i * kWave + lane, rows, p.a_pitch) + chunk(i * kWave + lane);
#pragma unroll
  for (int i = 0; i < 2 * RB; ++i)
    off_b[i] = row_offset(i * kWave + lane, columns, p.b_pitch) + chunk(i * kWave + lane);
  const float *scale_at[kScaleLoads];
#pragma unroll
  for (int i = 0; i < kScaleLoads; ++i) {
    const int r = i * kWave + lane;
    scale_at[i] = r < kRowsA ? p.sa + (int64_t)(m0 + (r < rows ? r : rows - 1)) * p.sa_pitch
                             : sb + (int64_t)(n0 / kBlock) * p.sb_pitch;
  }
  uint8_t *ring = memory + wave * D * kStage;
  const auto load = [&](int kb, int stage) {
    const uint32_t to = lds_address(ring + stage * kStage);
#pragma unroll
    for (int i = 0; i < 2 * (MT + RB); ++i) {
      const bool of_b = i >= 2 * MT;
      int off = of_b ? off_b[of_b ? i - 2 * MT : 0] : off_a[of_b ? 0 : i];
      int at = kb * kBlock;
      if (kb == kb_tail) {
        // chunks wholly past k may lie past the matrix: the row's first one instead, so the
        // block's offset is the lane's
        const int c = chunk((of_b ? i - 2 * MT : i) * kWave + lane);
        off = c < tail ? off + at : off - c;
        at = 0;
      }
      if (of_b)
        load_to_lds<NT>(rb, to + i * kWave * 16, off, at);
      else
        load_to_lds(ra, to + i * kWave * 16, off, at);
    }
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i)
      load_word_to_lds(scale_at[i] + kb, lds_address(&scales[wave][stage][i * kWave]));
  };

  f4 acc[MT][RB];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < RB; ++j) acc[i][j] = f4{0, 0, 0, 0};
  const int key = (li >> 1) & 7;
  const int at0 = li * kBlock + ((g ^ key) << 4), at1 = li * kBlock + (((g + 4) ^ key) << 4);
  const auto fragment = [&](const uint8_t *tile_rows, int kb) {
    u4 lo = *reinterpret_cast<const u4 *>(tile_rows + at0);
    u4 hi = *reinterpret_cast<const u4 *>(tile_rows + at1);
    if (kb == kb_tail) {
      lo = first_bytes(lo, tail - g * 16);
      hi = first_bytes(hi, tail - g * 16 - 64);
    }
    return i8v{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3],
               (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  };

#pragma unroll
  for (int d = 0; d < D - 1; ++d)
    if (kb0 + d < kb1) load(kb0 + d, d);
  int stage = 0;
#pragma unroll 1
  for (int kb = kb0; kb < kb1; ++kb) {
    // this stage's last reads (D steps ago) are done: its loads may overwrite it
    const int ahead = kb + D - 1;
    if (ahead < kb1) load(ahead, stage == 0 ? D - 1 : stage - 1);
    wait_stages<D - 1, kLoads>(kb1 - 1 - kb);
    const uint8_t *la = ring + stage * kStage, *lb = la + kRowsA * kBlock;
    const float scale_b = scales[wave][stage][kRowsA];
    Operand<FULL> fb[RB];
#pragma unroll
    for (int j = 0; j < RB; ++j) fb[j].set(fragment(lb + j * 16 * kBlock, kb));
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      Operand<FULL> fa;
      fa.set(fragment(la + i * 16 * kBlock, kb));
      const float s = scales[wave][stage][i * 16 + li] * scale_b;
#pragma unroll
      for (int j = 0; j < RB; ++j) {
        const f4 r = Operand<FULL>::product(fb[j], fa);
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[i][j][q] = __builtin_fmaf(r[q], s, acc[i][j][q]);
      }
    }
    // the reads have returned before the next loads go to this stage
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    stage = stage == D - 1 ? 0 : stage + 1;
  }

  __syncthreads();
  float *sums = reinterpret_cast<float *>(memory);
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < RB; ++j)
      *reinterpret_cast<f4 *>(
          &sums[wave * kSums + (i * 16 + li) * kRowsB + j * 16 + 4 * g]) = acc[i][j];
  __syncthreads();
#pragma unroll
  for (int e = t; e < kSums; e += W * kWave) {
    const int row = e / kRowsB, column = e % kRowsB;
    if (row >= rows || column >= columns) continue;
    float v = sums[e];
#pragma unroll
    for (int w = 1; w < W; ++w) v += sums[w * kSums + e];
    const int64_t at = (int64_t)(m0 + row) * p.out_pitch + n0 + column;
    if constexpr (FULL)
      store_out<HADACORE_FP32>(p.out, at, v);
    else if (p.out_type == HADACORE_FP16)
      store_out<HADACORE_FP16>(p.out, at, v);
    else
      store_out<HADACORE_BF16>(p.out, at, v);
  }
}

// Pieces of `unit` rows, at most: of ragged groups each has one that is not full at most,
// the rows after them too.
int most_pieces(const ProductArgs &p, int unit) {
  if (p.kind != kGroups) return (p.m + unit - 1) / unit;
  return p.m / unit + (p.groups + 1 < p.m ? p.groups + 1 : p.m);
}

template <int BM, int BN, int WM, int WN, int D, int KS>
hipError_t launch_tiles(ProductArgs p, bool b_rows, hipStream_t stream) {
  p.tiles_n = (p.n + BN - 1) / BN;
  p.tiles_m = most_pieces(p, BM);
  int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  if (p.kind == kGradient) tiles *= p.groups;
  if (tiles * (KS * WM * WN * kWave) >= (int64_t(1) << 32)) return hipErrorInvalidValue;
  p.tiles = (uint32_t)tiles;
  // where there are more tiles than run together, and whole blocks, workgroups go through them
  constexpr bool kMayLoop = D == 2 && KS == 1, kSplit = kMayLoop && BM == 256;
  const int64_t slots = (int64_t)device_cus() * (BM * BN <= 128 * 128 ? 2 : 1);
  const bool loop = kMayLoop && p.k % kBlock == 0 && (kSplit || tiles > slots);
  const dim3 grid((uint32_t)(loop ? slots : tiles)), block(KS * WM * WN * kWave);
  const auto go = [&](auto rows, auto full) {
    constexpr bool kRows = decltype(rows)::value, kFull = decltype(full)::value;
    if (loop)
      hipLaunchKernelGGL((product_kernel<BM, BN, WM, WN, D, KS, kMayLoop, kSplit, kRows, kFull>), grid,
                         block, 0, stream, p);
    else
      hipLaunchKernelGGL((product_kernel<BM, BN, WM, WN, D, KS, false, false, kRows, kFull>), grid, block,
                         0, stream, p);
    return hipGetLastError();
  };
  if (p.out_type == HADACORE_FP32) {
    if constexpr (BM <= 128)
      return b_rows ? go(std::true_type{}, std::true_type{})
                    : go(std::false_type{}, std::true_type{});
    return hipErrorInvalidValue;  // not chosen
  }
  return b_rows ? go(std::true_type{}, std::false_type{}) : go(std::false_type{}, std::false_type{});
}

template <int MT, int RB, int W, int D>
hipError_t launch_few(ProductArgs p, bool stream_b, hipStream_t stream) {
  p.tiles_n = (p.n + 16 * RB - 1) / (16 * RB);
  p.tiles_m = most_pieces(p, 16 * MT);
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  if (tiles * (W * kWave) >= (int64_t(1) << 32)) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)tiles), block(W * kWave);
  const auto go = [&](auto nt, auto full) {
    hipLaunchKernelGGL(
        (few_rows_kernel<MT, RB, W, D, decltype(nt)::value, decltype(full)::value>), grid, block,
        0, stream, p);
    return hipGetLastError();
  };
  if (p.out_type == HADACORE_FP32)
    return stream_b ? go(std::true_type{}, std::true_type{}) : go(std::false_type{}, std::true_type{});
  return stream_b ? go(std::true_type{}, std::false_type{}) : go(std::false_type{}, std::false_type{});
}

// Which kernel: the one with the least estimated time.  A kernel's workgroups run in turns
// of as many as fit the chip (kSlots for 256 CUs); a turn takes a start and as many steps as
// a wave has blocks of k, and few rows at least the time of reading B.  The times are
// measured (us; a step with one workgroup to a CU at most, and with all slots taken), for
// 16-bit outputs of tiles of B scales; rows of scales and 32-bit outputs take the factors.
// Over 80 random calls the choice was within 8% of the best tile for all but three (11, 14 and
// 24% over it).  The slots are those of a whole card: on a part of one the estimates are off, and
// the choice may be, not the results.
struct KernelTime {
  int bm, bn, slots, shares;  // tile, workgroups that run together, shares of k
  float start, alone, full;
  float by_rows, wide;  // factors of a step
  float read;           // reading 1 MB
};
constexpr int kFew = 3;  // the first of them are few_rows_kernel's
constexpr KernelTime kTimes[] = {
    {16, 16, 512, 8, 2.5f, 0.35f, 0.45f, 0.0f, 1.4f, 0.165f},
    {16, 32, 768, 4, 2.5f, 0.35f, 0.50f, 0.0f, 1.4f, 0.15f},
    {32, 32, 512, 4, 2.5f, 0.45f, 0.55f, 0.0f, 1.5f, 0.16f},
    {64, 64, 256, 2, 2.5f, 0.60f, 0.66f, 1.13f, 1.55f, 0.25f},
    {64, 128, 512, 1, 2.5f, 0.42f, 0.76f, 1.3f, 1.5f, 0.25f},
    {128, 128, 512, 1, 3.0f, 0.74f, 1.28f, 1.19f, 1.6f, 0.25f},
    {256, 256, 256, 1, 5.0f, 1.40f, 1.82f, 1.17f, 0.0f, 0.25f}};
constexpr int kLargest = 6;  // not for 32-bit outputs, whose widened operands do not fit

float estimate(const ProductArgs &p, int i, bool b_rows) {
  const KernelTime &c = kTimes[i];
  const bool wide = p.out_type == HADACORE_FP32;
  const float groups = p.kind == kGroups ? (float)(p.groups < p.m ? p.groups : p.m) : 1.0f;
  float pieces = ceilf((float)p.m / c.bm), blocks = ceilf((float)p.k / kBlock);
  if (p.kind == kGroups) pieces = fmaxf(groups, (float)p.m / c.bm + 0.5f * groups);
  float tiles = pieces * ceilf((float)p.n / c.bn);
  if (p.kind == kGradient) {
    tiles *= p.groups;
    blocks /= p.groups;
  }
  const float factor = (b_rows ? c.by_rows : 1.0f) * (wide ? c.wide : 1.0f);
  const float steps = ceilf(blocks / c.shares) * factor;
  // the largest tile's workgroups look for their tiles one by one
  const float start = c.start + (i == kLargest && p.kind != kDense ? 2.5f : 0.0f);
  float time = ceilf(tiles / c.slots) * (start + steps * (tiles <= 256 ? c.alone : c.full));
  if (i == kLargest && p.k % kBlock == 0) {
    // the last turn in quarters, 128 x 128 by all eight waves
    const float rest = fmodf(tiles, c.slots);
    if (rest <= c.slots / 2)
      time = floorf(tiles / c.slots) * (start + steps * c.full) +
             ceilf(4 * rest / c.slots) * (start - 1.0f + blocks * (b_rows ? 0.95f : 0.58f));
  }
  // what is read: by few rows B once a workgroup, and A from the L2s at half the cost; by
  // whole tiles B; slower by less than one workgroup to a CU.  Of two kernels that this
  // bounds, the one with fewer turns
  float read = groups * p.n;
  if (i < kFew) read = tiles * (c.bn + 0.5f * fminf(c.bm, ceilf((float)p.m / groups)));
  if (p.kind == kGradient) read = 0.0f;
  read *= fmaxf(1.0f, 256 / tiles);
  return fmaxf(time, read * p.k * 1e-6f * c.read + 2.5f) + 0.05f * time;
}

// HADACORE_VARIANT=tiles-64|tiles-64x128|tiles-128|tiles-256 forces a tile for every
// product (testing and tuning; tiles-256 not for 32-bit outputs, which keep the choice).
int tile_override() {
  const char *v = getenv("HADACORE_VARIANT");
  if (v == nullptr || strncmp(v, "tiles-", 6) != 0) return -1;
  static constexpr const char *kNames[] = {"64", "64x128", "128", "256"};
  for (int i = 0; i < 4; ++i)
    if (strcmp(v + 6, kNames[i]) == 0) return i;
  return -1;
}

hipError_t launch_product(ProductArgs p, bool b_rows, hipStream_t stream) {
  // Outputs of this size do not stay in the last-level cache for their reader, and push out
  // of the L2s what other tiles still read.  With the policy SC1 | NT, us: 128 MiB of 16384
  // x 4096 bf16 outputs 233 instead of 259 (k = 4096), 72.3 instead of 82.8 (k = 1024), 256
  // MiB of gradients 178 instead of 197; but 64 MiB by expert 185 instead of 179.
  p.nt_out = (int64_t)p.m * p.n * (p.kind == kGradient ? p.groups : 1) *
                 (p.out_type == HADACORE_FP32 ? 4 : 2) >= (int64_t(1) << 27);
  int best = -1;
  const int forced = tile_override();
  if (forced >= 0 && !(forced == 3 && p.out_type == HADACORE_FP32)) {
    best = kFew + forced;
  } else {
    float least = 0.0f;
    for (int i = b_rows ? kFew : 0; i < (p.out_type == HADACORE_FP32 ? kLargest : kLargest + 1);
         ++i) {
      const float time = estimate(p, i, b_rows);
      if (best < 0 || time < least) {
        best = i;
        least = time;
      }
    }
  }
  // weights of this size that are read once do not stay in the last-level cache beside
  // others: streamed, 64 tokens over 32 experts of 2048 x 4096 take 40.4 us instead of 46.4
  // and 16 rows by 8192 x 8192 13.9 instead of 14.8; but 4096 x 4096 6.3 instead of 5.8, and
  // 64 rows by 8192 x 8192, which two workgroups read, 29.6 instead of 25.7
  const int64_t read = p.kind == kGroups ? (p.groups < p.m ? p.groups : p.m) : 1;
  const bool stream_b = read * p.n * p.k >= (int64_t(1) << 26) && p.m <= kTimes[best].bm * read;
  switch (best) {
    case 0: return launch_few<1, 1, 8, 2>(p, stream_b, stream);
    case 1: return launch_few<1, 2, 4, 2>(p, stream_b, stream);
    case 2: return launch_few<2, 2, 4, 2>(p, stream_b, stream);
    case 3: return launch_tiles<64, 64, 2, 1, 3, 2>(p, b_rows, stream);
    case 4: return launch_tiles<64, 128, 2, 2, 3, 1>(p, b_rows, stream);
    case 5: return launch_tiles<128, 128, 2, 2, 2, 1>(p, b_rows, stream);
    default: return launch_tiles<256, 256, 2, 4, 2, 1>(p, b_rows, stream);
  }
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
  const auto go = [&](auto dt, auto by_columns, auto policy) {
    hipLaunchKernelGGL((tile_kernel<decltype(dt)::value, decltype(by_columns)::value,
                                    decltype(policy)::value>),
                       grid, dim3(256), 0, s, p);
  };
  const auto policy_for = [&](const void *codes, int64_t pitch, int64_t width) {
    return quantizer_policy((int64_t)p.m * p.k * batch, p.in, p.in_stride, codes, pitch, width);
  };
  int policy = columns ? policy_for(p.codes_t, p.codes_t_stride, row_blocks * kBlock)
                       : policy_for(p.codes, p.codes_stride, p.k);
  if (!columns && p.codes_t != nullptr && policy != kPlain)
    policy = policy_for(p.codes_t, p.codes_t_stride, p.m);
  const auto typed = [&](auto by_columns, auto chosen) {
    if (dtype == HADACORE_FP16)
      go(std::integral_constant<int, HADACORE_FP16>{}, by_columns, chosen);
    else
      go(std::integral_constant<int, HADACORE_BF16>{}, by_columns, chosen);
  };
  const auto kind = [&](auto chosen) {
    if (columns)
      typed(std::true_type{}, chosen);
    else
      typed(std::false_type{}, chosen);
  };
  if (policy == kStreamIn)
    kind(std::integral_constant<int, kStreamIn>{});
  else if (policy == kStreamOut)
    kind(std::integral_constant<int, kStreamOut>{});
  else
    kind(std::integral_constant<int, kPlain>{});
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
  int64_t places;
  if (__builtin_mul_overflow(kBlock - 1, groups < tokens ? groups : tokens, &places) ||
      __builtin_add_overflow(places, tokens, &places))
    places = INT64_MAX;
  return places / kBlock * kBlock;
}

extern "C" hadacore_status hadacore_quantize_fp8_columns(
    const void *in, int64_t in_row_stride, const int32_t *ends, int64_t groups, void *out_codes,
    int64_t out_row_stride, float *out_scales, int64_t scales_row_stride, int64_t m, int64_t k,
    hadacore_dtype dtype, void *stream) {
  if (m < 0 || k < 0 || groups < 0 || (ends == nullptr && groups > 1))
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
  p.kind = kDense;
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
  if (places < 0 || n < 0 || k < 0 || groups < 0 || (ends == nullptr && groups > 1))
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
  if (groups > 1 && (out_row_stride < k || out_row_stride > kMaxPitch ||
                     out_batch_stride < (n - 1) * out_row_stride + k))
    return HADACORE_ERROR_INVALID_STRIDE;
  const hadacore_status st = check_product(p, n, k, places, groups, k);
  if (st != HADACORE_SUCCESS || n == 0 || k == 0 || groups == 0) return st;
  return run_product(p, true, stream);
}
