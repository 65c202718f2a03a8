// adapters.hip -- low-rank adapters of many requests beside a shared projection.
//
// Token t of group (adapter) g, with down[g] (rank x k) and up[g] (rank x n):
//
//   h_t = down[g] x_t,   out_t = y_t + s_g up[g]^T h_t                        (two launches)
//
// and the gradients are the same two products with the roles changed,
//
//   dh_t = up[g] dout_t,   dx_t = s_g down[g]^T dh_t,
//
// and dW[g] = s_g sum_t h_t x_t^T for either weight.  With both weights stored rank-major the
// three kernels serve forward and backward, and no weight is transposed in memory.
//
// What bounds them is HBM: x is read once, y and out once each, and the weights of the groups
// that have tokens; 2 rank operations for each 2 bytes are far below what the matrix cores do.
//
// Sums are the matrix cores' fp32.  h stays in fp32 between the two products: the second takes it
// in three parts of 16 bits that add up to all 24 bits of it, for 16-bit results too, since the
// adapter's part may cancel against y and leave any bit of h to be seen.  (Two parts, which keep 16
// bits of it in bf16, save 0 to 4% of a call.)  fp16 parts are made of h times a power of two (largest
// value of the row near 2^10): all bits of values down to 2^-11 of the row's largest, and of smaller
// ones those above 2^-35 of it.  A value of h, a weight or an x that is Inf gives a NaN where the sum
// without parts may give Inf: Inf times a part of 0 is NaN.

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "adapters_cut.h"
#include "groups.h"
#include "hadacore.h"
#include "internal.h"
#include "lds_loads.h"

namespace hadacore {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef u4 u4_any __attribute__((aligned(2)));
typedef u2 u2_any __attribute__((aligned(2)));

// D (16 x 16) += A B: lane l holds A[l % 16][8 (l / 16) + j], B[8 (l / 16) + j][l % 16] and
// D[4 (l / 16) + v][l % 16].
template <int DT>
__device__ __forceinline__ f4 mfma(u4 a, u4 b, f4 c) {
  if constexpr (DT == HADACORE_FP16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a),
                                                  __builtin_bit_cast(h8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a),
                                                   __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}

template <int DT>
__device__ __forceinline__ uint16_t narrow(float v) {
  if constexpr (DT == HADACORE_FP16)
    return __builtin_bit_cast(uint16_t, (_Float16)v);
  else
    return __builtin_bit_cast(uint16_t, (__bf16)v);
}

template <int DT>
__device__ __forceinline__ float widen(uint16_t h) {
  if constexpr (DT == HADACORE_FP16)
    return (float)__builtin_bit_cast(_Float16, h);
  else
    return __builtin_bit_cast(float, (uint32_t)h << 16);
}

// Takes part i off v, a sum of kParts values of 16 bits.  Parts of bf16 but the last are cut off, so that a
// NaN stays one (what is left of it is a quiet NaN) and no part rounds up to Inf.
template <int DT>
__device__ __forceinline__ uint16_t take_part(float &v, int i) {
  const uint16_t part = DT == HADACORE_FP16 || i == kParts - 1
                            ? narrow<DT>(v)
                            : (uint16_t)(__builtin_bit_cast(uint32_t, v) >> 16);
  v -= widen<DT>(part);
  return part;
}
// The same for two values, as a word.
template <int DT>
__device__ __forceinline__ uint32_t take_parts(float &low, float &high, int i) {
  const uint32_t part = take_part<DT>(low, i);
  return part | (uint32_t)take_part<DT>(high, i) << 16;
}

// The power of two that brings values of at most `most` to at most 2^11: exponent of its inverse.
// Zero, subnormal, infinite and NaN take the nearest that is finite.
__device__ __forceinline__ int scale_exponent(float most) {
  const int e = (int)((__builtin_bit_cast(uint32_t, most) >> 23) & 255) - 127 - 10;
  return e < -100 ? -100 : e > 100 ? 100 : e;
}
__device__ __forceinline__ float power_of_two(int e) {
  return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
}

// 8 values of a row (`valid` of them there, zeros behind).  Rows may start at any value's address.
__device__ __forceinline__ u4 load8(const uint16_t *p, int64_t valid) {
  if (valid >= 8) return *reinterpret_cast<const u4_any *>(p);
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < valid) w[i / 2] |= (uint32_t)p[i] << (16 * (i % 2));
  return u4{w[0], w[1], w[2], w[3]};
}

// The words moved down by `by` of them, zeros behind; of more than N, any of them.
template <int N>
__device__ __forceinline__ void move_words(uint32_t (&w)[N], int by) {
#pragma unroll
  for (int step = N / 2; step > 0; step /= 2)
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = (by & step) != 0 ? (i + step < N ? w[i + step < N ? i + step : 0] : 0) : w[i];
}
// The same for 16-bit values, two a word.
template <int N>
__device__ __forceinline__ void move_values(uint32_t (&w)[N], int by) {
  move_words<N>(w, by / 2);
#pragma unroll
  for (int i = 0; i < N; ++i)
    w[i] = (by & 1) != 0 ? (w[i] >> 16) | (i + 1 < N ? w[i + 1 < N ? i + 1 : 0] << 16 : 0) : w[i];
}

// Eight values moved down by any number of them, zeros behind.
__device__ __forceinline__ u4 moved(u4 v, int by) {
  uint32_t w[4] = {v[0], v[1], v[2], v[3]};
  move_values<4>(w, by);
  return by < 8 ? u4{w[0], w[1], w[2], w[3]} : u4{0, 0, 0, 0};
}

// How far before its own place a lane loads N values, `valid` of which are there, so that they end
// with the row: in a row of N and more they are inside it, and no load stands in a branch, where a
// wave would wait for each by itself.  move_values() then brings them to their places.  (When it came in:
// up_kernel, 3525 x 997, rank 95: 20 us instead of 55; gradient_any_kernel, 1957 x 5597, rank 9: 18
// instead of 35.)
template <int N>
__device__ __forceinline__ int ahead_of(int64_t valid) {
  return valid >= N ? 0 : N - (int)valid;
}

// Eight rows of 8 (or 4) consecutive columns, turned: column i's eight values in `col[i]`.
template <int CT>
__device__ __forceinline__ void turn(const uint32_t (&row)[8][CT / 2], u4 (&col)[CT]) {
#pragma unroll
  for (int q = 0; q < CT / 2; ++q) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t pick = h == 0 ? 0x05040100u : 0x07060302u;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        col[2 * q + h][j] = __builtin_amdgcn_perm(row[2 * j + 1][q], row[2 * j][q], pick);
    }
  }
}

// CT consecutive columns of a row as pairs.
template <int CT>
__device__ __forceinline__ void load_columns(const uint16_t *p, int64_t valid, uint32_t (&w)[CT / 2]) {
  if constexpr (CT == 8) {
    const u4 v = load8(p, valid);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = v[i];
  } else {
    w[0] = w[1] = 0;
    if (valid >= 4) {
      const u2 v = *reinterpret_cast<const u2_any *>(p);
      w[0] = v[0];
      w[1] = v[1];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < valid) w[i / 2] |= (uint32_t)p[i] << (16 * (i % 2));
    }
  }
}

// Maximum over groups of `lanes` lanes of a wave, in steps of xor.
__device__ __forceinline__ float max_lanes(float x, int lanes) {
  for (int step = 1; step < lanes; step *= 2) x = fmaxf(x, __shfl_xor(x, step));
  return x;
}

struct AdapterArgs {
  const uint16_t *x, *down, *up;
  int64_t x_stride, down_stride, down_batch, up_stride, up_batch;
  const float *scales;
  const int32_t *ends, *slots;
  const void *y;
  void *out;
  int64_t y_stride, out_stride;
  float *part;  // h of each share of k: [splits][m][part_pitch], zero behind the rank up to `padded`
  int64_t part_pitch, part_step;
  float *hidden;  // where h goes besides
  int64_t hidden_stride;
  int m, k, n, rank, padded, groups, splits, unit, chunks;  // padded: the rank in whole tiles
};

// The token of a place; a wrong slot gives a wrong row, but no access out of bounds.
__device__ __forceinline__ int token_of(const int32_t *slots, int place, int m) {
  if (slots == nullptr) return place;
  const int s = slots[place];
  return s < 0 ? 0 : s >= m ? m - 1 : s;
}

// Without ends all rows are one group.
__device__ __forceinline__ Piece piece_of(const int32_t *ends, int groups, int m, int unit, int id,
                                          bool rest) {
  if (ends != nullptr || groups == 0) return find_piece(ends, groups, m, unit, id, rest);
  return {id * (int64_t)unit < m ? 0 : -1, id * unit, m};
}

// h for 16 TT tokens of a group, 16 RT of its ranks and one of `splits` shares of k.  W waves
// take a part of the share each and add up at the end, so that each value of x and of
// the weights is loaded by one wave, straight into the operands of the matrix products: both
// have k along their rows.  U steps of k are loaded ahead of the U being multiplied.
template <int DT, int TT, int RT, int U, int W>
__global__ __launch_bounds__(W *kWave) void down_kernel(AdapterArgs p) {
  constexpr int kTiles = TT * RT;
  __shared__ f4 sums[W][kTiles][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c = lane % kTile, quarter = lane / kTile;
  const Piece piece = piece_of(p.ends, p.groups, p.m, kTile * TT, blockIdx.x, false);
  if (piece.group < 0) return;
  const int rank0 = blockIdx.z * (kTile * RT);
  // whole steps of k, then (by the last wave) the rest of it
  const int64_t steps = p.k / kStep;
  const int shares = p.splits * W, share = blockIdx.y * W + wave;
  const int from = (int)(steps * share / shares), to = (int)(steps * (share + 1) / shares);
  const uint16_t *xp[TT], *wp[RT];
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    const int place = piece.low + t * kTile + c;
    xp[t] = p.x + token_of(p.slots, place < piece.high ? place : piece.high - 1, p.m) * p.x_stride +
            quarter * 8 + (int64_t)from * kStep;
  }
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = rank0 + r * kTile + c;
    wp[r] = p.down + piece.group * p.down_batch + (row < p.rank ? row : p.rank - 1) * p.down_stride +
            quarter * 8 + (int64_t)from * kStep;
  }
  f4 acc[TT][RT] = {};
  u4 xv[2][U][TT], wv[2][U][RT];
  const auto load = [&](int buffer) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int t = 0; t < TT; ++t)
        xv[buffer][u][t] = *reinterpret_cast<const u4_any *>(xp[t] + u * kStep);
#pragma unroll
      for (int r = 0; r < RT; ++r)
        wv[buffer][u][r] = *reinterpret_cast<const u4_any *>(wp[r] + u * kStep);
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) xp[t] += U * kStep;
#pragma unroll
    for (int r = 0; r < RT; ++r) wp[r] += U * kStep;
  };
  const auto multiply = [&](int buffer) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int r = 0; r < RT; ++r)
          acc[t][r] = mfma<DT>(wv[buffer][u][r], xv[buffer][u][t], acc[t][r]);
  };
  const int turns = (to - from) / U;
  if (turns > 0) load(0);
  for (int s = 0; s < turns; s += 2) {
    if (s + 1 < turns) load(1);
    multiply(0);
    if (s + 1 >= turns) break;
    if (s + 2 < turns) load(0);
    multiply(1);
  }
  const int left = (to - from) % U + (share == shares - 1 && p.k % kStep != 0);
  for (int s = 0; s < left; ++s) {
    const int valid = (from + turns * U + s < to ? kStep : p.k % kStep) - quarter * 8;
    if (p.k >= 8) {
      const int by = ahead_of<8>(valid);
#pragma unroll
      for (int t = 0; t < TT; ++t)
        xv[0][0][t] = *reinterpret_cast<const u4_any *>(xp[t] + s * kStep - by);
#pragma unroll
      for (int r = 0; r < RT; ++r)
        wv[0][0][r] = *reinterpret_cast<const u4_any *>(wp[r] + s * kStep - by);
      if (by > 0) {
#pragma unroll
        for (int t = 0; t < TT; ++t) xv[0][0][t] = moved(xv[0][0][t], by);
#pragma unroll
        for (int r = 0; r < RT; ++r) wv[0][0][r] = moved(wv[0][0][r], by);
      }
    } else {
#pragma unroll
      for (int t = 0; t < TT; ++t) xv[0][0][t] = load8(xp[t] + s * kStep, valid);
#pragma unroll
      for (int r = 0; r < RT; ++r) wv[0][0][r] = load8(wp[r] + s * kStep, valid);
    }
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int r = 0; r < RT; ++r) acc[t][r] = mfma<DT>(wv[0][0][r], xv[0][0][t], acc[t][r]);
  }
#pragma unroll
  for (int i = 0; i < kTiles; ++i) sums[wave][i][lane] = acc[i / RT][i % RT];
  __syncthreads();
  for (int i = wave; i < kTiles; i += W) {
    f4 v = sums[0][i][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) v += sums[w][i][lane];
    const int place = piece.low + i / RT * kTile + c;
    const int rank = rank0 + i % RT * kTile + 4 * quarter;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (rank + j >= p.rank) v[j] = 0.0f;
    if (place < piece.high && rank < p.padded)
      *reinterpret_cast<f4 *>(p.part + blockIdx.y * p.part_step + place * p.part_pitch + rank) = v;
  }
}

// Values that are read or written once: where rows are whole lines, the streaming policy (NT)
// keeps them from pushing the weights and h out of the L2 (16384 x 8192: up_kernel 122 us instead of
// 133, a call 158 instead of 168).  Rows that share lines are slower with it (1733 x 5003 in 32 bits: 28 instead of 23).
template <bool NT, class V>
__device__ __forceinline__ V stream_in(const void *p) {
  if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const V *>(p));
  return *reinterpret_cast<const V *>(p);
}
template <bool NT, class V>
__device__ __forceinline__ void stream_out(void *p, V v) {
  if constexpr (NT)
    __builtin_nontemporal_store(v, reinterpret_cast<V *>(p));
  else
    *reinterpret_cast<V *>(p) = v;
}

// CT consecutive outputs of a row as words.
template <int OUT, int CT, bool NT>
struct OutRow {
  static constexpr int kWords = CT * (OUT == HADACORE_FP32 ? 4 : 2) / 4;
  uint32_t w[kWords];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (OUT == HADACORE_FP32)
      return __builtin_bit_cast(float, w[i]);
    else
      return widen<OUT>((uint16_t)(w[i / 2] >> (16 * (i % 2))));
  }
  __device__ __forceinline__ void set(const float (&v)[CT]) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (OUT == HADACORE_FP32)
        w[i] = __builtin_bit_cast(uint32_t, v[i]);
      else
        w[i] = narrow<OUT>(v[2 * i]) | (uint32_t)narrow<OUT>(v[2 * i + 1]) << 16;
    }
  }
  // Rows may start at any value's address.
  __device__ __forceinline__ void load(const uint8_t *p) {
    if constexpr (kWords == 2) {
      const u2 v = stream_in<NT, u2_any>(p);
      w[0] = v[0];
      w[1] = v[1];
    } else {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const u4 v = stream_in<NT, u4_any>(p + 16 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
      }
    }
  }
  // the first `valid` of the CT values
  __device__ __forceinline__ void load(const uint8_t *p, int64_t valid) {
    if (valid >= CT) return load(p);
    clear();
#pragma unroll
    for (int i = 0; i < CT; ++i) {
      if (i >= valid) continue;
      if constexpr (OUT == HADACORE_FP32)
        w[i] = reinterpret_cast<const uint32_t *>(p)[i];
      else
        w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << (16 * (i % 2));
    }
  }
  __device__ __forceinline__ void move(int by) {
    if constexpr (OUT == HADACORE_FP32)
      move_words<kWords>(w, by);
    else
      move_values<kWords>(w, by);
  }
  __device__ __forceinline__ void store(uint8_t *p) const {
    if constexpr (kWords == 2) {
      stream_out<NT, u2_any>(p, u2{w[0], w[1]});
    } else {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i)
        stream_out<NT, u4_any>(p + 16 * i, u4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]});
    }
  }
  __device__ __forceinline__ void store(uint8_t *p, int64_t valid) const {
    if (valid >= CT) return store(p);
#pragma unroll
    for (int i = 0; i < CT; ++i) {
      if (i >= valid) continue;
      if constexpr (OUT == HADACORE_FP32)
        reinterpret_cast<uint32_t *>(p)[i] = w[i];
      else
        reinterpret_cast<uint16_t *>(p)[i] = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
    }
  }
};

// out for up to `unit` tokens of a group and 4 * 16 CT columns.  A wave keeps the weights of its
// 16 CT columns in registers for all these tokens: 8 rows of CT columns a lane, turned in
// registers so that the ranks lie along an operand.  A lane then has CT consecutive columns of each
// of four tokens, which it loads and stores whole, the next four's y under the products of these.
// h, joined and split, goes through LDS.  Tokens behind the last end get y.
template <int DT, int OUT, int RB, int CT, int D, bool EVEN>
__global__ __launch_bounds__(256) void up_kernel(AdapterArgs p) {
  constexpr int P = kParts, kPitch = kStep * RB + 8;
  constexpr int kSize = OUT == HADACORE_FP32 ? 4 : 2;
  extern __shared__ __attribute__((aligned(16))) uint8_t room[];
  uint16_t *parts = reinterpret_cast<uint16_t *>(room);  // [unit][P][kPitch]
  float *back = reinterpret_cast<float *>(parts + P * p.unit * kPitch);
  int *tokens = reinterpret_cast<int *>(back + p.unit);
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int c = lane % kTile, quarter = lane / kTile;
  const int chunk = blockIdx.x % p.chunks;
  const Piece piece = piece_of(p.ends, p.groups, p.m, p.unit, blockIdx.x / p.chunks, true);
  if (piece.group < 0) return;
  const bool bare = piece.group == p.groups;  // no adapter
  if (bare && p.y == p.out) return;
  const int count = piece.high - piece.low < p.unit ? piece.high - piece.low : p.unit;
  const int col = (chunk * 4 + wave) * (kTile * CT) + c * CT;
  const int64_t valid = EVEN ? CT : (int64_t)p.n - col;
  // a wave behind the last column loads the first ones in their place
  const bool behind = (chunk * 4 + wave) * (kTile * CT) >= p.n;
  const bool wide = !EVEN && p.n >= CT;
  const int by = wide ? ahead_of<CT>(valid) : 0;
  uint32_t raw[RB][8][CT / 2];
  if (!bare) {
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int row = b * kStep + quarter * 8 + j;
        // ranks that are not there: any values, cleared below
        const uint16_t *at = p.up + piece.group * p.up_batch + (row < p.rank ? row : 0) * p.up_stride +
                             (EVEN && behind ? c * CT : col);
        if (wide)
          load_columns<CT>(at - by, CT, raw[b][j]);
        else
          load_columns<CT>(at, valid, raw[b][j]);
      }
  }
  const uint8_t *y = static_cast<const uint8_t *>(p.y);
  uint8_t *out = static_cast<uint8_t *>(p.out);
  using Row = OutRow<OUT, CT, EVEN>;
  // Whole tiles of 16 tokens whose columns are all there go without a branch in a lane, so that
  // loads stay in flight over stores and products.
  const bool whole = (chunk * 4 + wave + 1) * (kTile * CT) <= p.n;
  const int fast = whole && y != nullptr ? count / kTile * kTile : 0;
  Row old[D][4];
#pragma unroll
  for (int d = 0; d < D; ++d) {
    if (d * kTile >= fast) break;
#pragma unroll
    for (int v = 0; v < 4; ++v)
      old[d][v].load(y + (token_of(p.slots, piece.low + d * kTile + 4 * quarter + v, p.m) * p.y_stride +
                          col) * kSize);
  }
  const float scale = !bare && p.scales != nullptr ? p.scales[piece.group] : 1.0f;
  for (int t0 = 0; t0 < count; t0 += 256 / kTile) {
    const int t = t0 + tid / kTile, q = tid % kTile;
    if (t >= count) continue;
    const int place = piece.low + t;
    if (q == 0) tokens[t] = token_of(p.slots, place, p.m);
    if (bare) continue;
    constexpr int kEach = (kStep * RB + 63) / 64;
    f4 h[kEach];
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int r = i * 64 + q * 4;
      f4 v = f4{0, 0, 0, 0};
      if (r < p.padded) {
        const float *at = p.part + place * p.part_pitch + r;
        v = *reinterpret_cast<const f4 *>(at);
        // four shares' loads at a time, joined in order
        for (int s = 1; s < p.splits; s += 4) {
          f4 more[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            more[j] = s + j < p.splits ? *reinterpret_cast<const f4 *>(at + (s + j) * p.part_step)
                                       : f4{0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < 4; ++j) v += more[j];
        }
        if (p.hidden != nullptr && p.splits > 1 && chunk == 0)
          *reinterpret_cast<f4 *>(p.hidden + place * p.hidden_stride + r) = v;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] *= scale;
        most = fmaxf(most, fabsf(v[j]));
      }
      h[i] = v;
    }
    float shift = 1.0f;
    if constexpr (DT == HADACORE_FP16) {
      const int e = scale_exponent(max_lanes(most, kTile));
      shift = power_of_two(-e);
      if (q == 0) back[t] = power_of_two(e);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int r = i * 64 + q * 4;
      if (r >= kStep * RB) continue;
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = h[i][j] * shift;
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const uint32_t low = take_parts<DT>(v[0], v[1], k);
        *reinterpret_cast<u2 *>(parts + (t * P + k) * kPitch + r) =
            u2{low, take_parts<DT>(v[2], v[3], k)};
      }
    }
  }
  u4 w[RB][CT];
  if (!bare) {
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      if ((b + 1) * kStep > p.rank) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < CT / 2; ++i)
            raw[b][j][i] = b * kStep + quarter * 8 + j < p.rank ? raw[b][j][i] : 0;
      }
      if (by > 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) move_values<CT / 2>(raw[b][j], by);
      }
      turn<CT>(raw[b], w[b]);
    }
  }
  __syncthreads();
  // whole waves only: a matrix instruction reads the registers of all 64 lanes
  if (behind) return;
  const auto multiply = [&](int t0, f4 (&acc)[CT]) {
    if (bare) return;
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int k = P - 1; k >= 0; --k) {
        const u4 a = *reinterpret_cast<const u4 *>(
            parts + ((t0 + c) * P + k) * kPitch + b * kStep + quarter * 8);
#pragma unroll
        for (int i = 0; i < CT; ++i) acc[i] = mfma<DT>(a, w[b][i], acc[i]);
      }
  };
  const auto add = [&](int t, int v, const f4 (&acc)[CT], Row &row) {
    if (bare) return;  // y as it is
    const float unshift = DT == HADACORE_FP16 ? back[t] : 1.0f;
    float sum[CT];
#pragma unroll
    for (int i = 0; i < CT; ++i) sum[i] = fmaf(acc[i][v], unshift, row.get(i));
    row.set(sum);
  };
  for (int t0 = 0; t0 < fast; t0 += D * kTile) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int now = t0 + d * kTile, mine = now + 4 * quarter, next = now + D * kTile;
      if (now >= fast) break;
      f4 acc[CT] = {};
      multiply(now, acc);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        add(mine + v, v, acc, old[d][v]);
        old[d][v].store(out + (tokens[mine + v] * p.out_stride + col) * kSize);
      }
      if (next < fast) {
#pragma unroll
        for (int v = 0; v < 4; ++v)
          old[d][v].load(y + (tokens[next + 4 * quarter + v] * p.y_stride + col) * kSize);
      }
    }
  }
  // the rest; rows held a tile ahead, as above, cost a wave of four on a SIMD (7028 x 4304, rank 8: 24
  // us instead of 21)
  const bool early = y != nullptr && (EVEN || wide);
  for (int t0 = fast; t0 < count; t0 += kTile) {
    Row rest[4];
    if (early) {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int t = t0 + 4 * quarter + v < count ? t0 + 4 * quarter + v : count - 1;
        rest[v].load(y + (tokens[t] * p.y_stride + col - by) * kSize);
      }
      if (by > 0) {
#pragma unroll
        for (int v = 0; v < 4; ++v) rest[v].move(by);
      }
    } else {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int t = t0 + 4 * quarter + v;
        rest[v].clear();
        if (y != nullptr && t < count) rest[v].load(y + (tokens[t] * p.y_stride + col) * kSize, valid);
      }
    }
    f4 acc[CT] = {};
    multiply(t0, acc);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int t = t0 + 4 * quarter + v;
      if (t >= count) continue;
      add(t, v, acc, rest[v]);
      rest[v].store(out + (tokens[t] * p.out_stride + col) * kSize, valid);
    }
  }
}

// Both products in one launch, for up to 16 tokens of a group and 1024 columns: every workgroup makes
// h itself, which costs it the group's `down` again (from the L2) but saves a launch and the
// way of h through memory.  Eight waves share k and add up; then each has its 128 columns, whose weights
// and y were loaded at the start.  Called one by one 1 token of rank 16, 4096 x 4096 takes 11.5 us
// instead of 15.0, and 64 tokens of 32 adapters 11.6 instead of 15.1; inside a graph, where a launch
// costs little, 8.6 instead of 7.4 and 11.5 instead of 8.9.  For ranks up to 16 and few workgroups:
// 256 tokens of 64 adapters gain nothing, rank 64 takes 20 instead of 9.
template <int DT, int OUT, bool EVEN>
__global__ __launch_bounds__(kFewWaves *kWave) void few_tokens_kernel(AdapterArgs p) {
  constexpr int CT = 8, U = 4, P = kParts, kPitch = kStep + 8;
  constexpr int kSize = OUT == HADACORE_FP32 ? 4 : 2;
  __shared__ f4 sums[kFewWaves][kWave];
  __shared__ __attribute__((aligned(16))) float hs[kTile][kTile + 4];
  __shared__ __attribute__((aligned(16))) uint16_t parts[P][kTile][kPitch];
  __shared__ float back[kTile];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int c = lane % kTile, quarter = lane / kTile;
  const int chunk = blockIdx.x % p.chunks;
  const Piece piece = piece_of(p.ends, p.groups, p.m, kTile, blockIdx.x / p.chunks, true);
  if (piece.group < 0) return;
  const bool bare = piece.group == p.groups;  // no adapter
  if (bare && p.y == p.out) return;
  const int count = piece.high - piece.low < kTile ? piece.high - piece.low : kTile;
  const int col = (chunk * kFewWaves + wave) * (kTile * CT) + c * CT;
  const int64_t valid = EVEN ? (col < p.n ? CT : 0) : (int64_t)p.n - col;
  using Row = OutRow<OUT, CT, false>;
  const uint8_t *y = static_cast<const uint8_t *>(p.y);
  uint8_t *out = static_cast<uint8_t *>(p.out);
  int token[4];
  Row old[4];
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const int t = 4 * quarter + v;
    token[v] = token_of(p.slots, piece.low + (t < count ? t : 0), p.m);
    old[v].clear();
    if (y != nullptr && t < count && valid > 0)
      old[v].load(y + (token[v] * p.y_stride + col) * kSize, EVEN ? CT : valid);
  }
  f4 acc[CT] = {};
  if (!bare) {
    uint32_t raw[8][CT / 2];
    const int by = !EVEN && p.n >= CT ? ahead_of<CT>(valid) : 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int row = quarter * 8 + j;
      // ranks and columns that are not there: any values, cleared below or not stored
      const uint16_t *at = p.up + piece.group * p.up_batch + (row < p.rank ? row : 0) * p.up_stride +
                           (EVEN && valid == 0 ? 0 : col);
      if (EVEN || p.n >= CT)
        load_columns<CT>(at - by, CT, raw[j]);
      else
        load_columns<CT>(at, valid, raw[j]);
    }
    const int64_t steps = p.k / kStep;
    const int from = (int)(steps * wave / kFewWaves), to = (int)(steps * (wave + 1) / kFewWaves);
    const int mine = piece.low + (c < count ? c : count - 1);
    const uint16_t *xp = p.x + token_of(p.slots, mine, p.m) * p.x_stride + quarter * 8;
    const uint16_t *wp = p.down + piece.group * p.down_batch +
                         (c < p.rank ? c : p.rank - 1) * p.down_stride + quarter * 8;
    f4 h = f4{0, 0, 0, 0};
    u4 xv[2][U], wv[2][U];
    const auto load = [&](int s, int now) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = (int64_t)(s + u) * kStep;
        xv[now][u] = *reinterpret_cast<const u4_any *>(xp + at);
        wv[now][u] = *reinterpret_cast<const u4_any *>(wp + at);
      }
    };
    const auto multiply = [&](int now) {
#pragma unroll
      for (int u = 0; u < U; ++u) h = mfma<DT>(wv[now][u], xv[now][u], h);
    };
    const int turns = (to - from) / U;
    if (turns > 0) load(from, 0);
    for (int i = 0; i < turns; i += 2) {
      if (i + 1 < turns) load(from + (i + 1) * U, 1);
      multiply(0);
      if (i + 1 >= turns) break;
      if (i + 2 < turns) load(from + (i + 2) * U, 0);
      multiply(1);
    }
    int s = from + turns * U;
    // the rest of k by the last wave
    const int last = to + (wave == kFewWaves - 1 && p.k % kStep != 0);
#pragma unroll 1
    for (; s < last; ++s) {
      const int there = (s < to ? kStep : p.k % kStep) - quarter * 8;
      const uint16_t *wa = wp + (int64_t)s * kStep, *xa = xp + (int64_t)s * kStep;
      if (p.k >= 8) {
        const int back_by = ahead_of<8>(there);
        const u4 wl = *reinterpret_cast<const u4_any *>(wa - back_by);
        const u4 xl = *reinterpret_cast<const u4_any *>(xa - back_by);
        h = mfma<DT>(moved(wl, back_by), moved(xl, back_by), h);
      } else {
        h = mfma<DT>(load8(wa, there), load8(xa, there), h);
      }
    }
    sums[wave][lane] = h;
    __syncthreads();
    if (wave == 0) {
      f4 v = sums[0][lane];
#pragma unroll
      for (int w = 1; w < kFewWaves; ++w) v += sums[w][lane];
      const int rank = 4 * quarter;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (rank + j >= p.rank) v[j] = 0.0f;
      *reinterpret_cast<f4 *>(&hs[c][rank]) = v;
      if (p.hidden != nullptr && chunk == 0 && c < count)
        *reinterpret_cast<f4 *>(p.hidden + (int64_t)(piece.low + c) * p.hidden_stride + rank) = v;
    }
    u4 w[CT];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int i = 0; i < CT / 2; ++i) raw[j][i] = quarter * 8 + j < p.rank ? raw[j][i] : 0;
    if (by > 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) move_values<CT / 2>(raw[j], by);
    }
    turn<CT>(raw, w);
    __syncthreads();
    if (tid < 256) {
      const int t = tid / kTile, q = tid % kTile, r = 4 * q;
      const float scale = p.scales != nullptr ? p.scales[piece.group] : 1.0f;
      f4 v = f4{0, 0, 0, 0};
      if (r < kTile) v = *reinterpret_cast<const f4 *>(&hs[t][r]);
      float most = 0.0f, shift = 1.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] *= scale;
        most = fmaxf(most, fabsf(v[j]));
      }
      if constexpr (DT == HADACORE_FP16) {
        const int e = scale_exponent(max_lanes(most, kTile));
        shift = power_of_two(-e);
        if (q == 0) back[t] = power_of_two(e);
      }
      if (r < kStep) {
        float rest[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) rest[j] = v[j] * shift;
#pragma unroll
        for (int k = 0; k < P; ++k) {
          const uint32_t low = take_parts<DT>(rest[0], rest[1], k);
          *reinterpret_cast<u2 *>(&parts[k][t][r]) = u2{low, take_parts<DT>(rest[2], rest[3], k)};
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = P - 1; k >= 0; --k) {
      const u4 a = *reinterpret_cast<const u4 *>(&parts[k][c][quarter * 8]);
#pragma unroll
      for (int i = 0; i < CT; ++i) acc[i] = mfma<DT>(a, w[i], acc[i]);
    }
  }
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const int t = 4 * quarter + v;
    if (t >= count || valid <= 0) continue;
    if (!bare) {
      const float unshift = DT == HADACORE_FP16 ? back[t] : 1.0f;
      float sum[CT];
#pragma unroll
      for (int i = 0; i < CT; ++i) sum[i] = fmaf(acc[i][v], unshift, old[v].get(i));
      old[v].set(sum);
    }
    old[v].store(out + (token[v] * p.out_stride + col) * kSize, EVEN ? CT : valid);
  }
}

// ---- gradients of the weights -----------------------------------------------------------

struct GradientArgs {
  const float *h;
  const uint16_t *x;
  int64_t h_stride, x_stride;
  const float *scales;
  const int32_t *ends, *slots;
  void *out;
  int64_t out_stride, out_batch;
  float *part;  // sums of each share of a group's tokens: [splits][groups][rank][width]
  int m, width, rank, groups, splits;
};

template <int OUT>
__device__ __forceinline__ void store_value(void *out, int64_t at, float v) {
  if constexpr (OUT == HADACORE_FP32)
    static_cast<float *>(out)[at] = v;
  else
    static_cast<uint16_t *>(out)[at] = narrow<OUT>(v);
}

// A step of 32 tokens of dW[g]: their h (hv: rank c of 16 and tokens 8 quarter + j) times their x
// (raw: the same tokens, 8 columns).  fp16: h is taken times 2^-shift, a power of its own for each rank
// that grows with its values: what is large in one rank, or Inf, takes no bits of the others.
template <int DT, int RT>
__device__ __forceinline__ void gradient_step(const uint32_t (&raw)[8][4], const float (&hv)[RT][8],
                                              int (&shift)[RT], f4 (&acc)[RT][8]) {
  constexpr int P = kParts;
  if constexpr (DT == HADACORE_FP16) {
    int next[RT];
    bool grows = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float most = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(hv[r][j]));
      most = fmaxf(most, __shfl_xor(most, kTile));
      const int e = scale_exponent(fmaxf(most, __shfl_xor(most, 2 * kTile)));
      next[r] = e > shift[r] ? e : shift[r];
      grows |= e > shift[r];
    }
    if (__any(grows)) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const float less = shift[r] - next[r] < -126 ? 0.0f : power_of_two(shift[r] - next[r]);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          // the sums of rank 4 quarter + v
          const float by = __shfl(less, 4 * (threadIdx.x % kWave / kTile) + v);
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[r][i][v] *= by;
        }
        shift[r] = next[r];
      }
    }
  }
  u4 xc[8];
  turn<8>(raw, xc);
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float scale = DT == HADACORE_FP16 ? power_of_two(-shift[r]) : 1.0f;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = hv[r][j] * scale;
    u4 a[P];
#pragma unroll
    for (int k = 0; k < P; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) a[k][j] = take_parts<DT>(v[2 * j], v[2 * j + 1], k);
#pragma unroll
    for (int k = P - 1; k >= 0; --k)
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[r][i] = mfma<DT>(a[k], xc[i], acc[r][i]);
  }
}

// Adds up the W waves' sums and stores them, or leaves them in the workspace.
template <int DT, int OUT, int RT, int W>
__device__ __forceinline__ void store_gradient(const GradientArgs &p, int g, int rank0,
                                               const int (&shift)[RT], const f4 (&acc)[RT][8],
                                               f4 (*sums)[8][kWave + 1]) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const float factor = p.scales != nullptr ? p.scales[g] : 1.0f;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    f4 unshift = f4{1, 1, 1, 1};
    if constexpr (DT == HADACORE_FP16) {
#pragma unroll
      for (int v = 0; v < 4; ++v) unshift[v] = power_of_two(__shfl(shift[r], 4 * (lane / kTile) + v));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[wave][i][lane] = acc[r][i] * unshift;
    __syncthreads();
    // four ranks of a column for each thread in turn
    for (int id = threadIdx.x; id < 4 * kGradColumns; id += W * kWave) {
      const int at = id % kGradColumns, four = id / kGradColumns;  // column: 8 c + i
      const int64_t column = (int64_t)blockIdx.x * kGradColumns + at;
      f4 v = sums[0][at % 8][four * kTile + at / 8];
#pragma unroll
      for (int w = 1; w < W; ++w) v += sums[w][at % 8][four * kTile + at / 8];
      if (column >= p.width) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int rank = rank0 + r * kTile + 4 * four + j;
        if (rank >= p.rank) continue;
        if (p.splits > 1)
          p.part[((int64_t)blockIdx.y * p.rank + rank) * p.width + column] = v[j];
        else
          store_value<OUT>(p.out, g * p.out_batch + rank * p.out_stride + column, factor * v[j]);
      }
    }
  }
}

// dW[g] for 16 RT ranks and 128 columns: the sum over a share of the group's tokens, 32 at a time by
// two waves in turn.  Both operands have the tokens along their depth: x is turned in registers, h
// is split.  Each wave streams its own rows of x and h into a ring in LDS, two steps ahead, and
// their tokens three: no barriers, and few instructions, which are loaded anew by every call
// (8191 x 4096, four adapters of rank 16: 27 us; when it came in, 31 with the loads in registers, a step
// ahead).
template <int DT, int OUT, int RT>
__global__ __launch_bounds__(kGradWaves *kWave) void gradient_kernel(GradientArgs p) {
  constexpr int D = RT == 4 ? 2 : 3;  // stages of the ring: two workgroups to a CU
  constexpr int kX = kStep * kGradColumns * 2, kH = RT * kStep * kTile * 4;
  constexpr int kLoads = 8 + 8 * RT;  // of a step's x and h
  static_assert(kLoads + 1 < 64, "loads in flight that one wait can count");
  constexpr int kRing = D * (kX + kH);
  constexpr int kSums = kGradWaves * 8 * (kWave + 1) * 16;
  __shared__ __attribute__((aligned(16))) uint8_t
      room[kGradWaves * kRing > kSums ? kGradWaves * kRing : kSums];
  __shared__ int32_t token_room[kGradWaves][5][kWave];
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int c = lane % kTile, quarter = lane / kTile;
  const int g = blockIdx.y % p.groups, share = blockIdx.y / p.groups;
  const int rank0 = blockIdx.z * (kTile * RT);
  int col = blockIdx.x * kGradColumns + c * 8;  // a multiple of 8, as the width is
  col = col < p.width ? col : p.width - 8;
  const int low = p.ends != nullptr && g > 0 ? clamp_end(p.ends[g - 1], p.m) : 0;
  const int high = p.ends != nullptr ? clamp_end(p.ends[g], p.m) : p.m;
  const int stride = kStep * kGradWaves * p.splits;
  const int first = low + (share * kGradWaves + wave) * kStep;
  const int steps = first < high ? (high - first + stride - 1) / stride : 0;
  uint8_t *ring = room + wave * kRing;
  // places behind the group's end take its last; they are cleared before the products
  const auto place_of = [&](int i, int t) {
    const int place = first + i * stride + t;
    return place < high ? place : high - 1;
  };
  const auto load_tokens = [&](int i) {
    int32_t *to = &token_room[wave][i & 3][0];
    const int place = place_of(i, lane % kStep);
    if (p.slots != nullptr) {
      load_word_to_lds(p.slots + place, lds_address(to));
    } else {
      to[lane] = place;
      load_word_to_lds(p.h, lds_address(&token_room[wave][4][0]));  // for the count of loads
    }
  };
  const auto load_rows = [&](int i, int stage) {
    uint8_t *to = ring + stage * (kX + kH);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int s = token_room[wave][i & 3][4 * j + quarter];
      const int token = s < 0 ? 0 : s >= p.m ? p.m - 1 : s;
      load_lane_to_lds(p.x + token * p.x_stride + col, lds_address(to + j * 1024));
    }
    // h so that a lane finds its eight tokens' values at its own place
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int row = rank0 + r * kTile + c;
      const float *rank = p.h + (row < p.rank ? row : p.rank - 1);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        load_word_to_lds(rank + place_of(i, 8 * quarter + j) * p.h_stride,
                         lds_address(to + kX + (r * 8 + j) * 256));
    }
  };
  f4 acc[RT][8] = {};
  int shift[RT], stage = 1;
#pragma unroll
  for (int r = 0; r < RT; ++r) shift[r] = -100;
  // Turn i loads the tokens of step i + D and the rows of step i + D - 1, and multiplies step i.
  // In flight before its wait, in order (D = 3): the rows of step i, the tokens of i + 2, the rows of
  // i + 1, the tokens of i + 3; all but the last two have to be there.  (D = 2: the tokens of
  // i + 1, the rows of i, the tokens of i + 2; all but the last.)
#pragma unroll 1
  for (int i = -D; i < steps; ++i) {
    const bool more = i + D < steps;
    if (more) load_tokens(i + D);
    if (i == -D) continue;
    if (more && i == 1 - D) {
      asm volatile("s_waitcnt vmcnt(1)" ::: "memory");
    } else if (more) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 2) * kLoads + 1) : "memory");
    } else if (D > 2 && i > 1 - D && i + 1 < steps) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 2) * kLoads) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    // step i is in `stage`, and step i + D - 1 goes where i - 1 was
    const uint8_t *from = ring + stage * (kX + kH);
    if (i + D - 1 < steps) load_rows(i + D - 1, stage == 0 ? D - 1 : stage - 1);
    stage = stage == D - 1 ? 0 : stage + 1;
    if (i < 0) continue;
    uint32_t raw[8][4];
    float hv[RT][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const u4 v = *reinterpret_cast<const u4 *>(from + (8 * quarter + j) * 256 + c * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) raw[j][e] = v[e];
#pragma unroll
      for (int r = 0; r < RT; ++r)
        hv[r][j] = *reinterpret_cast<const float *>(from + kX + (r * 8 + j) * 256 + lane * 4);
    }
    // the reads have returned before the next loads go to this stage
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    const int s = first + i * stride;
    if (s + kStep > high) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool on = s + 8 * quarter + j < high;
#pragma unroll
        for (int e = 0; e < 4; ++e) raw[j][e] = on ? raw[j][e] : 0;
#pragma unroll
        for (int r = 0; r < RT; ++r) hv[r][j] = on ? hv[r][j] : 0.0f;
      }
    }
    gradient_step<DT, RT>(raw, hv, shift, acc);
  }
  store_gradient<DT, OUT, RT, kGradWaves>(p, g, rank0, shift, acc,
                                          reinterpret_cast<f4(*)[8][kWave + 1]>(room));
}

// The same for rows of x off 16 bytes: loads of any address, in registers, by more waves since nothing
// is loaded ahead.
constexpr int kAnyWaves = 8;

template <int DT, int OUT, int RT>
__global__ __launch_bounds__(kAnyWaves *kWave) void gradient_any_kernel(GradientArgs p) {
  __shared__ f4 sums[kAnyWaves][8][kWave + 1];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c = lane % kTile, quarter = lane / kTile;
  const int g = blockIdx.y % p.groups, share = blockIdx.y / p.groups;
  const int rank0 = blockIdx.z * (kTile * RT);
  const int col = blockIdx.x * kGradColumns + c * 8;
  const int64_t valid = (int64_t)p.width - col;
  const bool wide = p.width >= 8;
  const int by = wide ? ahead_of<8>(valid) : 0;
  const int low = p.ends != nullptr && g > 0 ? clamp_end(p.ends[g - 1], p.m) : 0;
  const int high = p.ends != nullptr ? clamp_end(p.ends[g], p.m) : p.m;
  f4 acc[RT][8] = {};
  int shift[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) shift[r] = -100;
  const int stride = kStep * kAnyWaves * p.splits;
#pragma unroll 1
  for (int64_t s = low + (int64_t)(share * kAnyWaves + wave) * kStep; s < high; s += stride) {
    uint32_t raw[8][4];
    float hv[RT][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool on = s + 8 * quarter + j < high;
      const int at = on ? (int)s + 8 * quarter + j : high - 1;
      const uint16_t *row_of = p.x + token_of(p.slots, at, p.m) * p.x_stride + col;
      if (wide)
        load_columns<8>(row_of - by, 8, raw[j]);
      else
        load_columns<8>(row_of, valid, raw[j]);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const int row = rank0 + r * kTile + c;
        const float v = p.h[at * p.h_stride + (row < p.rank ? row : p.rank - 1)];
        hv[r][j] = on ? v : 0.0f;
      }
    }
    if (by > 0) {
#pragma unroll
      for (int j = 0; j < 8; ++j) move_values<4>(raw[j], by);
    }
    if (s + kStep > high) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) raw[j][e] = s + 8 * quarter + j < high ? raw[j][e] : 0;
    }
    gradient_step<DT, RT>(raw, hv, shift, acc);
  }
  store_gradient<DT, OUT, RT, kAnyWaves>(p, g, rank0, shift, acc, sums);
}

// Four values a thread where rows have whole fours.
template <int OUT, int N>
__global__ __launch_bounds__(256) void join_gradient_kernel(GradientArgs p) {
  const int64_t all = (int64_t)p.groups * p.rank * p.width;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N; i < all; i += (int64_t)gridDim.x * 256 * N) {
    float v[N] = {};
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) {
      if constexpr (N == 4) {
        const f4 more = *reinterpret_cast<const f4 *>(p.part + s * all + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += more[j];
      } else {
        v[0] += p.part[s * all + i];
      }
    }
    const int64_t row = i / p.width;
    const int g = (int)(row / p.rank), rank = (int)(row % p.rank);
    const float factor = p.scales != nullptr ? p.scales[g] : 1.0f;
#pragma unroll
    for (int j = 0; j < N; ++j)
      store_value<OUT>(p.out, g * p.out_batch + rank * p.out_stride + i % p.width + j, factor * v[j]);
  }
}

bool aligned_to(const void *p, uintptr_t bytes) {
  return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
}

template <class F>
void for_type(hadacore_dtype dtype, F f) {
  if (dtype == HADACORE_FP16)
    f(std::integral_constant<int, HADACORE_FP16>{});
  else
    f(std::integral_constant<int, HADACORE_BF16>{});
}

template <int DT>
void launch_down(const AdapterArgs &p, const Cut &cut, hipStream_t stream) {
  const int64_t pieces = most_pieces(p.m, p.groups, 16 * cut.tiles);
  const dim3 grid((uint32_t)pieces, (uint32_t)cut.splits, (uint32_t)divide_up(p.rank, 16 * cut.ranks));
  const auto go = [&](auto tt, auto rt, auto u, auto w) {
    constexpr int W = decltype(w)::value;
    hipLaunchKernelGGL(
        (down_kernel<DT, decltype(tt)::value, decltype(rt)::value, decltype(u)::value, W>), grid,
        dim3(W * kWave), 0, stream, p);
  };
  using std::integral_constant;
  const integral_constant<int, 1> one{};
  const integral_constant<int, 2> two{};
  const integral_constant<int, 4> four{};
  if (cut.tiles == 1) {
    if (cut.ranks == 1)
      go(one, one, four, four);
    else if (cut.ranks == 2)
      go(one, two, four, four);
    else
      go(one, four, two, four);
  } else if (cut.ranks == 1) {
    go(four, one, two, four);
  } else if (cut.ranks == 2) {
    go(four, two, two, four);
  } else {
    go(four, four, two, four);
  }
}

template <int DT, int OUT>
void launch_up(AdapterArgs p, hipStream_t stream) {
  const int64_t pieces = most_pieces(p.m, p.groups, p.unit);
  // EVEN: columns in whole tiles, and rows of y and out from the start of a line
  constexpr int64_t kLine = 128 / (OUT == HADACORE_FP32 ? 4 : 2);
  const bool lines = aligned_to(p.out, 128) && p.out_stride % kLine == 0 &&
                     (p.y == nullptr || (aligned_to(p.y, 128) && p.y_stride % kLine == 0));
  constexpr int kAhead = 2;
  const auto go = [&](auto rb, auto ct) {
    constexpr int RB = decltype(rb)::value, CT = decltype(ct)::value;
    static_assert(CT == 8 || RB == 8, "columns of a workgroup: up_columns");
    const size_t lds = (size_t)up_room(p.unit, p.rank);
    // the columns of a token's row run together: whole rows of y and out, and with as many chunks as
    // XCDs (or a multiple) each of them meets only its own columns of the weights
    p.chunks = p.n > 0 ? (int)divide_up(p.n, 4 * 16 * CT) : 1;  // without columns h is joined
    const dim3 grid((uint32_t)(pieces * p.chunks));
    if (p.n > 0 && p.n % (16 * CT) == 0 && lines)
      hipLaunchKernelGGL((up_kernel<DT, OUT, RB, CT, kAhead, true>), grid, dim3(256), lds, stream, p);
    else
      hipLaunchKernelGGL((up_kernel<DT, OUT, RB, CT, kAhead, false>), grid, dim3(256), lds, stream, p);
  };
  using std::integral_constant;
  const integral_constant<int, 8> eight{};
  const int64_t steps = up_steps(p.rank);
  if (steps == 1)
    go(integral_constant<int, 1>{}, eight);
  else if (steps == 2)
    go(integral_constant<int, 2>{}, eight);
  else if (steps == 4)
    go(integral_constant<int, 4>{}, eight);
  else
    go(eight, integral_constant<int, 4>{});
}

template <int DT, int OUT>
void launch_few(AdapterArgs p, hipStream_t stream) {
  p.chunks = p.n > 0 ? (int)divide_up(p.n, kFewWaves * 128) : 1;
  const dim3 grid((uint32_t)(most_pieces(p.m, p.groups, kTile) * p.chunks));
  if (p.n > 0 && p.n % 128 == 0)
    hipLaunchKernelGGL((few_tokens_kernel<DT, OUT, true>), grid, dim3(kFewWaves * kWave), 0, stream, p);
  else
    hipLaunchKernelGGL((few_tokens_kernel<DT, OUT, false>), grid, dim3(kFewWaves * kWave), 0, stream, p);
}

template <int DT, int OUT>
void launch_gradient(const GradientArgs &p, hipStream_t stream) {
  const int ranks = p.rank <= 16 ? 1 : p.rank <= 32 ? 2 : 4;
  const dim3 grid((uint32_t)divide_up(p.width, kGradColumns), (uint32_t)(p.groups * p.splits),
                  (uint32_t)divide_up(p.rank, 16 * ranks));
  const bool streams = aligned_to(p.x, 16) && p.x_stride % 8 == 0 && p.width % 8 == 0;
  const auto go = [&](auto rt) {
    if (streams)
      hipLaunchKernelGGL((gradient_kernel<DT, OUT, decltype(rt)::value>), grid,
                         dim3(kGradWaves * kWave), 0, stream, p);
    else
      hipLaunchKernelGGL((gradient_any_kernel<DT, OUT, decltype(rt)::value>), grid,
                         dim3(kAnyWaves * kWave), 0, stream, p);
  };
  using std::integral_constant;
  if (ranks == 1)
    go(integral_constant<int, 1>{});
  else if (ranks == 2)
    go(integral_constant<int, 2>{});
  else
    go(integral_constant<int, 4>{});
  if (p.splits > 1) {
    const auto join = [&](auto n) {
      const int64_t blocks = divide_up((int64_t)p.groups * p.rank * p.width, 256 * decltype(n)::value);
      hipLaunchKernelGGL((join_gradient_kernel<OUT, decltype(n)::value>),
                         dim3((uint32_t)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, stream, p);
    };
    if (p.width % 4 == 0)
      join(integral_constant<int, 4>{});
    else
      join(integral_constant<int, 1>{});
  }
}

// ---- arguments -----------------------------------------------------------------------

constexpr int64_t kMaxPitch = int64_t(1) << 26;
constexpr int64_t kMaxBytes = int64_t(1) << 42;
constexpr int64_t kMaxTokens = int64_t(1) << 27;  // a launch stays below 2^32 work-items
constexpr int64_t kMaxWidth = int64_t(1) << 22;

// `batch` matrices of `rows` rows: strides, size, address.
hadacore_status check_matrices(const void *p, int64_t batch, int64_t step, int64_t rows, int64_t pitch,
                               int64_t width, int64_t size) {
  if (pitch < width || pitch > kMaxPitch || (batch > 1 && step < 0))
    return HADACORE_ERROR_INVALID_STRIDE;
  if (batch == 0 || rows == 0 || width == 0) return HADACORE_SUCCESS;
  if (pitch > kMaxBytes / rows || (batch > 1 && step > kMaxBytes / batch))
    return HADACORE_ERROR_TOO_LARGE;
  if (p == nullptr) return HADACORE_ERROR_INVALID_VALUE;
  return aligned_to(p, size) ? HADACORE_SUCCESS : HADACORE_ERROR_MISALIGNED;
}

Span matrices(const void *p, int64_t batch, int64_t step, int64_t rows, int64_t pitch, int64_t width,
              int64_t size) {
  if (p == nullptr || batch == 0) return span(p, 0, 0, 0, 1);
  Span s = span(p, rows, pitch, width, size);
  if (batch > 1 && s.hi > s.lo) s.hi += (uintptr_t)((batch - 1) * step * size);
  return s;
}

Span words(const void *p, int64_t n) { return span(p, p != nullptr, n, n, 4); }

// Groups of tokens: ends, slots and scales.
hadacore_status check_plan(const float *scales, const int32_t *ends, const int32_t *slots,
                           int64_t groups) {
  if (ends == nullptr && groups > 1) return HADACORE_ERROR_INVALID_VALUE;
  if (!aligned_to(ends, 4) || !aligned_to(slots, 4) || !aligned_to(scales, 4))
    return HADACORE_ERROR_MISALIGNED;
  return HADACORE_SUCCESS;
}

hadacore_status check_sizes(int64_t m, int64_t k, int64_t n, int64_t rank, int64_t groups) {
  if (m < 0 || k < 0 || n < 0 || groups < 0) return HADACORE_ERROR_INVALID_VALUE;
  if (rank < 1 || rank > HADACORE_MAX_RANK) return HADACORE_ERROR_INVALID_SIZE;
  if (m >= kMaxTokens || k > kMaxWidth || n > kMaxWidth || groups > HADACORE_MAX_GROUPS)
    return HADACORE_ERROR_TOO_LARGE;
  return HADACORE_SUCCESS;
}

bool is_pair(hadacore_dtype dtype, hadacore_dtype out) {
  return (dtype == HADACORE_FP16 || dtype == HADACORE_BF16) &&
         (out == dtype || out == HADACORE_FP32);
}

}  // namespace
}  // namespace hadacore

using namespace hadacore;

extern "C" int64_t hadacore_adapters_workspace_size(int64_t m, int64_t k, int64_t n, int64_t rank,
                                                    int64_t groups) {
  if (check_sizes(m, k, n, rank, groups) != HADACORE_SUCCESS) return 0;
  const Cut cut = cut_of(m, k, n, rank, groups);
  return cut.fused ? 0 : cut.splits * m * round_up(rank, 16) * 4;
}

extern "C" hadacore_status hadacore_adapters(
    const void *x, int64_t x_row_stride, const void *down, int64_t down_row_stride,
    int64_t down_batch_stride, const void *up, int64_t up_row_stride, int64_t up_batch_stride,
    const float *scales, const int32_t *ends, const int32_t *slots, int64_t groups, const void *y,
    int64_t y_row_stride, void *out, int64_t out_row_stride, hadacore_dtype dtype,
    hadacore_dtype out_dtype, float *hidden, int64_t hidden_row_stride, int64_t m, int64_t k,
    int64_t n, int64_t rank, void *workspace, int64_t workspace_bytes, void *stream) {
  hadacore_status st = check_sizes(m, k, n, rank, groups);
  if (st != HADACORE_SUCCESS) return st;
  if (!is_pair(dtype, out_dtype)) return HADACORE_ERROR_INVALID_DTYPE;
  const int64_t size = out_dtype == HADACORE_FP32 ? 4 : 2, padded = round_up(rank, 16);
  st = check_plan(scales, ends, slots, groups);
  if (st != HADACORE_SUCCESS) return st;
  for (hadacore_status s :
       {check_matrices(x, 1, 0, m, x_row_stride, k, 2),
        check_matrices(down, groups, down_batch_stride, rank, down_row_stride, k, 2),
        check_matrices(up, groups, up_batch_stride, rank, up_row_stride, n, 2),
        check_matrices(out, 1, 0, m, out_row_stride, n, size)})
    if (s != HADACORE_SUCCESS) return s;
  if (y != nullptr) {
    st = check_matrices(y, 1, 0, m, y_row_stride, n, size);
    if (st != HADACORE_SUCCESS) return st;
  }
  if (hidden != nullptr) {
    if (hidden_row_stride < padded || hidden_row_stride % 4 != 0 || hidden_row_stride > kMaxPitch)
      return HADACORE_ERROR_INVALID_STRIDE;
    if (!aligned_to(hidden, 16)) return HADACORE_ERROR_MISALIGNED;
  }
  if (m == 0) return HADACORE_SUCCESS;
  const int64_t need = hadacore_adapters_workspace_size(m, k, n, rank, groups);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return HADACORE_ERROR_WORKSPACE;
  if (!aligned_to(workspace, 16)) return HADACORE_ERROR_MISALIGNED;
  const Span so = matrices(out, 1, 0, m, out_row_stride, n, size),
             sh = matrices(hidden, 1, 0, m, hidden_row_stride, padded, 4),
             sw = span(workspace, need > 0, need, need, 1),
             sy = matrices(y, 1, 0, m, y_row_stride, n, size);
  const Span in[] = {matrices(x, 1, 0, m, x_row_stride, k, 2),
                     matrices(down, groups, down_batch_stride, rank, down_row_stride, k, 2),
                     matrices(up, groups, up_batch_stride, rank, up_row_stride, n, 2),
                     words(scales, groups),
                     words(ends, groups),
                     words(slots, m)};
  for (const Span &s : in)
    if (spans_overlap(so, s) || spans_overlap(sh, s) || spans_overlap(sw, s))
      return HADACORE_ERROR_OVERLAP;
  if (spans_overlap(so, sh) || spans_overlap(so, sw) || spans_overlap(sh, sw) ||
      spans_overlap(sy, sh) || spans_overlap(sy, sw) ||
      (spans_overlap(so, sy) && !(out == y && (out_row_stride == y_row_stride || m == 1))))
    return HADACORE_ERROR_OVERLAP;
  const Cut cut = cut_of(m, k, n, rank, groups);
  // up_kernel's launch, the largest
  if (!cut.fused && most_pieces(m, groups, cut.unit) * divide_up(n, up_columns(rank)) * 256 >=
                        (int64_t(1) << 32))
    return HADACORE_ERROR_TOO_LARGE;
  st = check_device();
  if (st != HADACORE_SUCCESS) return st;
  AdapterArgs p{};
  p.x = static_cast<const uint16_t *>(x);
  p.x_stride = x_row_stride;
  p.down = static_cast<const uint16_t *>(down);
  p.down_stride = down_row_stride;
  p.down_batch = down_batch_stride;
  p.up = static_cast<const uint16_t *>(up);
  p.up_stride = up_row_stride;
  p.up_batch = up_batch_stride;
  p.scales = scales;
  p.ends = ends;
  p.slots = slots;
  p.y = y;
  p.y_stride = y_row_stride;
  p.out = out;
  p.out_stride = out_row_stride;
  p.splits = cut.splits;
  p.unit = cut.unit;
  p.hidden = hidden;
  p.hidden_stride = hidden_row_stride;
  const bool direct = hidden != nullptr && cut.splits == 1;
  p.part = direct ? hidden : static_cast<float *>(workspace);
  p.part_pitch = direct ? hidden_row_stride : padded;
  p.part_step = m * padded;
  p.m = (int)m;
  p.k = (int)k;
  p.n = (int)n;
  p.rank = (int)rank;
  p.padded = (int)padded;
  p.groups = (int)groups;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (n == 0 && (hidden == nullptr || groups == 0)) return HADACORE_SUCCESS;
  if (cut.fused) {
    for_type(dtype, [&](auto dt) {
      constexpr int DT = decltype(dt)::value;
      if (out_dtype == HADACORE_FP32)
        launch_few<DT, HADACORE_FP32>(p, s);
      else
        launch_few<DT, DT>(p, s);
    });
    return hipGetLastError() == hipSuccess ? HADACORE_SUCCESS : HADACORE_ERROR_LAUNCH;
  }
  if (groups > 0) {
    for_type(dtype, [&](auto dt) { launch_down<decltype(dt)::value>(p, cut, s); });
    if (hipGetLastError() != hipSuccess) return HADACORE_ERROR_LAUNCH;
  }
  if (n == 0 && direct) return HADACORE_SUCCESS;
  for_type(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    if (out_dtype == HADACORE_FP32)
      launch_up<DT, HADACORE_FP32>(p, s);
    else
      launch_up<DT, DT>(p, s);
  });
  return hipGetLastError() == hipSuccess ? HADACORE_SUCCESS : HADACORE_ERROR_LAUNCH;
}

extern "C" int64_t hadacore_adapter_gradient_workspace_size(int64_t m, int64_t width, int64_t rank,
                                                            int64_t groups) {
  if (check_sizes(m, width, 0, rank, groups) != HADACORE_SUCCESS) return 0;
  const int64_t splits = gradient_splits(m, width, rank, groups);
  return splits > 1 ? splits * groups * rank * width * 4 : 0;
}

extern "C" hadacore_status hadacore_adapter_gradient(
    const float *hidden, int64_t hidden_row_stride, const void *x, int64_t x_row_stride,
    hadacore_dtype dtype, const float *scales, const int32_t *ends, const int32_t *slots,
    int64_t groups, void *out, int64_t out_row_stride, int64_t out_batch_stride,
    hadacore_dtype out_dtype, int64_t m, int64_t width, int64_t rank, void *workspace,
    int64_t workspace_bytes, void *stream) {
  hadacore_status st = check_sizes(m, width, 0, rank, groups);
  if (st != HADACORE_SUCCESS) return st;
  if (!is_pair(dtype, out_dtype)) return HADACORE_ERROR_INVALID_DTYPE;
  st = check_plan(scales, ends, slots, groups);
  if (st != HADACORE_SUCCESS) return st;
  const int64_t size = out_dtype == HADACORE_FP32 ? 4 : 2;
  for (hadacore_status s :
       {check_matrices(hidden, 1, 0, m, hidden_row_stride, rank, 4),
        check_matrices(x, 1, 0, m, x_row_stride, width, 2),
        check_matrices(out, groups, out_batch_stride, rank, out_row_stride, width, size)})
    if (s != HADACORE_SUCCESS) return s;
  if (groups > 1 && out_batch_stride < (rank - 1) * out_row_stride + width)
    return HADACORE_ERROR_INVALID_STRIDE;
  if (groups == 0 || width == 0) return HADACORE_SUCCESS;
  const int64_t need = hadacore_adapter_gradient_workspace_size(m, width, rank, groups);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return HADACORE_ERROR_WORKSPACE;
  if (!aligned_to(workspace, 16)) return HADACORE_ERROR_MISALIGNED;
  const Span so = matrices(out, groups, out_batch_stride, rank, out_row_stride, width, size),
             sw = span(workspace, need > 0, need, need, 1);
  const Span in[] = {matrices(hidden, 1, 0, m, hidden_row_stride, rank, 4),
                     matrices(x, 1, 0, m, x_row_stride, width, 2), words(scales, groups),
                     words(ends, groups), words(slots, m)};
  for (const Span &s : in)
    if (spans_overlap(so, s) || spans_overlap(sw, s)) return HADACORE_ERROR_OVERLAP;
  if (spans_overlap(so, sw)) return HADACORE_ERROR_OVERLAP;
  st = check_device();
  if (st != HADACORE_SUCCESS) return st;
  GradientArgs p{};
  p.h = hidden;
  p.h_stride = hidden_row_stride;
  p.x = static_cast<const uint16_t *>(x);
  p.x_stride = x_row_stride;
  p.scales = scales;
  p.ends = ends;
  p.slots = slots;
  p.out = out;
  p.out_stride = out_row_stride;
  p.out_batch = out_batch_stride;
  p.part = static_cast<float *>(workspace);
  p.m = (int)m;
  p.width = (int)width;
  p.rank = (int)rank;
  p.groups = (int)groups;
  p.splits = (int)gradient_splits(m, width, rank, groups);
  for_type(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    if (out_dtype == HADACORE_FP32)
      launch_gradient<DT, HADACORE_FP32>(p, static_cast<hipStream_t>(stream));
    else
      launch_gradient<DT, DT>(p, static_cast<hipStream_t>(stream));
  });
  return hipGetLastError() == hipSuccess ? HADACORE_SUCCESS : HADACORE_ERROR_LAUNCH;
}
