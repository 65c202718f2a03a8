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
// in parts of 16 bits that add up to it.  Two parts of bf16 keep 16 bits of h, which a 16-bit
// result cannot tell from all (2^-17 against 2^-9); for a 32-bit result three parts keep all 24.
// fp16 parts are made of h times a power of two (largest value of the row near 2^10), so
// that they keep 22 bits whatever h's size.  A value of h, a weight or an x that is Inf gives a NaN
// where the sum without parts may give Inf: Inf times a part of 0 is NaN.

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "groups.h"
#include "hadacore.h"
#include "internal.h"

namespace hadacore {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef u4 u4_any __attribute__((aligned(2)));
typedef u2 u2_any __attribute__((aligned(2)));
typedef u4 u4_words __attribute__((aligned(4)));

constexpr int kTile = 16;   // rows and columns of a matrix product
constexpr int kStep = 32;   // its depth

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

// v as a sum of P values of 16 bits.  Parts of bf16 but the last are cut off, so that a NaN stays
// one (what is left of it is a quiet NaN) and no part rounds up to Inf.
template <int DT, int P>
__device__ __forceinline__ void split(float v, uint16_t (&part)[P]) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if constexpr (DT == HADACORE_FP16) {
      part[i] = narrow<DT>(v);
    } else {
      part[i] = i < P - 1 ? (uint16_t)(__builtin_bit_cast(uint32_t, v) >> 16) : narrow<DT>(v);
    }
    v -= widen<DT>(part[i]);
  }
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

// Sum, or maximum, over the lanes of a wave in steps of xor.
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
  int m, k, n, rank, padded, groups, splits, unit;  // padded: the rank in whole tiles
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

// h for 16 TT tokens of a group, 16 RT of its ranks and one of `splits` shares of k.  Four waves
// take a quarter of the share each and add up at the end, so that each value of x and of
// the weights is loaded by one wave, straight into the operands of the matrix products: both
// have k along their rows.  U steps of k are loaded ahead of the U being multiplied.
template <int DT, int TT, int RT, int U>
__global__ __launch_bounds__(256) void down_kernel(AdapterArgs p) {
  constexpr int kWaves = 4;
  __shared__ f4 sums[kWaves][TT * RT][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c = lane % kTile, quarter = lane / kTile;
  const Piece piece = piece_of(p.ends, p.groups, p.m, kTile * TT, blockIdx.x, false);
  if (piece.group < 0) return;
  const int rank0 = blockIdx.z * (kTile * RT);
  const uint16_t *xp[TT], *wp[RT];
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    const int place = piece.low + t * kTile + c;
    xp[t] = p.x + token_of(p.slots, place < piece.high ? place : piece.high - 1, p.m) * p.x_stride +
            quarter * 8;
  }
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = rank0 + r * kTile + c;
    wp[r] = p.down + piece.group * p.down_batch + (row < p.rank ? row : p.rank - 1) * p.down_stride +
            quarter * 8;
  }
  const int64_t steps = ((int64_t)p.k + kStep - 1) / kStep;
  const int shares = p.splits * kWaves, share = blockIdx.y * kWaves + wave;
  const int from = (int)(steps * share / shares), to = (int)(steps * (share + 1) / shares);
  f4 acc[TT][RT] = {};
  u4 xv[2][U][TT], wv[2][U][RT];
  const auto load = [&](int s0, int buffer) {
    if (s0 + U <= to && (s0 + U) * kStep <= p.k) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = (s0 + u) * kStep;
#pragma unroll
        for (int t = 0; t < TT; ++t) xv[buffer][u][t] = *reinterpret_cast<const u4_any *>(xp[t] + at);
#pragma unroll
        for (int r = 0; r < RT; ++r) wv[buffer][u][r] = *reinterpret_cast<const u4_any *>(wp[r] + at);
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = (s0 + u) * kStep;
        const int valid = s0 + u < to ? p.k - at - quarter * 8 : 0;
#pragma unroll
        for (int t = 0; t < TT; ++t) xv[buffer][u][t] = load8(xp[t] + at, valid);
#pragma unroll
        for (int r = 0; r < RT; ++r) wv[buffer][u][r] = load8(wp[r] + at, valid);
      }
    }
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
  if (from < to) load(from, 0);
  for (int s = from; s < to; s += 2 * U) {
    if (s + U < to) load(s + U, 1);
    multiply(0);
    if (s + U >= to) break;
    if (s + 2 * U < to) load(s + 2 * U, 0);
    multiply(1);
  }
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) sums[wave][t * RT + r][lane] = acc[t][r];
  __syncthreads();
  for (int i = wave; i < TT * RT; i += kWaves) {
    f4 v = sums[0][i][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += sums[w][i][lane];
    const int place = piece.low + i / RT * kTile + c;
    const int rank = rank0 + i % RT * kTile + 4 * quarter;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (rank + j >= p.rank) v[j] = 0.0f;
    if (place < piece.high && rank < p.padded)
      *reinterpret_cast<f4 *>(p.part + blockIdx.y * p.part_step + place * p.part_pitch + rank) = v;
  }
}

// out for up to `unit` tokens of a group and 4 * 16 CT columns.  A wave keeps the weights of its
// 16 CT columns in registers for all these tokens: 8 rows of CT columns a lane, turned in
// registers so that the ranks lie along an operand.  A lane then has CT consecutive columns of each
// of four tokens, which it loads and stores whole.  h, joined and split, goes through LDS.
// Tokens behind the last end get y.
template <int DT, int OUT, int RB, int CT, int P>
__global__ __launch_bounds__(256) void up_kernel(AdapterArgs p) {
  constexpr int kPitch = kStep * RB + 8;
  extern __shared__ __attribute__((aligned(16))) uint8_t room[];
  uint16_t *parts = reinterpret_cast<uint16_t *>(room);  // [P][unit][kPitch]
  float *back = reinterpret_cast<float *>(parts + P * p.unit * kPitch);
  int *tokens = reinterpret_cast<int *>(back + p.unit);
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int c = lane % kTile, quarter = lane / kTile;
  const Piece piece = piece_of(p.ends, p.groups, p.m, p.unit, blockIdx.x, true);
  if (piece.group < 0) return;
  const bool bare = piece.group == p.groups;  // no adapter
  if (bare && p.y == p.out) return;
  const int count = piece.high - piece.low < p.unit ? piece.high - piece.low : p.unit;
  const int col = (blockIdx.y * 4 + wave) * (kTile * CT) + c * CT;
  const int64_t valid = (int64_t)p.n - col;
  u4 w[RB][CT];
  if (!bare) {
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      uint32_t raw[8][CT / 2];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int row = b * kStep + quarter * 8 + j;
        load_columns<CT>(p.up + piece.group * p.up_batch + (row < p.rank ? row : 0) * p.up_stride + col,
                         row < p.rank ? valid : 0, raw[j]);
      }
      turn<CT>(raw, w[b]);
    }
  }
  for (int t0 = 0; t0 < count; t0 += 256 / kTile) {
    const int t = t0 + tid / kTile, q = tid % kTile;
    if (t >= count) continue;
    const int place = piece.low + t;
    if (q == 0) tokens[t] = token_of(p.slots, place, p.m);
    if (bare) continue;
    const float scale = p.scales != nullptr ? p.scales[piece.group] : 1.0f;
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
        for (int s = 1; s < p.splits; ++s) v += *reinterpret_cast<const f4 *>(at + s * p.part_step);
        if (p.hidden != nullptr && p.splits > 1 && blockIdx.y == 0)
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
      uint16_t v[4][P];
#pragma unroll
      for (int j = 0; j < 4; ++j) split<DT, P>(h[i][j] * shift, v[j]);
#pragma unroll
      for (int k = 0; k < P; ++k)
        *reinterpret_cast<u2 *>(parts + (k * p.unit + t) * kPitch + r) =
            u2{v[0][k] | (uint32_t)v[1][k] << 16, v[2][k] | (uint32_t)v[3][k] << 16};
    }
  }
  __syncthreads();
  // whole waves only: a matrix instruction reads the registers of all 64 lanes
  if ((blockIdx.y * 4 + wave) * (kTile * CT) >= p.n) return;
  using T = std::conditional_t<OUT == HADACORE_FP32, float, uint16_t>;
  struct __attribute__((packed, aligned(sizeof(T)))) Row {
    T v[CT];
  };
  const T *y = static_cast<const T *>(p.y);
  T *out = static_cast<T *>(p.out);
  const auto value = [](T v) {
    if constexpr (OUT == HADACORE_FP32)
      return v;
    else
      return widen<OUT>(v);
  };
  for (int t0 = 0; t0 < count; t0 += kTile) {
    const int mine = t0 + 4 * quarter;
    T old[4][CT];
    int token[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      token[v] = tokens[mine + v < count ? mine + v : t0];
#pragma unroll
      for (int i = 0; i < CT; ++i) old[v][i] = 0;
      if (y != nullptr && mine + v < count) {
        const T *from = y + token[v] * p.y_stride + col;
        if (valid >= CT) {  // (fewer, or none: value by value)
          const Row raw = *reinterpret_cast<const Row *>(from);
#pragma unroll
          for (int i = 0; i < CT; ++i) old[v][i] = raw.v[i];
        } else {
#pragma unroll
          for (int i = 0; i < CT; ++i)
            if (i < valid) old[v][i] = from[i];
        }
      }
    }
    f4 acc[CT] = {};
    if (!bare) {
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int k = P - 1; k >= 0; --k) {
          const u4 a = *reinterpret_cast<const u4 *>(
              parts + (k * p.unit + t0 + c) * kPitch + b * kStep + quarter * 8);
#pragma unroll
          for (int i = 0; i < CT; ++i) acc[i] = mfma<DT>(a, w[b][i], acc[i]);
        }
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if (mine + v >= count) continue;
      const float unshift = DT == HADACORE_FP16 && !bare ? back[mine + v] : 1.0f;
      T *to = out + token[v] * p.out_stride + col;
      Row row;
#pragma unroll
      for (int i = 0; i < CT; ++i) {
        const float sum = fmaf(acc[i][v], unshift, value(old[v][i]));
        if constexpr (OUT == HADACORE_FP32)
          row.v[i] = sum;
        else
          row.v[i] = narrow<OUT>(sum);
      }
      if (valid >= CT) {
        *reinterpret_cast<Row *>(to) = row;
      } else {
#pragma unroll
        for (int i = 0; i < CT; ++i)
          if (i < valid) to[i] = row.v[i];
      }
    }
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

constexpr int kGradWaves = 8;
constexpr int kGradColumns = kTile * 8;

// dW[g] for 16 RT ranks and 128 columns: the sum over a share of the group's tokens, 32 at a time by
// eight waves in turn.  Both operands have the tokens along their depth: x is turned in registers, h
// is read as it lies and split.
template <int DT, int OUT, int RT, int P>
__global__ __launch_bounds__(kGradWaves *kWave) void gradient_kernel(GradientArgs p) {
  __shared__ f4 sums[kGradWaves][8][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c = lane % kTile, quarter = lane / kTile;
  const int g = blockIdx.y % p.groups, share = blockIdx.y / p.groups;
  const int rank0 = blockIdx.z * (kTile * RT);
  const int col = blockIdx.x * kGradColumns + c * 8;
  const int64_t valid = (int64_t)p.width - col;
  const int low = p.ends != nullptr && g > 0 ? clamp_end(p.ends[g - 1], p.m) : 0;
  const int high = p.ends != nullptr ? clamp_end(p.ends[g], p.m) : p.m;
  f4 acc[RT][8] = {};
  int shift = -100;  // fp16: h is taken times 2^-shift
  const int stride = kStep * kGradWaves * p.splits;
  for (int64_t s = low + (int64_t)(share * kGradWaves + wave) * kStep; s < high; s += stride) {
    const int place = (int)s + 8 * quarter;
    uint32_t raw[8][4];
    float hv[RT][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool on = place + j < high;
      const int at = on ? place + j : high - 1;
      load_columns<8>(p.x + token_of(p.slots, at, p.m) * p.x_stride + col, on ? valid : 0, raw[j]);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const int row = rank0 + r * kTile + c;
        const float v = p.h[at * p.h_stride + (row < p.rank ? row : p.rank - 1)];
        hv[r][j] = on ? v : 0.0f;
      }
    }
    float scale = 1.0f;
    if constexpr (DT == HADACORE_FP16) {
      float most = 0.0f;
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(hv[r][j]));
      const int e = scale_exponent(max_lanes(most, kWave));
      if (e > shift) {
        const float less = shift - e < -126 ? 0.0f : power_of_two(shift - e);
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[r][i] *= less;
        shift = e;
      }
      scale = power_of_two(-shift);
    }
    u4 xc[8];
    turn<8>(raw, xc);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      uint16_t v[8][P];
#pragma unroll
      for (int j = 0; j < 8; ++j) split<DT, P>(hv[r][j] * scale, v[j]);
#pragma unroll
      for (int k = P - 1; k >= 0; --k) {
        u4 a;
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = v[2 * j][k] | (uint32_t)v[2 * j + 1][k] << 16;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[r][i] = mfma<DT>(a, xc[i], acc[r][i]);
      }
    }
  }
  const float unshift = DT == HADACORE_FP16 ? power_of_two(shift) : 1.0f;
  const float factor = p.scales != nullptr ? p.scales[g] : 1.0f;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    if (r > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[wave][i][lane] = acc[r][i] * unshift;
    __syncthreads();
    // wave w: rank w and w + 8 of the 16, 128 columns as two of a lane
    for (int half = 0; half < 2; ++half) {
      const int in_tile = wave + half * 8, rank = rank0 + r * kTile + in_tile;
      if (rank >= p.rank) continue;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int at = lane + e * kWave;  // column: 8 c + i
        if (blockIdx.x * kGradColumns + at >= p.width) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kGradWaves; ++w)
          v += sums[w][at % 8][in_tile / 4 * kTile + at / 8][in_tile % 4];
        const int64_t column = (int64_t)blockIdx.x * kGradColumns + at;
        if (p.splits > 1)
          p.part[((int64_t)blockIdx.y * p.rank + rank) * p.width + column] = v;
        else
          store_value<OUT>(p.out, g * p.out_batch + rank * p.out_stride + column, factor * v);
      }
    }
  }
}

template <int OUT>
__global__ __launch_bounds__(256) void join_gradient_kernel(GradientArgs p) {
  const int64_t all = (int64_t)p.groups * p.rank * p.width;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    float v = 0.0f;
    for (int s = 0; s < p.splits; ++s) v += p.part[s * all + i];
    const int64_t row = i / p.width;
    const int g = (int)(row / p.rank), rank = (int)(row % p.rank);
    const float factor = p.scales != nullptr ? p.scales[g] : 1.0f;
    store_value<OUT>(p.out, g * p.out_batch + rank * p.out_stride + i % p.width, factor * v);
  }
}

// ---- how a call is cut ---------------------------------------------------------------

constexpr int64_t kBlocksWanted = 512;  // two workgroups to a CU of a whole card

int64_t round_up(int64_t v, int64_t unit) { return (v + unit - 1) / unit * unit; }
int64_t divide_up(int64_t v, int64_t by) { return (v + by - 1) / by; }

// Pieces of `unit` rows that `groups` groups of m rows can have at most.
int64_t most_pieces(int64_t m, int64_t groups, int64_t unit) {
  return m / unit + (groups < m ? groups : m) + 1;
}

struct Cut {
  int ranks;   // tiles of ranks in a workgroup of down_kernel
  int tiles;   // tiles of tokens there
  int splits;  // shares of k
  int unit;    // tokens of a workgroup of up_kernel
};

Cut cut_of(int64_t m, int64_t k, int64_t n, int64_t rank, int64_t groups, int parts) {
  Cut cut{};
  cut.ranks = rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8;
  const int64_t live = groups < 1 || m < 1 ? 1 : groups < m ? groups : m;
  const bool few = m <= 32 * live;
  cut.tiles = few ? 1 : cut.ranks == 8 ? 2 : 4;
  const int64_t blocks =
      (divide_up(m, 16 * cut.tiles) + live - 1) * divide_up(rank, 16 * cut.ranks);
  int64_t splits = divide_up(kBlocksWanted, blocks < 1 ? 1 : blocks);
  const int64_t most = k / 512;  // four steps of k for a wave at least
  splits = splits > most ? most : splits;
  cut.splits = (int)(splits < 1 ? 1 : splits > 16 ? 16 : splits);
  const int64_t depth = round_up(rank, kStep), columns = divide_up(n, rank > 128 ? 256 : 512);
  cut.unit = 16;
  while (cut.unit < 128 && !few && 2 * cut.unit * (depth + 8) * 2 * parts <= 48 * 1024 &&
         m / (2 * cut.unit) * columns >= 2 * kBlocksWanted)
    cut.unit *= 2;
  return cut;
}

int64_t gradient_splits(int64_t m, int64_t width, int64_t rank, int64_t groups) {
  if (groups < 1 || width < 1) return 1;
  const int64_t blocks = divide_up(width, kGradColumns) * groups * divide_up(rank, 64);
  int64_t splits = divide_up(kBlocksWanted, blocks);
  // a workgroup goes through 256 tokens in a turn; a share has two turns at least
  const int64_t most = m / groups / (2 * kStep * kGradWaves);
  splits = splits > most ? most : splits;
  return splits < 1 ? 1 : splits > 16 ? 16 : splits;
}

template <class F>
void for_type(hadacore_dtype dtype, F f) {
  if (dtype == HADACORE_FP16)
    f(std::integral_constant<int, HADACORE_FP16>{});
  else
    f(std::integral_constant<int, HADACORE_BF16>{});
}

// Parts of h: see the top of the file.
constexpr int parts_of(int dtype, int out) {
  return dtype == HADACORE_BF16 && out == HADACORE_FP32 ? 3 : 2;
}

template <int DT>
void launch_down(const AdapterArgs &p, const Cut &cut, hipStream_t stream) {
  const int64_t pieces = most_pieces(p.m, p.groups, 16 * cut.tiles);
  const dim3 grid((uint32_t)pieces, (uint32_t)cut.splits, (uint32_t)divide_up(p.rank, 16 * cut.ranks));
  const auto go = [&](auto tt, auto rt, auto u) {
    hipLaunchKernelGGL((down_kernel<DT, decltype(tt)::value, decltype(rt)::value, decltype(u)::value>),
                       grid, dim3(256), 0, stream, p);
  };
  using std::integral_constant;
  const integral_constant<int, 1> one{};
  const integral_constant<int, 2> two{};
  const integral_constant<int, 4> four{};
  const integral_constant<int, 8> eight{};
  if (cut.tiles == 1) {
    if (cut.ranks == 1)
      go(one, one, four);
    else if (cut.ranks == 2)
      go(one, two, four);
    else if (cut.ranks == 4)
      go(one, four, two);
    else
      go(one, eight, two);
  } else if (cut.ranks == 1) {
    go(four, one, two);
  } else if (cut.ranks == 2) {
    go(four, two, two);
  } else if (cut.ranks == 4) {
    go(four, four, one);
  } else {
    go(two, eight, one);
  }
}

template <int DT, int OUT>
void launch_up(const AdapterArgs &p, hipStream_t stream) {
  constexpr int P = parts_of(DT, OUT);
  const int64_t pieces = most_pieces(p.m, p.groups, p.unit);
  const auto go = [&](auto rb, auto ct) {
    constexpr int RB = decltype(rb)::value, CT = decltype(ct)::value;
    const size_t lds = (size_t)p.unit * (P * (kStep * RB + 8) * 2 + 8);
    const int64_t columns = divide_up(p.n, 4 * 16 * CT);  // 0: h is joined all the same
    hipLaunchKernelGGL((up_kernel<DT, OUT, RB, CT, P>),
                       dim3((uint32_t)pieces, (uint32_t)(columns > 0 ? columns : 1)), dim3(256), lds,
                       stream, p);
  };
  using std::integral_constant;
  const integral_constant<int, 8> eight{};
  if (p.rank <= 32)
    go(integral_constant<int, 1>{}, eight);
  else if (p.rank <= 64)
    go(integral_constant<int, 2>{}, eight);
  else if (p.rank <= 128)
    go(integral_constant<int, 4>{}, eight);
  else
    go(eight, integral_constant<int, 4>{});
}

template <int DT, int OUT>
void launch_gradient(const GradientArgs &p, hipStream_t stream) {
  constexpr int P = parts_of(DT, OUT);
  const int ranks = p.rank <= 16 ? 1 : p.rank <= 32 ? 2 : 4;
  const dim3 grid((uint32_t)divide_up(p.width, kGradColumns), (uint32_t)(p.groups * p.splits),
                  (uint32_t)divide_up(p.rank, 16 * ranks));
  const auto go = [&](auto rt) {
    hipLaunchKernelGGL((gradient_kernel<DT, OUT, decltype(rt)::value, P>), grid,
                       dim3(kGradWaves * kWave), 0, stream, p);
  };
  using std::integral_constant;
  if (ranks == 1)
    go(integral_constant<int, 1>{});
  else if (ranks == 2)
    go(integral_constant<int, 2>{});
  else
    go(integral_constant<int, 4>{});
  if (p.splits > 1) {
    const int64_t blocks = divide_up((int64_t)p.groups * p.rank * p.width, 256);
    hipLaunchKernelGGL(join_gradient_kernel<OUT>, dim3((uint32_t)(blocks < 4096 ? blocks : 4096)),
                       dim3(256), 0, stream, p);
  }
}

// ---- arguments -----------------------------------------------------------------------

constexpr int64_t kMaxPitch = int64_t(1) << 26;
constexpr int64_t kMaxBytes = int64_t(1) << 42;
constexpr int64_t kMaxTokens = int64_t(1) << 27;  // a launch stays below 2^32 work-items
constexpr int64_t kMaxWidth = int64_t(1) << 22;

bool aligned_to(const void *p, uintptr_t bytes) {
  return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
}

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
  const int64_t splits = cut_of(m, k, n, rank, groups, 2).splits;
  return splits * m * round_up(rank, 16) * 4;
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
  if (workspace == nullptr || workspace_bytes < need) return HADACORE_ERROR_WORKSPACE;
  if (!aligned_to(workspace, 16)) return HADACORE_ERROR_MISALIGNED;
  const Span so = matrices(out, 1, 0, m, out_row_stride, n, size),
             sh = matrices(hidden, 1, 0, m, hidden_row_stride, padded, 4),
             sw = span(workspace, 1, need, need, 1), sy = matrices(y, 1, 0, m, y_row_stride, n, size);
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
  st = check_device();
  if (st != HADACORE_SUCCESS) return st;
  const Cut cut = cut_of(m, k, n, rank, groups, parts_of(dtype, out_dtype));
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
  if (groups > 0) {
    for_type(dtype, [&](auto dt) { launch_down<decltype(dt)::value>(p, cut, s); });
    if (hipGetLastError() != hipSuccess) return HADACORE_ERROR_LAUNCH;
  }
  if (n == 0 && (hidden == nullptr || direct)) return HADACORE_SUCCESS;
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
  if (!aligned_to(workspace, 4)) return HADACORE_ERROR_MISALIGNED;
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
