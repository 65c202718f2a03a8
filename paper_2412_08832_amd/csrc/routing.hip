// routing.hip -- from a router's logits to rows sorted by expert, and back.
//
//   route     the k experts of each token with their weights, how many tokens each expert
//             got, the balance loss; its gradient
//   group     the stable order of (token, choice) slots by group: ends, places, slots
//   dispatch  rows of tokens copied to the places of their slots
//   combine   the rows of a token's slots joined by weight; its gradient
//
// All of it moves few bytes (or each byte once): what bounds the large calls is HBM, and the small
// ones their launches, so every call is one launch where a workgroup can do it and two otherwise.
// No result depends on the order of atomics: they count in LDS, or find the last of the workgroups
// that join the balance loss, which adds up the others' parts in their order.

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

constexpr int kMaxChoices = HADACORE_MAX_CHOICES;
constexpr int kMaxExperts = HADACORE_MAX_EXPERTS;

template <int DT>
struct Stored {
  using type = uint16_t;
};
template <>
struct Stored<HADACORE_FP32> {
  using type = float;
};

template <int DT>
__device__ __forceinline__ float widen(typename Stored<DT>::type h) {
  if constexpr (DT == HADACORE_FP32)
    return h;
  else if constexpr (DT == HADACORE_FP16)
    return (float)__builtin_bit_cast(_Float16, h);
  else
    return __builtin_bit_cast(float, (uint32_t)h << 16);
}

// One rounding, to nearest even.
template <int DT>
__device__ __forceinline__ typename Stored<DT>::type narrow(float v) {
  if constexpr (DT == HADACORE_FP32)
    return v;
  else if constexpr (DT == HADACORE_FP16)
    return __builtin_bit_cast(uint16_t, (_Float16)v);
  else
    return __builtin_bit_cast(uint16_t, (__bf16)v);
}

// N consecutive values of a row.  Rows may start at any value's address; the hardware takes wide loads
// and stores from there.  NT: with the streaming policy, for data that is touched once and more
// than the caches keep.
template <int DT, int N>
struct Values {
  using T = typename Stored<DT>::type;
  struct Raw {
    T v[N];
  };
  typedef uint32_t Words __attribute__((ext_vector_type(sizeof(Raw) / 4)));
  typedef Words Words_any __attribute__((aligned(sizeof(T))));
  Raw raw;

  // the first `valid` of them; zeros behind
  template <bool NT = false>
  __device__ __forceinline__ void load(const T *p, int valid) {
    if (valid >= N) {
      if constexpr (NT)
        raw = __builtin_bit_cast(Raw, __builtin_nontemporal_load(reinterpret_cast<const Words_any *>(p)));
      else
        raw = __builtin_bit_cast(Raw, *reinterpret_cast<const Words_any *>(p));
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) raw.v[i] = i < valid ? p[i] : T(0);
    }
  }
  template <bool NT = false>
  __device__ __forceinline__ void store(T *p, int valid) const {
    if (valid >= N) {
      if constexpr (NT)
        __builtin_nontemporal_store(__builtin_bit_cast(Words, raw), reinterpret_cast<Words_any *>(p));
      else
        *reinterpret_cast<Words_any *>(p) = __builtin_bit_cast(Words, raw);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < valid) p[i] = raw.v[i];
    }
  }
  __device__ __forceinline__ float get(int i) const { return widen<DT>(raw.v[i]); }
  __device__ __forceinline__ void set(const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) raw.v[i] = narrow<DT>(v[i]);
  }
};

template <int DT, int N>
__device__ __forceinline__ void load_row(const typename Stored<DT>::type *p, int valid, float rest,
                                         float (&v)[N]) {
  Values<DT, N> row;
  row.load(p, valid);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = i < valid ? row.get(i) : rest;
}

template <int DT, int N>
__device__ __forceinline__ void store_row(typename Stored<DT>::type *p, int valid, const float (&v)[N]) {
  Values<DT, N> row;
  row.set(v);
  row.store(p, valid);
}

// ---- reductions over the L lanes (a power of two, at least 8) that share a row ----------

template <class F>
__device__ __forceinline__ uint32_t across(uint32_t x, int lanes, F f) {
  const auto dpp = [](uint32_t v, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, false);
  };
  x = f(x, dpp(x, std::integral_constant<int, 0xB1>{}));   // quad_perm: xor 1
  x = f(x, dpp(x, std::integral_constant<int, 0x4E>{}));   // quad_perm: xor 2
  x = f(x, dpp(x, std::integral_constant<int, 0x141>{}));  // row_half_mirror
  if (lanes >= 16) x = f(x, dpp(x, std::integral_constant<int, 0x140>{}));  // row_mirror
  if (lanes >= 32) {
    const auto s = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = f(s[0], s[1]);
  }
  if (lanes >= 64) {
    const auto s = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = f(s[0], s[1]);
  }
  return x;
}

template <int L>
__device__ __forceinline__ uint32_t max_across(uint32_t x) {
  return across(x, L, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

template <int L>
__device__ __forceinline__ uint32_t min_across(uint32_t x) {
  return across(x, L, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}

// In an order of its own for every L, the same in every lane.
template <int L>
__device__ __forceinline__ float sum_across(float x) {
  return __builtin_bit_cast(
      float, across(__builtin_bit_cast(uint32_t, x), L, [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t,
                                  __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
      }));
}

// Sum over a workgroup of THREADS, in every thread; `room` holds a value for each wave.
template <int THREADS, class T>
__device__ __forceinline__ T sum_workgroup(T x, T *room) {
#pragma unroll
  for (int step = 1; step < kWave; step *= 2) x += __shfl_xor(x, step);
  __syncthreads();
  if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) x += room[w];
  return x;
}

// exp(x) for x <= 0 (NaN: some value), 0 below 2^-126: 2^t for the rounded t = x log2(e), and what t
// lacks as a factor.  Within 2 units of the last place, in six operations.
__device__ __forceinline__ float exp_down(float x) {
  x = fmaxf(x, -200.0f);
  const float t = x * 1.44269504f;
  float rest = fmaf(x, 1.44269504f, -t);
  rest = fmaf(x, 1.92596303e-8f, rest);
  const float e = __builtin_amdgcn_exp2f(t);
  return fmaf(e, rest * 0.69314718f, e);
}

// What one lane of a wave wrote to LDS is there for its others: LDS works through a wave's
// accesses in order, and the compiler may not move them over this.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---- choice of experts --------------------------------------------------------------
//
// p = softmax(l), S the k largest logits, f_e the share of expert e in all choices, T the tokens:
//   loss = E sum_e f_e (1/T) sum_t p_te,   slopes_e = d loss / d p_te = E f_e / T.
// L lanes share a row; each has V experts, four consecutive ones of each 4 L (expert_of).  A choice is a
// maximum over the lanes, and the least index that has it.  Sums of p stay in the lanes' registers
// over a workgroup's rows; workgroups leave theirs and their counts in the workspace, and other
// workgroups, one for 64 experts, join them in order.

struct RouteArgs {
  const void *logits;
  int64_t stride;
  const uint8_t *valid;
  int m, experts, k, renormalize;
  int32_t *chosen;
  float *weights;
  int32_t *counts;
  float *loss, *slopes;
  // of each workgroup: sums of p, counts (`pitch` of each, in fours), how many tokens have an expert
  // and how many they have
  int pitch;
  float *part_p;
  int32_t *part_counts, *part_tokens, *part_choices;
  // of each joining workgroup its share of the loss, and how many are done
  uint64_t *part_loss;
  uint32_t *done;
};

constexpr int kRouteThreads = 512;

// Larger logits have larger keys, NaN the largest, and -0 is 0.  0: no logit.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
  if (x != x) return 0xFFFFFFFFu;
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
constexpr uint32_t kNone = 0x007FFFFFu;  // -inf, which is never chosen

__device__ __forceinline__ float from_key(uint32_t k) {
  return __builtin_bit_cast(float, (k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}

typedef int i4 __attribute__((ext_vector_type(4)));

constexpr int kJoinExperts = 64;

// 64 experts: four a thread, as many threads to four experts as there are.  Returns their part
// of the loss.
__device__ double join_routes(const RouteArgs &p, int parts, int first) {
  constexpr int kWaves = kRouteThreads / kWave, kWide = kJoinExperts / 4;
  __shared__ f4 sum_p[kRouteThreads];
  __shared__ i4 sum_c[kRouteThreads];
  __shared__ int room_i[kWaves];
  __shared__ double room_d[kWaves];
  const int tid = threadIdx.x, rank = tid / kWide, e0 = first + 4 * (tid % kWide);
  constexpr int kRanks = kRouteThreads / kWide;
  f4 a = f4{0, 0, 0, 0};
  i4 c = i4{0, 0, 0, 0};
  int tokens = 0, all = 0;
  if (e0 < p.pitch) {
#pragma unroll 4
    for (int b = rank; b < parts; b += kRanks) {
      a += *reinterpret_cast<const f4 *>(p.part_p + (int64_t)b * p.pitch + e0);
      c += *reinterpret_cast<const i4 *>(p.part_counts + (int64_t)b * p.pitch + e0);
    }
  }
  for (int b = tid; b < parts; b += kRouteThreads) {
    tokens += p.part_tokens[b];
    all += p.part_choices[b];
  }
  sum_p[tid] = a;
  sum_c[tid] = c;
  tokens = sum_workgroup<kRouteThreads>(tokens, room_i);
  all = sum_workgroup<kRouteThreads>(all, room_i);
  for (int half = kRanks / 2; half > 0; half /= 2) {
    if (rank < half) {
      sum_p[tid] += sum_p[tid + half * kWide];
      sum_c[tid] += sum_c[tid + half * kWide];
    }
    __syncthreads();
  }
  double loss = 0.0;
  if (rank == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (e0 + i >= p.experts) break;
      const double slope =
          all > 0 ? (double)p.experts * sum_c[tid][i] / ((double)all * tokens) : 0.0;
      loss += slope * sum_p[tid][i];
      p.counts[e0 + i] = sum_c[tid][i];
      p.slopes[e0 + i] = (float)slope;
    }
  }
  return sum_workgroup<kRouteThreads>(loss, room_d);
}

// The last workgroup adds the losses up, in order.
__global__ __launch_bounds__(kRouteThreads) void join_routes_kernel(RouteArgs p, int parts) {
  const double loss = join_routes(p, parts, blockIdx.x * kJoinExperts);
  if (threadIdx.x != 0) return;
  if (gridDim.x == 1) {
    *p.loss = (float)loss;
    return;
  }
  __hip_atomic_store(&p.part_loss[blockIdx.x], __builtin_bit_cast(uint64_t, loss), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
  const uint32_t before =
      __hip_atomic_fetch_add(p.done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
  if (before != gridDim.x - 1) return;
  double sum = 0.0;
  for (int b = 0; b < (int)gridDim.x; ++b)
    sum += __builtin_bit_cast(
        double, __hip_atomic_load(&p.part_loss[b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
  *p.loss = (float)sum;
}

// The expert of a lane's place v.
template <int L>
__device__ __forceinline__ int expert_of(int q, int v) {
  return v / 4 * (4 * L) + 4 * q + v % 4;
}

// A row's values at a lane's places; `rest` where there are none.
template <int DT, int L, int V>
__device__ __forceinline__ void load_experts(const typename Stored<DT>::type *row, int q, int experts,
                                             float rest, float (&x)[V]) {
#pragma unroll
  for (int v = 0; v < V; v += 4) {
    const int e = expert_of<L>(q, v);
    Values<DT, 4> four;
    four.load(row + e, experts - e);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[v + i] = e + i < experts ? four.get(i) : rest;
  }
}

// Sum over the rows of a wave, in all of its lanes.
template <int L>
__device__ __forceinline__ float sum_rows(float x) {
  if (L <= 8)
    x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x128, 0xF,
                                                               0xF, false));  // row_ror:8
  if (L <= 16) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    const auto s = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    x = __builtin_bit_cast(float, (uint32_t)s[0]) + __builtin_bit_cast(float, (uint32_t)s[1]);
  }
  if (L <= 32) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    const auto s = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    x = __builtin_bit_cast(float, (uint32_t)s[0]) + __builtin_bit_cast(float, (uint32_t)s[1]);
  }
  return x;
}

template <int DT, int L, int V>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(RouteArgs p) {
  constexpr int kRows = kRouteThreads / L, kWaves = kRouteThreads / kWave;
  struct Pick {
    int expert;
    uint32_t key;
  };
  __shared__ Pick picks[kRows][kMaxChoices];
  __shared__ __attribute__((aligned(16))) int hist[L * V];
  __shared__ __attribute__((aligned(16))) float sums[kWaves][L * V];
  __shared__ int routed, choices;
  const int tid = threadIdx.x, q = tid % L, row = tid / L;
  for (int i = tid; i < L * V; i += kRouteThreads) hist[i] = 0;
  if (tid == 0) {
    routed = choices = 0;
    if (blockIdx.x == 0 && gridDim.x > 1) *p.done = 0;  // for the joining kernel behind this one
  }
  __syncthreads();
  float acc[V] = {};
  int mine_routed = 0, mine_choices = 0;
  const auto *logits = static_cast<const typename Stored<DT>::type *>(p.logits);
  for (int base = blockIdx.x * kRows; base < p.m; base += gridDim.x * kRows) {
    const int t = base + row;
    const bool on = t < p.m && (p.valid == nullptr || p.valid[t] != 0);
    float l[V];
    load_experts<DT, L, V>(logits + (on ? t : 0) * p.stride, q, on ? p.experts : 0, 0.0f, l);
    uint32_t key[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
      key[v] = on && expert_of<L>(q, v) < p.experts ? order_key(l[v]) : 0;
    uint32_t top = 0;
    for (int j = 0; j < p.k; ++j) {
      uint32_t best = 0;
#pragma unroll
      for (int v = 0; v < V; ++v) best = key[v] > best ? key[v] : best;
      const uint32_t most = max_across<L>(best);
      if (j == 0) top = most;
      // the least index of those that are it, which is taken out
      uint32_t at = 0xFFFFu;
#pragma unroll
      for (int v = V - 1; v >= 0; --v) at = key[v] == most ? expert_of<L>(q, v) : at;
      const int chosen = (int)min_across<L>(at);
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = expert_of<L>(q, v) == chosen ? 0 : key[v];
      if (q == 0) picks[row][j] = {most > kNone ? chosen : -1, most};
    }
    wave_sync();
    const bool any = top > kNone;
    const float high = from_key(top);
    // +Inf and NaN make all of the row NaN
    const float one = high < INFINITY ? 1.0f : NAN;
    float sum = 0.0f, ex[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      ex[v] = expert_of<L>(q, v) < p.experts ? exp_down(l[v] - high) : 0.0f;
      sum += ex[v];
    }
    sum = sum_across<L>(sum);
    const float share = any ? one / sum : 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) acc[v] += any ? ex[v] * share : 0.0f;
    mine_routed += any && q == 0;
    float weigh = share;
    if (p.renormalize) {
      float below = 0.0f;
      for (int j = q; j < p.k; j += L)
        below += picks[row][j].expert < 0 ? 0.0f : exp_down(from_key(picks[row][j].key) - high);
      weigh = one / sum_across<L>(below);
    }
    if (t < p.m) {
      for (int j = q; j < p.k; j += L) {
        const Pick pick = picks[row][j];
        const bool there = pick.expert >= 0;
        p.chosen[(int64_t)t * p.k + j] = pick.expert;
        p.weights[(int64_t)t * p.k + j] = there ? exp_down(from_key(pick.key) - high) * weigh : 0.0f;
        if (there) atomicAdd(&hist[pick.expert], 1);
        mine_choices += there;
      }
    }
    wave_sync();
  }
  if (mine_routed > 0) atomicAdd(&routed, mine_routed);
  if (mine_choices > 0) atomicAdd(&choices, mine_choices);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const float a = sum_rows<L>(acc[v]);
    if (tid % kWave < L) sums[tid / kWave][expert_of<L>(q, v)] = a;
  }
  __syncthreads();
  const bool alone = gridDim.x == 1;  // then nothing goes through the workspace
  for (int e = tid; e < p.pitch; e += kRouteThreads) {
    float a = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) a += sums[w][e];
    if (alone) {
      sums[0][e] = a;
    } else {
      p.part_p[(int64_t)blockIdx.x * p.pitch + e] = a;
      p.part_counts[(int64_t)blockIdx.x * p.pitch + e] = hist[e];
    }
  }
  if (tid == 0 && !alone) {
    p.part_tokens[blockIdx.x] = routed;
    p.part_choices[blockIdx.x] = choices;
  }
  if (alone) {
    RouteArgs here = p;
    here.part_p = sums[0];
    here.part_counts = hist;
    here.part_tokens = &routed;
    here.part_choices = &choices;
    double loss = 0.0;
    for (int first = 0; first < p.experts; first += kJoinExperts) {
      __syncthreads();
      loss += join_routes(here, 1, first);
    }
    if (tid == 0) *p.loss = (float)loss;
  }
}

struct RouteGradArgs {
  const void *logits;
  int64_t stride;
  const int32_t *chosen;
  const float *weights, *slopes, *dweights, *dloss;
  int m, experts, k, renormalize;
  void *out;
  int64_t out_stride;
};

// u_e = dloss slopes_e (and, not renormalized, dw_j at the chosen e): dl = p (u - sum p u);
// renormalized, dl_e gets w_j (dw_j - sum_S w dw) besides, the softmax over the chosen.
// p is made again from the logits, which is less to read than p would be.
template <int DT, int L, int V>
__global__ __launch_bounds__(256) void route_gradient_kernel(RouteGradArgs p) {
  constexpr int kRows = 256 / L;
  __shared__ float extra[kRows][L * V];
  const int tid = threadIdx.x, q = tid % L, row = tid / L;
  const auto *logits = static_cast<const typename Stored<DT>::type *>(p.logits);
  auto *out = static_cast<typename Stored<DT>::type *>(p.out);
  float slope[V];
  load_experts<HADACORE_FP32, L, V>(p.slopes, q, p.dloss != nullptr ? p.experts : 0, 0.0f, slope);
  const float g = p.dloss != nullptr ? *p.dloss : 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    slope[v] *= g;
    extra[row][expert_of<L>(q, v)] = 0.0f;
  }
  wave_sync();
  for (int base = blockIdx.x * kRows; base < p.m; base += gridDim.x * kRows) {
    const int t = base + row;
    const bool on = t < p.m && p.chosen[(int64_t)(t < p.m ? t : 0) * p.k] >= 0;
    float l[V];
    load_experts<DT, L, V>(logits + (on ? t : 0) * p.stride, q, on ? p.experts : 0, -INFINITY, l);
    uint32_t best = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const uint32_t key = order_key(l[v]);
      best = key > best ? key : best;
    }
    const float high = from_key(max_across<L>(best));
    float sum = 0.0f, pr[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      pr[v] = on ? exp_down(l[v] - high) : 0.0f;
      sum += pr[v];
    }
    sum = sum_across<L>(sum);
    const float share = on ? (high < INFINITY ? 1.0f : NAN) / sum : 0.0f;
    if (p.dweights != nullptr) {
      float wd = 0.0f;
      if (p.renormalize) {
        for (int j = q; on && j < p.k; j += L)
          wd += p.weights[(int64_t)t * p.k + j] * p.dweights[(int64_t)t * p.k + j];
        wd = sum_across<L>(wd);
      }
      for (int j = q; on && j < p.k; j += L) {
        const int64_t at = (int64_t)t * p.k + j;
        const int e = p.chosen[at];
        const float dw = p.dweights[at];
        if (e >= 0 && e < p.experts) extra[row][e] = p.renormalize ? p.weights[at] * (dw - wd) : dw;
      }
      wave_sync();
    }
    float pu = 0.0f, u[V], add[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      pr[v] *= share;
      add[v] = 0.0f;
      if (p.dweights != nullptr) {
        add[v] = extra[row][expert_of<L>(q, v)];
        extra[row][expert_of<L>(q, v)] = 0.0f;
      }
      u[v] = slope[v] + (p.renormalize ? 0.0f : add[v]);
      pu += pr[v] * u[v];
    }
    pu = sum_across<L>(pu);
#pragma unroll
    for (int v = 0; v < V; v += 4) {
      const int e = expert_of<L>(q, v);
      float four[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        four[i] = on ? pr[v + i] * (u[v + i] - pu) + (p.renormalize ? add[v + i] : 0.0f) : 0.0f;
      if (t < p.m) store_row<DT, 4>(out + t * p.out_stride + e, p.experts - e, four);
    }
    wave_sync();
  }
}

// Lanes to a row and experts to a lane.  What bounds large calls is the issue of vector operations, and a
// step of a choice costs about as many for 16 experts in each of 16 lanes, which does four rows at
// once, as for 4 in each of 64 (16384 x 256, eight choices: 17 us instead of 22).
template <class F>
void for_experts(int64_t experts, F f) {
  using std::integral_constant;
  if (experts <= 32)
    f(integral_constant<int, 8>{}, integral_constant<int, 4>{});
  else if (experts <= 64)
    f(integral_constant<int, 8>{}, integral_constant<int, 8>{});
  else if (experts <= 128)
    f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
  else if (experts <= 256)
    f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
  else if (experts <= 512)
    f(integral_constant<int, 32>{}, integral_constant<int, 16>{});
  else
    f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

template <class F>
void for_type(hadacore_dtype dtype, F f) {
  if (dtype == HADACORE_FP16)
    f(std::integral_constant<int, HADACORE_FP16>{});
  else if (dtype == HADACORE_BF16)
    f(std::integral_constant<int, HADACORE_BF16>{});
  else
    f(std::integral_constant<int, HADACORE_FP32>{});
}

// Words of the workspace behind the parts: the joining workgroups' losses, and how many are done.
constexpr int64_t kRouteWords = 2 * kMaxExperts / kJoinExperts + 2;

// Workgroups of a route: one for each set of rows, at most 256, and no more than the joining
// workgroups read in a few microseconds (2^16 sums and counts).
int64_t route_parts(int64_t m, int64_t experts) {
  int64_t rows = 0;
  for_experts(experts, [&](auto l, auto) { rows = kRouteThreads / decltype(l)::value; });
  int64_t parts = (m + rows - 1) / rows;
  const int64_t most = (1 << 16) / experts < 256 ? (1 << 16) / experts : 256;
  if (parts > most) parts = most;
  return parts > 0 ? parts : 1;
}

// ---- slots by group ------------------------------------------------------------------
//
// A stable counting sort.  A wave takes a run of slots of its workgroup's, counts its groups, and
// gives places 64 slots at a time: lanes of the same group find each other by a ballot for each
// bit of the id, and rank themselves by their lanes.  A workgroup starts from the slots of earlier
// groups, and of its own group in earlier workgroups, which it adds up from all counts.

struct GroupArgs {
  const int32_t *ids;
  int slots, groups;
  int32_t *ends, *rows, *order;
  int32_t *parts;  // counts of each workgroup's slots, groups + 1 each
  int per_block;   // slots of a workgroup, a multiple of 64 for each wave
};

constexpr int kGroupThreads = 1024;
constexpr int kGroupWaves = kGroupThreads / kWave;

__device__ __forceinline__ int group_of(const GroupArgs &p, int slot) {
  const int id = p.ids[slot];
  return (uint32_t)id < (uint32_t)p.groups ? id : p.groups;
}

__global__ __launch_bounds__(kGroupThreads) void count_groups_kernel(GroupArgs p) {
  extern __shared__ int hist[];
  const int bins = p.groups + 1;
  for (int g = threadIdx.x; g < bins; g += kGroupThreads) hist[g] = 0;
  __syncthreads();
  const int low = blockIdx.x * p.per_block;
  const int high = low + p.per_block < p.slots ? low + p.per_block : p.slots;
  for (int s = low + threadIdx.x; s < high; s += kGroupThreads) atomicAdd(&hist[group_of(p, s)], 1);
  __syncthreads();
  for (int g = threadIdx.x; g < bins; g += kGroupThreads)
    p.parts[(int64_t)blockIdx.x * bins + g] = hist[g];
}

// W: how many waves share the slots (fewer where the counts of 16 would take more than 64 KiB of LDS).
template <int W>
__global__ __launch_bounds__(kGroupThreads) void place_groups_kernel(GroupArgs p) {
  extern __shared__ int counts[];  // [W][bins], then of each group: its slots, those before this workgroup
  __shared__ int wave_sums[kGroupWaves];
  const int bins = p.groups + 1, tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  int *all = counts + W * bins, *before = all + bins;
  for (int i = tid; i < (W + 2) * bins; i += kGroupThreads) counts[i] = 0;
  __syncthreads();
  const int low = blockIdx.x * p.per_block;
  const int high = low + p.per_block < p.slots ? low + p.per_block : p.slots;
  const int run = p.per_block / W;
  const int from = low + wave * run, to = from + run < high ? from + run : high;
  if (wave < W)
    for (int s = from + lane; s < to; s += kWave) atomicAdd(&counts[wave * bins + group_of(p, s)], 1);
  __syncthreads();
  if (gridDim.x == 1) {
    for (int g = tid; g < bins; g += kGroupThreads)
      for (int w = 0; w < W; ++w) all[g] += counts[w * bins + g];
  } else {
    int wide = kWave;
    while (wide < bins && wide < kGroupThreads) wide *= 2;
    for (int g = tid % wide; g < bins; g += wide) {
      int sum = 0, early = 0;
#pragma unroll 4
      for (int b = tid / wide; b < (int)gridDim.x; b += kGroupThreads / wide) {
        const int c = p.parts[(int64_t)b * bins + g];
        sum += c;
        early += b < (int)blockIdx.x ? c : 0;
      }
      atomicAdd(&all[g], sum);
      atomicAdd(&before[g], early);
    }
  }
  __syncthreads();
  const int each = (bins + kGroupThreads - 1) / kGroupThreads;
  int sum = 0;
  for (int i = 0; i < each; ++i) sum += tid * each + i < bins ? all[tid * each + i] : 0;
  // the groups before this thread's
  const int upto = prefix_sum(sum);
  if (lane == kWave - 1) wave_sums[wave] = upto;
  __syncthreads();
  int start = upto - sum;
  for (int w = 0; w < wave; ++w) start += wave_sums[w];
  for (int i = 0; i < each; ++i) {
    const int g = tid * each + i;
    if (g >= bins) break;
    // a group's end is where the next one starts: group 0's start is 0
    if (blockIdx.x == 0 && g > 0) p.ends[g - 1] = start;
    int at = start + before[g];
    start += all[g];
    for (int w = 0; w < W; ++w) {
      const int c = counts[w * bins + g];
      counts[w * bins + g] = at;
      at += c;
    }
  }
  __syncthreads();
  if (wave >= W) return;
  int bits = 0;
  while ((1 << bits) < bins) ++bits;
  for (int s0 = from; s0 < to; s0 += kWave) {
    const int s = s0 + lane;
    const bool on = s < to;
    const int g = on ? group_of(p, s) : 0;
    uint64_t same = __ballot(on);
    for (int b = 0; b < bits; ++b) {
      const uint64_t one = __ballot((g >> b) & 1);
      same &= (g >> b) & 1 ? one : ~one;
    }
    const int ahead = __popcll(same & ((1ull << lane) - 1));
    int *next = &counts[wave * bins + g];
    const int at = on ? *next + ahead : 0;
    wave_sync();
    if (on && ahead == 0) *next = at + __popcll(same);
    wave_sync();
    if (on) {
      p.rows[s] = g < p.groups ? at : -1;
      p.order[at] = s;
    }
  }
}

// How many waves of a workgroup share its slots: the counts take 64 KiB of LDS at most.
int group_waves(int64_t groups) { return groups <= 900 ? 16 : groups <= 2700 ? 4 : 2; }

// Workgroups.  Up to 8192 slots one does it in one launch (8.7 us; two launches take 2.4 and 4.6 and
// the time between them); from there one for 2048 slots, 128 at most, since each adds up the counts
// of all (131072 slots of 256 groups: 2.4 and 9.5 us).
int64_t group_blocks_of(int64_t slots, int64_t groups) {
  if (slots <= 8192) return 1;
  const int64_t blocks = (slots + 2047) / 2048, most = (1 << 16) / (groups + 1);
  return blocks < most ? blocks < 128 ? blocks : 128 : most < 128 ? most : 128;
}

// ---- rows to their places, and back --------------------------------------------------

struct DispatchArgs {
  const uint8_t *in;
  int64_t in_stride, out_stride;  // bytes
  const int32_t *rows, *ends;
  uint8_t *out;
  int m, k, groups, bytes, size;  // bytes of a row, of a value
  int chunks;
};

typedef u4 u4_any __attribute__((aligned(1)));

// One wave copies 4 KiB of a token's row to the places of its slots: the row is read once.  It also
// clears that part of those of its own slots' places that lie behind the last end.
constexpr int kDispatchLoads = 4;
constexpr int kDispatchChunk = kWave * 16 * kDispatchLoads;

template <bool NT>
__global__ __launch_bounds__(256) void dispatch_kernel(DispatchArgs p) {
  const int lane = threadIdx.x % kWave;
  const int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int t = (int)(id / p.chunks), chunk = (int)(id % p.chunks);
  if (t >= p.m) return;
  const int slots = p.m * p.k;
  const int used = p.groups > 0 ? clamp_end(p.ends[p.groups - 1], slots) : 0;
  const int start = chunk * kDispatchChunk + lane * 16;
  const uint8_t *from = p.in + t * p.in_stride;
  u4 v[kDispatchLoads];
#pragma unroll
  for (int i = 0; i < kDispatchLoads; ++i) {
    const int at = start + i * kWave * 16;
    v[i] = u4{0, 0, 0, 0};
    if (at + 16 <= p.bytes) v[i] = *reinterpret_cast<const u4_any *>(from + at);
  }
  const auto copy = [&](int row, bool zero) {
    uint8_t *to = p.out + row * p.out_stride;
#pragma unroll
    for (int i = 0; i < kDispatchLoads; ++i) {
      const int at = start + i * kWave * 16;
      if (at + 16 <= p.bytes) {
        const u4 put = zero ? u4{0, 0, 0, 0} : v[i];
        if constexpr (NT)
          __builtin_nontemporal_store(put, reinterpret_cast<u4_any *>(to + at));
        else
          *reinterpret_cast<u4_any *>(to + at) = put;
      } else {
        // the row's last bytes, value by value
        for (int b = at; b < p.bytes; b += p.size) {
          if (p.size == 1)
            to[b] = zero ? 0 : from[b];
          else if (p.size == 2)
            *reinterpret_cast<uint16_t *>(to + b) =
                zero ? 0 : *reinterpret_cast<const uint16_t *>(from + b);
          else
            *reinterpret_cast<uint32_t *>(to + b) =
                zero ? 0 : *reinterpret_cast<const uint32_t *>(from + b);
        }
      }
    }
  };
  for (int j = 0; j < p.k; ++j) {
    const int slot = t * p.k + j;
    const int row = p.rows[slot];
    if ((uint32_t)row < (uint32_t)used) copy(row, false);
    if (slot >= used) copy(slot, true);
  }
}

struct CombineArgs {
  const void *in;
  int64_t in_stride, out_stride;
  const int32_t *rows;
  const float *weights;
  void *out;
  int places, m, k, width, chunks;
};

// One wave joins 64 N columns of a token's rows: the loads of K slots before their sums.
template <int DT, int N, int K, bool NT>
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs p) {
  using T = typename Stored<DT>::type;
  const int lane = threadIdx.x % kWave;
  const int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int t = (int)(id / p.chunks), chunk = (int)(id % p.chunks);
  if (t >= p.m) return;
  const int col = chunk * (kWave * N) + lane * N, valid = p.width - col;
  const T *in = static_cast<const T *>(p.in) + col;
  float acc[N] = {};
  const int32_t *rows = p.rows + (int64_t)t * p.k;
  const float *weights = p.weights != nullptr ? p.weights + (int64_t)t * p.k : nullptr;
  for (int j0 = 0; j0 < p.k; j0 += K) {
    Values<DT, N> v[K];
    float w[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
      const int row = j0 + j < p.k ? rows[j0 + j] : -1;
      const bool there = (uint32_t)row < (uint32_t)p.places;
      w[j] = !there ? 0.0f : weights != nullptr ? weights[j0 + j] : 1.0f;
      // a row that is not there adds nothing, whatever its weight: zeros times 0
      v[j].template load<NT>(in + (there ? row : 0) * p.in_stride, there ? valid : 0);
    }
#pragma unroll
    for (int j = 0; j < K; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) acc[i] = fmaf(w[j], v[j].get(i), acc[i]);
  }
  Values<DT, N> out;
  out.set(acc);
  out.template store<NT>(static_cast<T *>(p.out) + t * p.out_stride + col, valid);
}

struct CombineGradArgs {
  const void *dout, *y;
  int64_t dout_stride, y_stride, dy_stride;
  const int32_t *rows, *ends;
  const float *weights;
  void *dy;
  float *dweights;
  int groups, m, k, width;
};

// dy[rows[t,j]] = w_tj dout[t], dw_tj = <dout[t], y[rows[t,j]]>; places behind the last end get zeros.
// W waves go through a token's row together, K slots at a time: dout is read once for them.
template <int DT, int N, int W, int K, bool NT>
__global__ __launch_bounds__(256) void combine_gradient_kernel(CombineGradArgs p) {
  using T = typename Stored<DT>::type;
  __shared__ float parts[4][K];
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int64_t id = (int64_t)blockIdx.x * (4 / W) + (W == 1 ? wave : 0);
  if (W == 1 && id >= p.m) return;
  const int t = (int)id, slots = p.m * p.k;
  const int used = p.groups > 0 ? clamp_end(p.ends[p.groups - 1], slots) : 0;
  const T *dout = static_cast<const T *>(p.dout) + t * p.dout_stride;
  const T *y = static_cast<const T *>(p.y);
  T *dy = static_cast<T *>(p.dy);
  const int first = (W == 1 ? 0 : wave) * kWave * N + lane * N;
  for (int j0 = 0; j0 < p.k; j0 += K) {
    int row[K];
    float w[K], dot[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
      const int64_t at = (int64_t)t * p.k + (j0 + j < p.k ? j0 + j : 0);
      row[j] = p.rows[at];
      if (j0 + j >= p.k || (uint32_t)row[j] >= (uint32_t)used) row[j] = -1;
      w[j] = p.weights != nullptr ? p.weights[at] : 1.0f;
      dot[j] = 0.0f;
    }
    for (int at = first; at < p.width; at += W * kWave * N) {
      const int valid = p.width - at;
      Values<DT, N> d, v[K];
      d.template load<NT>(dout + at, valid);
      if (p.dweights != nullptr) {
#pragma unroll
        for (int j = 0; j < K; ++j)
          v[j].template load<NT>(y + (row[j] >= 0 ? row[j] : 0) * p.y_stride + at, row[j] >= 0 ? valid : 0);
#pragma unroll
        for (int j = 0; j < K; ++j) {
#pragma unroll
          for (int i = 0; i < N; ++i) dot[j] = fmaf(d.get(i), v[j].get(i), dot[j]);
        }
      }
      if (dy != nullptr) {
#pragma unroll
        for (int j = 0; j < K; ++j) {
          if (row[j] >= 0) {
            float s[N];
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] = w[j] * d.get(i);
            v[j].set(s);
            v[j].template store<NT>(dy + row[j] * p.dy_stride + at, valid);
          }
          const int slot = t * p.k + j0 + j;
          if (j0 + j < p.k && slot >= used) {
            const float zero[N] = {};
            v[j].set(zero);
            v[j].template store<NT>(dy + slot * p.dy_stride + at, valid);
          }
        }
      }
    }
    if (p.dweights == nullptr) continue;
#pragma unroll
    for (int j = 0; j < K; ++j) dot[j] = sum_across<kWave>(dot[j]);
    if constexpr (W > 1) {
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (lane == 0) parts[wave][j] = dot[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < K; ++j) dot[j] = ((parts[0][j] + parts[1][j]) + parts[2][j]) + parts[3][j];
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < K; ++j)
      if (threadIdx.x % (W * kWave) == 0 && j0 + j < p.k)
        p.dweights[(int64_t)t * p.k + j0 + j] = row[j] >= 0 ? dot[j] : 0.0f;
  }
}

// ---- arguments -----------------------------------------------------------------------

constexpr int64_t kMaxPitch = int64_t(1) << 26;
constexpr int64_t kMaxBytes = int64_t(1) << 42;
constexpr int64_t kMaxDim = int64_t(1) << 30;

bool aligned_to(const void *p, uintptr_t bytes) {
  return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0;
}

bool is_type(hadacore_dtype t) {
  return t == HADACORE_FP16 || t == HADACORE_BF16 || t == HADACORE_FP32;
}

int64_t size_of(hadacore_dtype t) { return t == HADACORE_FP32 ? 4 : 2; }

hadacore_status status_of(hipError_t e) {
  return e == hipSuccess ? HADACORE_SUCCESS : HADACORE_ERROR_LAUNCH;
}

// A matrix of `rows` rows: its stride, size and address.
hadacore_status check_rows(const void *p, int64_t rows, int64_t pitch, int64_t width, int64_t size) {
  if (pitch < width || pitch > kMaxPitch) return HADACORE_ERROR_INVALID_STRIDE;
  if (rows == 0 || width == 0) return HADACORE_SUCCESS;
  if (pitch > kMaxBytes / rows) return HADACORE_ERROR_TOO_LARGE;
  if (p == nullptr) return HADACORE_ERROR_INVALID_VALUE;
  return aligned_to(p, size) ? HADACORE_SUCCESS : HADACORE_ERROR_MISALIGNED;
}

// An array of `n` values of 4 bytes that has to be there where n > 0.
hadacore_status check_words(const void *p, int64_t n) {
  if (n > 0 && p == nullptr) return HADACORE_ERROR_INVALID_VALUE;
  return aligned_to(p, 4) ? HADACORE_SUCCESS : HADACORE_ERROR_MISALIGNED;
}

template <int N>
hadacore_status first_error(const hadacore_status (&st)[N]) {
  for (hadacore_status s : st)
    if (s != HADACORE_SUCCESS) return s;
  return HADACORE_SUCCESS;
}

// Whether one of the outputs overlaps another or an input.
template <int O, int I>
bool any_overlap(const Span (&out)[O], const Span (&in)[I]) {
  for (int i = 0; i < O; ++i) {
    for (int j = 0; j < i; ++j)
      if (spans_overlap(out[i], out[j])) return true;
    for (const Span &s : in)
      if (spans_overlap(out[i], s)) return true;
  }
  return false;
}

Span words(const void *p, int64_t n) { return span(p, p != nullptr, n, n, 4); }

// Whether rows go with the streaming policy: `bytes` of them, and each of whole lines.
struct Lines {
  const void *p;
  int64_t stride, width;  // bytes
};
bool streams(int64_t bytes, Lines a, Lines b = {nullptr, 0, 0}) {
  return bytes >= (int64_t(1) << 24) && aligned_to(a.p, 128) && (a.stride | a.width) % 128 == 0 &&
         aligned_to(b.p, 128) && (b.stride | b.width) % 128 == 0;
}

hadacore_status check_choices(int64_t m, int64_t experts, int64_t k, hadacore_dtype dtype) {
  if (m < 0) return HADACORE_ERROR_INVALID_VALUE;
  if (experts < 1 || experts > kMaxExperts || k < 1 || k > experts || k > kMaxChoices)
    return HADACORE_ERROR_INVALID_SIZE;
  if (!is_type(dtype)) return HADACORE_ERROR_INVALID_DTYPE;
  return m * k >= kMaxDim || m >= kMaxDim ? HADACORE_ERROR_TOO_LARGE : HADACORE_SUCCESS;
}

// Tokens, choices and columns of the exchange.
hadacore_status check_exchange(int64_t m, int64_t k, int64_t width, int64_t groups) {
  if (m < 0 || k < 1 || width < 0 || groups < 0) return HADACORE_ERROR_INVALID_VALUE;
  if (m >= kMaxDim || k >= kMaxDim || m * k >= kMaxDim || width > kMaxPitch || groups >= kMaxDim)
    return HADACORE_ERROR_TOO_LARGE;
  return HADACORE_SUCCESS;
}

}  // namespace
}  // namespace hadacore

using namespace hadacore;

extern "C" int64_t hadacore_route_workspace_size(int64_t m, int64_t experts) {
  if (m < 0 || m >= kMaxDim || experts < 1 || experts > kMaxExperts) return 0;
  const int64_t parts = route_parts(m, experts);
  return parts > 1 ? parts * (2 * ((experts + 3) & ~3) + 2) * 4 + kRouteWords * 4 : 0;
}

extern "C" hadacore_status hadacore_route(const void *logits, int64_t logits_row_stride,
                                          hadacore_dtype dtype, const uint8_t *valid, int64_t m,
                                          int64_t experts, int64_t k, int32_t renormalize,
                                          int32_t *out_experts, float *out_weights,
                                          int32_t *out_counts, float *out_loss, float *out_slopes,
                                          void *workspace, int64_t workspace_bytes, void *stream) {
  hadacore_status st = check_choices(m, experts, k, dtype);
  if (st != HADACORE_SUCCESS) return st;
  st = check_rows(logits, m, logits_row_stride, experts, size_of(dtype));
  if (st != HADACORE_SUCCESS) return st;
  st = first_error({check_words(out_experts, m * k), check_words(out_weights, m * k),
                    check_words(out_counts, experts), check_words(out_loss, 1),
                    check_words(out_slopes, experts)});
  if (st != HADACORE_SUCCESS) return st;
  const int64_t need = hadacore_route_workspace_size(m, experts);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return HADACORE_ERROR_WORKSPACE;
  if (!aligned_to(workspace, 16)) return HADACORE_ERROR_MISALIGNED;
  if (any_overlap({words(out_experts, m * k), words(out_weights, m * k), words(out_counts, experts),
                   words(out_loss, 1), words(out_slopes, experts),
                   span(workspace, need > 0, need, need, 1)},
                  {span(logits, m, logits_row_stride, experts, size_of(dtype)),
                   span(valid, valid != nullptr, m, m, 1)}))
    return HADACORE_ERROR_OVERLAP;
  st = check_device();
  if (st != HADACORE_SUCCESS) return st;
  const int64_t parts = route_parts(m, experts);
  RouteArgs p{};
  p.logits = logits;
  p.stride = logits_row_stride;
  p.valid = valid;
  p.m = (int)m;
  p.experts = (int)experts;
  p.k = (int)k;
  p.renormalize = renormalize != 0;
  p.chosen = out_experts;
  p.weights = out_weights;
  p.counts = out_counts;
  p.loss = out_loss;
  p.slopes = out_slopes;
  p.pitch = ((int)experts + 3) & ~3;
  p.part_p = static_cast<float *>(workspace);
  p.part_counts = static_cast<int32_t *>(workspace) + parts * p.pitch;
  p.part_tokens = p.part_counts + parts * p.pitch;
  p.part_choices = p.part_tokens + parts;
  p.part_loss = reinterpret_cast<uint64_t *>(p.part_choices + parts);  // 8-byte aligned: 2 parts and fours
  p.done = reinterpret_cast<uint32_t *>(p.part_loss + kMaxExperts / kJoinExperts);
  hipStream_t s = static_cast<hipStream_t>(stream);
  for_type(dtype, [&](auto dt) {
    for_experts(experts, [&](auto l, auto v) {
      hipLaunchKernelGGL((route_kernel<decltype(dt)::value, decltype(l)::value, decltype(v)::value>),
                         dim3((uint32_t)parts), dim3(kRouteThreads), 0, s, p);
    });
  });
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && parts > 1) {
    const int64_t joins = (experts + kJoinExperts - 1) / kJoinExperts;
    hipLaunchKernelGGL(join_routes_kernel, dim3((uint32_t)joins), dim3(kRouteThreads), 0, s, p, (int)parts);
    e = hipGetLastError();
  }
  return status_of(e);
}

extern "C" hadacore_status hadacore_route_gradient(
    const void *logits, int64_t logits_row_stride, hadacore_dtype dtype, const int32_t *chosen,
    const float *weights, const float *slopes, const float *dweights, const float *dloss, int64_t m,
    int64_t experts, int64_t k, int32_t renormalize, void *out, int64_t out_row_stride,
    void *stream) {
  hadacore_status st = check_choices(m, experts, k, dtype);
  if (st != HADACORE_SUCCESS) return st;
  const int64_t size = size_of(dtype);
  st = first_error({check_rows(logits, m, logits_row_stride, experts, size),
                    check_rows(out, m, out_row_stride, experts, size)});
  if (st != HADACORE_SUCCESS || m == 0) return st;
  st = first_error({check_words(chosen, m * k), check_words(weights, dweights != nullptr ? m * k : 0),
                    check_words(slopes, dloss != nullptr ? experts : 0), check_words(dweights, 0),
                    check_words(dloss, 0)});
  if (st != HADACORE_SUCCESS) return st;
  if (any_overlap({span(out, m, out_row_stride, experts, size)},
                  {span(logits, m, logits_row_stride, experts, size), words(chosen, m * k),
                   words(weights, m * k), words(slopes, experts), words(dweights, m * k),
                   words(dloss, 1)}))
    return HADACORE_ERROR_OVERLAP;
  st = check_device();
  if (st != HADACORE_SUCCESS) return st;
  RouteGradArgs p{};
  p.logits = logits;
  p.stride = logits_row_stride;
  p.chosen = chosen;
  p.weights = weights;
  p.slopes = slopes;
  p.dweights = dweights;
  p.dloss = dloss;
  p.m = (int)m;
  p.experts = (int)experts;
  p.k = (int)k;
  p.renormalize = renormalize != 0;
  p.out = out;
  p.out_stride = out_row_stride;
  for_type(dtype, [&](auto dt) {
    for_experts(experts, [&](auto l, auto v) {
      constexpr int kRows = 256 / decltype(l)::value;
      const int64_t blocks = (m + kRows - 1) / kRows, most = (int64_t)device_cus() * 8;
      hipLaunchKernelGGL(
          (route_gradient_kernel<decltype(dt)::value, decltype(l)::value, decltype(v)::value>),
          dim3((uint32_t)(blocks < most ? blocks : most)), dim3(256), 0,
          static_cast<hipStream_t>(stream), p);
    });
  });
  return status_of(hipGetLastError());
}

extern "C" int64_t hadacore_group_workspace_size(int64_t slots, int64_t groups) {
  if (slots < 0 || slots >= kMaxDim || groups < 0 || groups > HADACORE_MAX_GROUPS) return 0;
  const int64_t blocks = group_blocks_of(slots, groups);
  return blocks > 1 ? blocks * (groups + 1) * 4 : 0;
}

extern "C" hadacore_status hadacore_group_tokens(const int32_t *ids, int64_t slots, int64_t groups,
                                                 int32_t *out_ends, int32_t *out_rows,
                                                 int32_t *out_slots, void *workspace,
                                                 int64_t workspace_bytes, void *stream) {
  if (slots < 0 || groups < 0) return HADACORE_ERROR_INVALID_VALUE;
  if (groups > HADACORE_MAX_GROUPS) return HADACORE_ERROR_INVALID_SIZE;
  if (slots >= kMaxDim) return HADACORE_ERROR_TOO_LARGE;
  hadacore_status st = first_error({check_words(ids, slots), check_words(out_ends, groups),
                                    check_words(out_rows, slots), check_words(out_slots, slots)});
  if (st != HADACORE_SUCCESS) return st;
  const int64_t need = hadacore_group_workspace_size(slots, groups);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return HADACORE_ERROR_WORKSPACE;
  if (!aligned_to(workspace, 4)) return HADACORE_ERROR_MISALIGNED;
  if (any_overlap({words(out_ends, groups), words(out_rows, slots), words(out_slots, slots),
                   span(workspace, need > 0, need, need, 1)},
                  {words(ids, slots)}))
    return HADACORE_ERROR_OVERLAP;
  if (groups == 0 && slots == 0) return HADACORE_SUCCESS;
  st = check_device();
  if (st != HADACORE_SUCCESS) return st;
  const int64_t blocks = group_blocks_of(slots, groups);
  const int waves = group_waves(groups);
  GroupArgs p{};
  p.ids = ids;
  p.slots = (int)slots;
  p.groups = (int)groups;
  p.ends = out_ends;
  p.rows = out_rows;
  p.order = out_slots;
  p.parts = static_cast<int32_t *>(workspace);
  const int64_t unit = kWave * waves;
  p.per_block = (int)(((slots + blocks - 1) / blocks + unit - 1) / unit * unit);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const size_t bins = (size_t)(groups + 1) * 4;
  if (blocks > 1) {
    hipLaunchKernelGGL(count_groups_kernel, dim3((uint32_t)blocks), dim3(kGroupThreads), bins, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return status_of(e);
  }
  if (waves == 16)
    hipLaunchKernelGGL(place_groups_kernel<16>, dim3((uint32_t)blocks), dim3(kGroupThreads),
                       18 * bins, s, p);
  else if (waves == 4)
    hipLaunchKernelGGL(place_groups_kernel<4>, dim3((uint32_t)blocks), dim3(kGroupThreads), 6 * bins,
                       s, p);
  else
    hipLaunchKernelGGL(place_groups_kernel<2>, dim3((uint32_t)blocks), dim3(kGroupThreads), 4 * bins,
                       s, p);
  return status_of(hipGetLastError());
}

extern "C" hadacore_status hadacore_dispatch_rows(const void *in, int64_t in_row_stride,
                                                  int32_t value_bytes, const int32_t *rows,
                                                  const int32_t *ends, int64_t groups, void *out,
                                                  int64_t out_row_stride, int64_t m, int64_t k,
                                                  int64_t width, void *stream) {
  hadacore_status st = check_exchange(m, k, width, groups);
  if (st != HADACORE_SUCCESS) return st;
  if (value_bytes != 1 && value_bytes != 2 && value_bytes != 4) return HADACORE_ERROR_INVALID_DTYPE;
  st = first_error({check_rows(in, m, in_row_stride, width, value_bytes),
                    check_rows(out, m * k, out_row_stride, width, value_bytes),
                    check_words(rows, m * k), check_words(ends, groups)});
  if (st != HADACORE_SUCCESS || m == 0 || width == 0) return st;
  if (any_overlap({span(out, m * k, out_row_stride, width, value_bytes)},
                  {span(in, m, in_row_stride, width, value_bytes), words(rows, m * k),
                   words(ends, groups)}))
    return HADACORE_ERROR_OVERLAP;
  DispatchArgs p{};
  p.in = static_cast<const uint8_t *>(in);
  p.in_stride = in_row_stride * value_bytes;
  p.out_stride = out_row_stride * value_bytes;
  p.rows = rows;
  p.ends = ends;
  p.out = static_cast<uint8_t *>(out);
  p.m = (int)m;
  p.k = (int)k;
  p.groups = (int)groups;
  p.bytes = (int)(width * value_bytes);
  p.size = value_bytes;
  p.chunks = (p.bytes + kDispatchChunk - 1) / kDispatchChunk;
  const int64_t blocks = (m * p.chunks + 3) / 4;
  if (blocks * 256 >= (int64_t(1) << 32)) return HADACORE_ERROR_TOO_LARGE;
  st = check_device();
  if (st != HADACORE_SUCCESS) return st;
  if (streams(m * k * p.bytes, {out, p.out_stride, p.bytes}))
    hipLaunchKernelGGL(dispatch_kernel<true>, dim3((uint32_t)blocks), dim3(256), 0,
                       static_cast<hipStream_t>(stream), p);
  else
    hipLaunchKernelGGL(dispatch_kernel<false>, dim3((uint32_t)blocks), dim3(256), 0,
                       static_cast<hipStream_t>(stream), p);
  return status_of(hipGetLastError());
}

extern "C" hadacore_status hadacore_combine_rows(const void *in, int64_t in_row_stride,
                                                 int64_t places, hadacore_dtype dtype,
                                                 const int32_t *rows, const float *weights,
                                                 void *out, int64_t out_row_stride, int64_t m,
                                                 int64_t k, int64_t width, void *stream) {
  hadacore_status st = check_exchange(m, k, width, 0);
  if (st != HADACORE_SUCCESS) return st;
  if (places < 0) return HADACORE_ERROR_INVALID_VALUE;
  if (!is_type(dtype)) return HADACORE_ERROR_INVALID_DTYPE;
  if (places >= kMaxDim) return HADACORE_ERROR_TOO_LARGE;
  const int64_t size = size_of(dtype);
  st = first_error({check_rows(in, places, in_row_stride, width, size),
                    check_rows(out, m, out_row_stride, width, size), check_words(rows, m * k),
                    check_words(weights, 0)});
  if (st != HADACORE_SUCCESS || m == 0 || width == 0) return st;
  if (any_overlap({span(out, m, out_row_stride, width, size)},
                  {span(in, places, in_row_stride, width, size), words(rows, m * k),
                   words(weights, m * k)}))
    return HADACORE_ERROR_OVERLAP;
  CombineArgs p{};
  p.in = in;
  p.in_stride = in_row_stride;
  p.out_stride = out_row_stride;
  p.rows = rows;
  p.weights = weights;
  p.out = out;
  p.places = (int)places;
  p.m = (int)m;
  p.k = (int)k;
  p.width = (int)width;
  hadacore_status result = HADACORE_SUCCESS;
  for_type(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value, N = DT == HADACORE_FP32 ? 4 : 8;
    p.chunks = (p.width + kWave * N - 1) / (kWave * N);
    const int64_t blocks = (m * p.chunks + 3) / 4;
    if (blocks * 256 >= (int64_t(1) << 32)) {
      result = HADACORE_ERROR_TOO_LARGE;
      return;
    }
    result = check_device();
    if (result != HADACORE_SUCCESS) return;
    const auto go = [&](auto slots, auto nt) {
      hipLaunchKernelGGL((combine_kernel<DT, N, decltype(slots)::value, decltype(nt)::value>),
                         dim3((uint32_t)blocks), dim3(256), 0, static_cast<hipStream_t>(stream), p);
    };
    const auto by_slots = [&](auto nt) {
      if (k <= 2)
        go(std::integral_constant<int, 2>{}, nt);
      else
        go(std::integral_constant<int, 4>{}, nt);
    };
    if (streams(m * k * width * size, {in, in_row_stride * size, width * size},
                {out, out_row_stride * size, width * size}))
      by_slots(std::true_type{});
    else
      by_slots(std::false_type{});
    result = status_of(hipGetLastError());
  });
  return result;
}

extern "C" hadacore_status hadacore_combine_gradient(
    const void *dout, int64_t dout_row_stride, const void *y, int64_t y_row_stride,
    hadacore_dtype dtype, const int32_t *rows, const int32_t *ends, int64_t groups,
    const float *weights, void *dy, int64_t dy_row_stride, float *dweights, int64_t m, int64_t k,
    int64_t width, void *stream) {
  hadacore_status st = check_exchange(m, k, width, groups);
  if (st != HADACORE_SUCCESS) return st;
  if (!is_type(dtype)) return HADACORE_ERROR_INVALID_DTYPE;
  const int64_t size = size_of(dtype);
  const bool want_w = dweights != nullptr, want_y = dy != nullptr;
  st = first_error({check_rows(dout, m, dout_row_stride, width, size), check_words(rows, m * k),
                    check_words(ends, groups), check_words(weights, 0), check_words(dweights, 0)});
  if (st == HADACORE_SUCCESS && want_w) st = check_rows(y, m * k, y_row_stride, width, size);
  if (st == HADACORE_SUCCESS && want_y) st = check_rows(dy, m * k, dy_row_stride, width, size);
  if (st != HADACORE_SUCCESS || m == 0 || (!want_w && !want_y)) return st;
  if (any_overlap({span(dy, want_y ? m * k : 0, dy_row_stride, width, size), words(dweights, m * k)},
                  {span(dout, m, dout_row_stride, width, size),
                   span(y, want_w ? m * k : 0, y_row_stride, width, size), words(rows, m * k),
                   words(ends, groups), words(weights, m * k)}))
    return HADACORE_ERROR_OVERLAP;
  CombineGradArgs p{};
  p.dout = dout;
  p.y = y;
  p.dout_stride = dout_row_stride;
  p.y_stride = y_row_stride;
  p.dy_stride = dy_row_stride;
  p.rows = rows;
  p.ends = ends;
  p.weights = weights;
  p.dy = dy;
  p.dweights = dweights;
  p.groups = (int)groups;
  p.m = (int)m;
  p.k = (int)k;
  p.width = (int)width;
  if (m * 256 >= (int64_t(1) << 32)) return HADACORE_ERROR_TOO_LARGE;
  st = check_device();
  if (st != HADACORE_SUCCESS) return st;
  for_type(dtype, [&](auto dt) {
    constexpr int DT = decltype(dt)::value, N = DT == HADACORE_FP32 ? 4 : 8;
    const auto go = [&](auto waves, auto slots) {
      constexpr int W = decltype(waves)::value, K = decltype(slots)::value;
      const dim3 grid((uint32_t)((m * W + 3) / 4));
      hipStream_t s = static_cast<hipStream_t>(stream);
      if (streams(m * k * width * size, {want_y ? dy : y, (want_y ? dy_row_stride : y_row_stride) * size,
                                         width * size}))
        hipLaunchKernelGGL((combine_gradient_kernel<DT, N, W, K, true>), grid, dim3(256), 0, s, p);
      else
        hipLaunchKernelGGL((combine_gradient_kernel<DT, N, W, K, false>), grid, dim3(256), 0, s, p);
    };
    const auto by_slots = [&](auto waves) {
      if (k == 1)
        go(waves, std::integral_constant<int, 1>{});
      else if (k == 2)
        go(waves, std::integral_constant<int, 2>{});
      else
        go(waves, std::integral_constant<int, 4>{});
    };
    if (width <= kWave * N)
      by_slots(std::integral_constant<int, 1>{});
    else
      by_slots(std::integral_constant<int, 4>{});
  });
  return status_of(hipGetLastError());
}
