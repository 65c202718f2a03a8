// groups.h -- rows sorted by group: where each group lies, found on the device.
#ifndef HADACORE_GROUPS_H
#define HADACORE_GROUPS_H

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace hadacore {
namespace {

constexpr int kWave = 64;

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

}  // namespace
}  // namespace hadacore

#endif  // HADACORE_GROUPS_H
