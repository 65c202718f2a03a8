// adapters_cut.h -- how the adapters' calls are cut into workgroups; host rules only.
#ifndef HADACORE_ADAPTERS_CUT_H
#define HADACORE_ADAPTERS_CUT_H

#include <stdint.h>

namespace hadacore {
namespace {

constexpr int kTile = 16;   // rows and columns of a matrix product
constexpr int kStep = 32;   // its depth
constexpr int kParts = 3;   // 16-bit values that hold one of h

constexpr int kFewWaves = 8;                // of few_tokens_kernel
constexpr int kGradColumns = kTile * 8;     // of a workgroup of the gradients' kernels
constexpr int kGradWaves = 2;               // of gradient_kernel

constexpr int64_t kBlocksWanted = 512;  // two workgroups to a CU of a whole card

inline int64_t round_up(int64_t v, int64_t unit) { return (v + unit - 1) / unit * unit; }
inline int64_t divide_up(int64_t v, int64_t by) { return (v + by - 1) / by; }

// Pieces of `unit` rows that `groups` groups of m rows can have at most.
inline int64_t most_pieces(int64_t m, int64_t groups, int64_t unit) {
  return m / unit + (groups < m ? groups : m) + 1;
}

// Workgroups of few_tokens_kernel at most, and the longest k of which each makes its own h.
constexpr int64_t kFewBlocks = 192, kFewDepth = 8192;

// up_kernel: the steps of a product over the ranks, as its versions have them, and the columns of a
// workgroup of four waves.
inline int64_t up_steps(int64_t rank) { return rank <= 32 ? 1 : rank <= 64 ? 2 : rank <= 128 ? 4 : 8; }
inline int64_t up_columns(int64_t rank) { return rank > 128 ? 4 * 16 * 4 : 4 * 16 * 8; }

// Its LDS for `unit` tokens: the parts of h, a power of two and the token's row.  At most a third of a
// CU's: units of 128, 64, 64 and 32 tokens for its four versions.  (16384 x 4096 -> 8192, rank 64: 188 us a
// call, with units of 128 199; 16384 x 4096 -> 4096, rank 128: 230, with units of 32 277; 8192 x 4096 -> 4096,
// rank 160, and rank 256 in 32 bits: 181 and 221, with units of 64 206 and 245.)
constexpr int64_t kUpRoom = 53 * 1024;
inline int64_t up_room(int64_t unit, int64_t rank) {
  return unit * (kParts * (kStep * up_steps(rank) + 8) * 2 + 8);
}

struct Cut {
  bool fused;  // few_tokens_kernel
  int ranks;   // tiles of ranks in a workgroup of down_kernel
  int tiles;   // tiles of tokens there
  int splits;  // shares of k
  int unit;    // tokens of a workgroup of up_kernel
};

inline Cut cut_of(int64_t m, int64_t k, int64_t n, int64_t rank, int64_t groups) {
  Cut cut{};
  // 64 ranks at most: of more, another workgroup reads x again, but 128 in one leave no registers for
  // loads ahead (16384 x 4096 -> 4096, rank 128, when it came in: 222 us a call instead of 261)
  cut.ranks = rank <= 16 ? 1 : rank <= 32 ? 2 : 4;
  const int64_t live = groups < 1 || m < 1 ? 1 : groups < m ? groups : m;
  const bool few = m <= 32 * live;
  cut.tiles = few ? 1 : 4;
  cut.splits = 1;
  cut.unit = kTile;
  cut.fused = few && rank <= kTile && k <= kFewDepth &&
              most_pieces(m, groups, kTile) * divide_up(n, kFewWaves * 128) <= kFewBlocks;
  if (cut.fused) return cut;
  const int64_t blocks =
      (divide_up(m, 16 * cut.tiles) + live - 1) * divide_up(rank, 16 * cut.ranks);
  // Half of the workgroups with four tiles of ranks, though two of these fit a CU as well: more shares cost
  // more of h to write and join.  With all of them 1024 x 8192 -> 4096, rank 128, takes 51 us instead of 44,
  // 4096 x 4096 -> 4096 and 12000 x 4096 -> 4096, ranks 64 and 48, 49 and 89 instead of 46 and 85; others
  // gain: 8192 x 4096 -> 4096, ranks 64 and 80, 72 and 121 instead of 76 and 128.
  int64_t splits = divide_up(cut.ranks == 4 ? kBlocksWanted / 2 : kBlocksWanted, blocks < 1 ? 1 : blocks);
  const int64_t most = k / 512;  // four steps of k for a wave at least
  splits = splits > most ? most : splits;
  cut.splits = (int)(splits < 1 ? 1 : splits > 16 ? 16 : splits);
  const int64_t columns = divide_up(n, up_columns(rank));
  while (cut.unit < 128 && !few && up_room(2 * cut.unit, rank) <= kUpRoom &&
         m / (2 * cut.unit) * columns >= (rank > 64 ? 1 : 2) * kBlocksWanted)
    cut.unit *= 2;
  return cut;
}

inline int64_t gradient_splits(int64_t m, int64_t width, int64_t rank, int64_t groups) {
  if (groups < 1 || width < 1) return 1;
  const int64_t blocks = divide_up(width, kGradColumns) * groups * divide_up(rank, 64);
  // all at once, two to a CU; of one tile of ranks twice as many do as well or better
  int64_t splits = divide_up(rank <= kTile ? 2 * kBlocksWanted : kBlocksWanted, blocks);
  // a workgroup goes through 64 tokens in a turn; a share has two turns at least
  const int64_t most = m / groups / (2 * kStep * kGradWaves);
  splits = splits > most ? most : splits;
  return splits < 1 ? 1 : splits > 16 ? 16 : splits;
}

}  // namespace
}  // namespace hadacore

#endif  // HADACORE_ADAPTERS_CUT_H
