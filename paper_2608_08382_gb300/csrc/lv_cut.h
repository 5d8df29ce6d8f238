// How a product is cut between the two kernels of lv_linear.cuh, and what of shared
// memory a cut takes.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace lv {

constexpr int kPiece = 64;                    // of the sum, in a stage
constexpr int kRows = 128;                    // weight rows of a CTA's tile
constexpr int kWBytes = kRows * kPiece * 2;   // of a stage
constexpr int kColFloats = kRows + 4;         // a token's sums in shared memory: 16-byte steps, spread over the banks

constexpr size_t kOutRooms = 8 * 4096;        // of the eight warps that bring a tile out

// k_product.
constexpr int kSpTokens = 160;   // columns at most: with three stages, two CTAs an SM
constexpr int kSpSplit = 8;      // a portable cluster
constexpr int kSpStages = 16;    // at most
constexpr size_t split_stage(int tokens) { return kWBytes + (size_t)tokens * kPiece * 2; }
constexpr size_t split_sums(int tokens, int split) {
  return split == 1 ? kOutRooms : (tokens + (split - 1) * (size_t)((tokens + split - 1) / split)) * kColFloats * sizeof(float);
}
constexpr size_t kSpRoom = 111 << 10;      // of both: two CTAs an SM
constexpr size_t kSpRoomAlone = 222 << 10;  // where there is one for each SM at most
constexpr int split_stages(int tokens, bool alone) {
  const size_t n = (alone ? kSpRoomAlone : kSpRoom) / split_stage(tokens);
  return n < kSpStages ? (int)n : kSpStages;
}

// k_product_pair.
constexpr int kPaTokens = 256;   // columns at most
constexpr int kPaStages = 11;    // at most: what fits of a tile's width (a load takes about 1.1 us to come)
constexpr size_t pair_stage(int tokens) { return kWBytes + (size_t)(tokens / 2) * kPiece * 2; }
constexpr size_t kPaRoom = 6 * pair_stage(kPaTokens);
constexpr int pair_stages(int tokens) {
  return kPaRoom / pair_stage(tokens) < kPaStages ? (int)(kPaRoom / pair_stage(tokens)) : kPaStages;
}

// How a product is cut: by pairs of CTAs, or by CTAs of which `split` share a tile's
// sum; `tokens` columns a tile.
struct Shape {
  bool pair;
  int tokens, split;
};

// The cut that takes least by a model of both kernels' times, in ns: a piece of the sum
// costs its matrix instructions (4 of max(tokens / 2, the clocks that reading their
// operands from shared memory takes), at 1.9 GHz), never less than a turn of the loading
// and issuing loops, nor than its part of the 1.3 to 1.5 us that a load takes to come
// with all stages under way; a tile its way out; CTAs beyond what the device holds wait
// for others to end; of the split kernel an SM holds two.  Fitted to 1,556 measured
// times of 63 calls of 1 to 8,192 tokens (3 to 300 us): the cut that it takes is 1.4 %
// above the best one on average.
template <class Hold>
Shape choose(const Hold &hold, int64_t n_tok, int64_t row_tiles, int64_t chunks) {
  Shape best{true, 256, 1};
  int64_t least = INT64_MAX;
  const int64_t most = (std::min<int64_t>(n_tok, kPaTokens) + 15) / 16 * 16;
  for (int64_t t = 16; t <= most; t += 16) {
    const int64_t token_tiles = (n_tok + t - 1) / t;
    if ((n_tok + token_tiles - 1) / token_tiles + 15 < t && t > 16) continue;  // as many tiles of fewer tokens do
    const int64_t pairs = hold(2);
    const int64_t waves = ((row_tiles + 1) / 2 * token_tiles + pairs - 1) / pairs, out = 180 + 14 * t;
    const int64_t main = chunks * std::max(std::max<int64_t>(130, 1500 / pair_stages((int)t)), std::max(2 * t, 128 + t / 2) * 10 / 19);
    const int64_t cost = 2000 + main * waves + std::max<int64_t>(0, out - main) * (waves - 1) + out;
    if (cost < least) least = cost, best = Shape{true, (int)t, 1};
    if (t > kSpTokens || row_tiles * token_tiles > 4096) continue;
    for (int split = 1; split <= kSpSplit && split <= chunks; ++split) {
      const int64_t tiles = row_tiles * token_tiles, at_once = hold(split);
      if (split > 1 && (tiles > 2 * at_once || split_sums((int)t, split) > kSpRoom)) break;
      const int64_t share = tiles > at_once ? 2 : 1, rounds = (tiles + 2 * at_once - 1) / (2 * at_once);
      const int64_t piece = std::max(std::max<int64_t>(std::max<int64_t>(230, share * 140), 1300 / split_stages((int)t, share == 1)),
                                     share * std::max(2 * t, 128 + t) * 10 / 19);
      const int64_t cost = rounds * ((chunks + split - 1) / split * piece + 1300 + 17 * t) + (split > 1 ? 830 + 230 * split : 0);
      if (cost < least) least = cost, best = Shape{false, (int)t, split};
    }
  }
  return best;
}

}  // namespace lv
