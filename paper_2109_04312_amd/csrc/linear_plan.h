// How the products of a layer's feed-forward half are computed (linear_mfma.hip), by their sizes: shapes of workgroups, what they cost, and
// the choice among them.  (Host code; a test asks it for the form of each tested size.)
#pragma once
#include <algorithm>
#include <cstddef>

#include "product.h"

namespace mate {

// Which shape: a compute unit that gets n tiles of one needs about (k / 64) (c2 for every two tiles, c1 for an odd last one) + e n us.  The costs leave
// out what the epilogue does, which lengthens a launch (16384 tokens 1024 -> 4096: 125 us, 142 with gelu, 155 with z in 8 bits too, 165 with y as
// well) without changing much which shape is fastest.  Of 26 products of 304 to 16384 tokens, 128 to 4096 wide, each with five epilogues (none; gelu; gelu, z in 8
// bits; z and y in 8 bits; silu, residual and z), the form that a forward takes is 0.5 to 0.8 % behind the fastest in the mean, 6 to 10 % at most.
// dx alone, with and without slope and residual, is 6 to 9 % behind in the mean and 51 % at most (1036 tokens, 2176 <- 672, 15.1 us by tiles of
// 64 tokens, 10.0 by 128): it takes the form that it has beside dw, see below.
//                        features x tokens, wavefronts, stages, workgroups per CU, groups
using Tile256 = Shape<4, 4, 2, 4, 2, 1>;
using Tile128 = Shape<2, 2, 2, 2, 2, 2>;
using Tile128x2 = Shape<2, 2, 2, 2, 2, 1, 2>;
using Tile64 = Shape<2, 1, 2, 2, 3, 2>;
using Tile64x2 = Shape<2, 1, 2, 2, 3, 1, 2>;
enum ProductForm { kProduct256, kProduct128, kProduct128x2, kProduct64, kProduct64x2 };
struct ProductChoice {
  double cost, tile_cost;   // us, and of a tile alone on its unit
  long tiles;
  int rows, groups;         // tokens of a tile; shapes with as many groups add up a product's stages in the same order
  ProductForm form;
};
template <class S>
ProductChoice product_as(ProductForm form, int T, int O, int K, double c1, double c2, double e) {
  const long tiles = (T + (long)S::kRowsB - 1) / S::kRowsB * ((O + S::kRowsA - 1) / S::kRowsA), n = (tiles + 255) / 256;
  const int stages = (K + 63) / 64;
  return {stages * ((n / 2) * c2 + (n % 2) * c1) + e * n, stages * c1 + e, tiles, S::kRowsB, S::kGroups, form};
}
inline ProductChoice choose_product(int T, int O, int K) {
  ProductChoice best = product_as<Tile256>(kProduct256, T, O, K, 1.37, 3.14, 5.33);
  for (const ProductChoice& c : {product_as<Tile128>(kProduct128, T, O, K, 0.62, 1.09, 1.1), product_as<Tile128x2>(kProduct128x2, T, O, K, 0.47, 1.2, 1.86),
                                 product_as<Tile64>(kProduct64, T, O, K, 0.46, 0.74, 0.53), product_as<Tile64x2>(kProduct64x2, T, O, K, 0.39, 0.8, 0.71)})
    if (c.cost < best.cost) best = c;
  return best;
}

struct FewForm {
  int rows, blocks, tokens;   // 16 x `blocks` features (or 4 or 8) by 16 x `tokens` tokens a workgroup; rows 0: none
};
struct FewChoice {
  double cost;
  FewForm form;
};
// us of a launch, beside those of tiles (which need three that their costs leave out): a unit reads its workgroups' rows at 35 GB/s.  Over 96
// products of 1 to 1024 tokens and eight pairs of widths (in a graph, weights not in the L2) what it takes is 2 % behind the best form in the
// mean, 24 % at most (where all take 3 to 4 us).  us, whole tiles and so: 1 token 768 -> 768 7.1 and 3.1, 128 8.0 and 4.5, 512 8.4 and 7.0; 1024 -> 4096 at 16
// 8.2 and 4.7, at 64 8.9 and 6.5; 4096 -> 1024 at 1 21 and 4.7, at 256 22 and 17; with z in 8 bits (and read back, 2.5) 303 tokens 3344 -> 216 18.7 and
// 12.6, 12 tokens 1656 -> 2360 15.2 and 9.1.
inline FewChoice few_as(FewForm f, int T, int O, int K) {
  const int features = f.rows * f.blocks, tokens = 16 * f.tokens;
  const long groups = (long)((O + features - 1) / features) * ((T + tokens - 1) / tokens);
  const double bytes = 2.0 * K * (features + std::min(T, tokens));
  return {2.6 + (double)((groups + 255) / 256) * bytes / 35e3, f};
}
constexpr int kFewTokens = 1024;   // (a grid's second dimension; more are never faster so)
inline FewChoice choose_few(int T, int O, int K, bool codes) {
  FewChoice best = {1e30, {0, 0, 0}};
  for (const FewForm& f : {FewForm{16, 2, 1}, FewForm{16, 2, 2}, FewForm{16, 2, 4}})
    if (const FewChoice c = few_as(f, T, O, K); c.cost < best.cost) best = c;
  if (codes) return best;   // (those have whole scale blocks)
  for (const FewForm& f : {FewForm{4, 1, 1}, FewForm{8, 1, 1}, FewForm{16, 1, 1}, FewForm{16, 1, 2}, FewForm{16, 1, 4}})
    if (const FewChoice c = few_as(f, T, O, K); c.cost < best.cost) best = c;
  return best;
}

template <class S>
size_t merge_bytes(size_t tiles, int splits) { return tiles * (splits * (size_t)(S::kRowsA * S::kRowsB * 4) + kMaxRanges * 8); }

// A split contraction: in ranges of 16 stages or more, at most one workgroup a unit.  Tiles of 64 tokens only: with those of 128 both the ranges and
// their addition take longer (1000 tokens 4096 -> 768, halves: 21.1 us, by 64 16.4), and where only they leave units without a tile, they gain
// nothing (1999 tokens 4096 -> 1024 24.8 whole, 25.3 in halves).  us, as above and split: 512 tokens 4096 -> 768 24.2 and 16.4, 2048 -> 768 13.8 and
// 11.4, 1000 tokens 4096 -> 256 17.1 and 13.5, -> 1024 22.0 and 17.5, 300 tokens 2048 -> 1024 13.4 and 11.3; 1024 long, halves would be no faster.
struct SplitChoice {
  double cost;
  int splits;
  size_t bytes;
};
using TileSplit = Tile64x2;
constexpr ProductForm kProductSplit = kProduct64x2;
inline SplitChoice choose_split(int T, int O, int K) {
  SplitChoice best = {1e30, 0, 0};
  const size_t tiles = (T + (size_t)TileSplit::kRowsB - 1) / TileSplit::kRowsB * ((O + TileSplit::kRowsA - 1) / TileSplit::kRowsA);
  const int stages = (K + 63) / 64;
  for (int splits = 2; splits <= kMaxRanges && tiles * splits <= 256 && stages >= 16 * splits; ++splits) {
    double cost = (stages + splits - 1) / splits * 0.29 + 0.9;
    for (int r = 1; r < splits; r *= 2) cost += 2.6 + 0.6 * (double)(tiles * splits) / 256;   // one addition of pairs
    if (cost < best.cost) best = {cost, splits, merge_bytes<TileSplit>(tiles, splits)};
  }
  return best;
}

// How a forward product is computed, by its sizes (and whether results in 8 bits are wanted).
struct ForwardPlan {
  ProductChoice tiles;
  FewChoice few;      // if its form has rows
  SplitChoice split;  // or if its splits are not 0
};
inline ForwardPlan plan_forward(int T, int O, int K, bool codes) {
  ForwardPlan p = {choose_product(T, O, K), {1e30, {0, 0, 0}}, choose_split(T, O, K)};
  if (p.split.cost >= p.tiles.cost) p.split = {p.tiles.cost, 0, 0};
  if (T <= kFewTokens) p.few = choose_few(T, O, K, codes);
  if (p.few.cost < p.split.cost + 3.0) p.split.splits = 0;
  else p.few.form.rows = 0;
  return p;
}

// Ranges of dw, in 64-token blocks.
constexpr int kMostBlocks = 1024;      // of a range
constexpr int kMergeBlocks = 160;      // of all ranges, where the launch adds them

using Wgrad256 = Shape<4, 4, 2, 4, 2, 1>;      // 256 x 256
using Wgrad128 = Shape<2, 2, 2, 2, 2, 1, 2>;   // 128 x 128, two groups

inline size_t align256(size_t n) { return (n + 255) & ~size_t(255); }
inline long tiles_of_size(int F, int E, int tile) { return (long)((F + tile - 1) / tile) * ((E + tile - 1) / tile); }

// How both gradients are computed.  It goes by the sizes, so that neither depends on whether the other one is wanted (or how x was kept).
struct BackwardPlan {
  bool one_launch;
  int splits, per_split, tile;   // of dw
  ProductChoice product;         // of dx
  int dx_splits;                 // ranges of its contraction, each of 16 stages or more (1, or in one launch, by tiles of 64 tokens)
  bool copy;                     // x in 8 bits is brought back first
  size_t bias_off, words_off, copy_off, dx_off, total;
  size_t dx_bytes;               // what dx needs alone
};
// When the last of `first` workgroups of t1 us and then `second` ones of t2 us ends, one at a time on each unit.
inline double end_of_both(int first, double t1, long second, double t2) {
  constexpr int kUnits = 256;
  const int late = first % kUnits, early = kUnits - late;   // units that end the first kind a round later, or not
  double early_at = first / kUnits * t1, late_at = early_at + t1, end = late ? late_at : early_at;
  while (second > 0) {
    const bool use_early = !late || early_at <= late_at;
    double& at = use_early ? early_at : late_at;
    at += t2;
    second -= use_early ? early : late;
    end = std::max(end, at);
  }
  return end;
}
inline BackwardPlan plan_backward(int T, int E, int F, bool codes) {
  BackwardPlan p = {};
  const long blocks = (T + 63L) / 64;
  constexpr int kSlots = 256;
  p.product = choose_product(T, E, F);
  p.dx_splits = 1;
  // Two launches: large tiles read half as much per contraction, small ones need fewer ranges, and every range leaves an fp32
  // matrix that is written and read again.  In us, one workgroup a compute unit: 1.45 a token block for 256 x 256, 0.58 for
  // 128 x 128 with two groups, 1 per 6.5 MB of partial sums.  (Measured and so, both gradients: 4072 tokens 2048 -> 768 43.6 and 45, 768 -> 2048 41
  // and 47, 2048 tokens 768 -> 768 22.0 and 21.5, 512 17.1 and 17.5.)
  double two = 1e30;
  for (int tile : {256, 128}) {
    const long tiles = tiles_of_size(F, E, tile);
    // enough workgroups for the chip, but ranges of at least eight token blocks
    const long want = std::max({1L, std::min(std::max(1L, kSlots / tiles), blocks / 8), (blocks + kMostBlocks - 1) / kMostBlocks});
    const long per = (blocks + want - 1) / want, splits = (blocks + per - 1) / per;
    const double rounds = (double)((tiles * splits + kSlots - 1) / kSlots);
    const double cost = rounds * per * (tile == 256 ? 1.45 : 0.58) + (tile == 256 ? 3.5 : 0.0) + (splits > 1 ? splits * 8.0 * F * E / 6.5e6 : 0.0);
    if (cost < two) {
      two = cost;
      p.tile = tile;
      p.per_split = (int)per;
      p.splits = (int)splits;
    }
  }
  two += 7.5 + p.product.cost;
  // One: the tiles of dw first, 128 x 128, each over all blocks or a few ranges of them that the launch adds; those of dx take the units that
  // are left.  Only for a dx whose tiles two groups of wavefronts share: beside tiles of 256 x 256 those of dw take half as long again.  (us, as two
  // launches and as one: 512 tokens 768 -> 768 17.1 and 10.4, 1024 768 -> 2048 26.9 and 16.5, 2048 768 -> 768 22.0 and 18.3, 4096 1024 -> 1024 35 and 28.)
  const long tiles = tiles_of_size(F, E, 128);
  if (blocks <= kMergeBlocks && p.product.groups == 2)
    for (int ranges = 1; ranges <= kMaxRanges && tiles * ranges <= kSlots && (ranges == 1 || blocks >= 8 * ranges); ++ranges) {
      const int first = (int)((tiles * ranges + 7) / 8 * 8);
      double t1 = (0.44 + 0.12 * std::min(1.0, first / 256.0)) * ((blocks + ranges - 1) / ranges) + 5.1;
      for (int r = 1; r < ranges; r *= 2) t1 += 2.7;   // one addition of pairs
      auto consider = [&](const ProductChoice& c, int dx_splits, double dx_cost) {
        // (Several must be worth 16 %, an allowance.  Where it decides, over 24 sizes of 1002 to 9311 tokens, both gradients without it take 0.99 of the time with
        // it where nothing is padding, 0.98 at a tenth and 0.96 at half, 0.86 to 1.10 each.)
        const double cost = (ranges > 1 ? 1.16 : 1.0) * (0.5 + end_of_both(first, t1, c.tiles * dx_splits, dx_cost));
        if (cost >= two) return;
        two = cost;
        p.one_launch = true;
        p.splits = ranges;
        p.tile = 128;
        p.per_split = (int)blocks;
        p.product = c;
        p.dx_splits = dx_splits;
      };
      const ProductChoice tall = product_as<Tile128x2>(kProduct128x2, T, E, F, 0.38, 0, 3.1), low = product_as<TileSplit>(kProductSplit, T, E, F, 0.35, 0, 1.8);
      consider(tall, 1, tall.tile_cost);
      consider(low, 1, low.tile_cost);
      // (dx of a long contraction in ranges too.  us, both gradients with a whole contraction and so: 32 tokens 216 -> 3656 24.3 and 15.4, 300 tokens
      // 520 -> 4104 30.7 and 20.9, 512 tokens 1024 -> 4096 33.3 and 26.2, 768 -> 2048 15.5 and 13.5; dx alone 24.6 and 15.0, 30.0 and 17.5, 25.7 and 16.3, 14.7 and 12.4)
      const int dx_stages = (F + 63) / 64;
      for (int n = 2; n <= kMaxRanges && dx_stages >= 16 * n && low.tiles * n <= kSlots; ++n) {
        double cost = (dx_stages + n - 1) / n * 0.35 + 1.8;
        for (int r = 1; r < n; r *= 2) cost += 2.7;
        consider(low, n, cost);
      }
    }
  const long rows = (F + p.tile - 1) / p.tile * p.tile, columns = (E + p.tile - 1) / p.tile * p.tile;   // whole tiles
  if (p.splits > 1) {
    p.bias_off = align256((size_t)p.splits * rows * columns * 4);
    p.words_off = p.bias_off + align256((size_t)p.splits * rows * 4);
    p.total = p.words_off + (p.one_launch ? (size_t)tiles * kMaxRanges * 8 : 0);
  }
  p.copy_off = align256(p.total);
  const double rounds = (double)((tiles_of_size(F, E, p.tile) * p.splits + kSlots - 1) / kSlots), stages = (double)((blocks + p.splits - 1) / p.splits);
  p.copy = 0.36 * rounds * stages > 2.5 + 3.0 * T * E / 4.6e6;
  p.dx_off = align256(p.copy_off + (p.copy && codes ? (size_t)T * E * 2 : 0));
  const size_t dx_part = p.dx_splits > 1 ? merge_bytes<TileSplit>((size_t)p.product.tiles, p.dx_splits) : 0;
  p.dx_bytes = dx_part ? dx_part + 16 : 0;
  p.total = p.dx_off + dx_part + 256;
  return p;
}

}  // namespace mate
