// How a product of 8-bit rows and weights is cut up (host arithmetic only): which of the two kernels, and the first one's tiles.
#pragma once

#include <algorithm>
#include <cstdint>

namespace vvs {

struct BlockMatmulPlan {
  bool pairs;        // block_matmul_pair.cu; the rest is of block_matmul.cu
  int tn;            // rows of a pass
  int passes;
  int splits;        // CTAs that share a tile's blocks of K (a cluster)
  int stages;        // blocks of K under way
};

constexpr int kMatmulMaxSplits = 8, kMatmulMaxStages = 8;
constexpr int kMatmulTileBytes = 128 * 128;                       // 128 rows of a block of K

inline int matmul_ctas_per_sm(int tn) { return tn <= 64 ? 2 : 1; }

inline BlockMatmulPlan plan_block_matmul(int64_t m, int64_t n, int64_t k, int n_sms) {
  BlockMatmulPlan pl{};
  const int64_t nkb = (k + 127) / 128;
  int64_t passes = (m + 127) / 128;
  const int64_t each = (m + passes - 1) / passes;
  pl.tn = each <= 16 ? 16 : each <= 32 ? 32 : each <= 64 ? 64 : each <= 96 ? 96 : 128;
  passes = (m + pl.tn - 1) / pl.tn;
  // As many CTAs as the device holds at once, of two blocks of K at least (288 rows of 3456 through 1280 weights, 30 tiles: 1 / 2 / 4 / 8 splits
  // 13.3 / 9.7 / 8.2 / 15.2 us, the last two rounds of CTAs; 18 rows of 4096 through 4096, 32 tiles: 11.2 / 8.7 / 7.2 / 7.1).
  const int64_t tiles = (n + 127) / 128 * passes, slots = (int64_t)n_sms * matmul_ctas_per_sm(pl.tn);
  int64_t splits = 1;
  while (splits < kMatmulMaxSplits && tiles * splits * 2 <= slots && nkb >= 4 * splits) splits *= 2;
  pl.splits = (int)splits;
  pl.stages = std::min(kMatmulMaxStages, (pl.tn <= 64 ? 108 : 200) * 1024 / (kMatmulTileBytes + pl.tn * 128));
  // Microseconds x 100 that either kernel takes: rounds of CTAs (pairs) x blocks of K, and what a round costs beside them.  Measured at 9 x 9
  // sizes from 96 to 2048 rows, it picks the faster one or one within 4 %: 128 rows of 4096 through 22016 weights 35.2 us here, 35.6 on pairs; 256
  // 53.9 / 36.8; 1024 194 / 104; 1024 rows of 1280 through 1280 9.3 / 9.4, 2048 18.3 / 9.8.
  const int64_t a_block = pl.tn <= 32 ? 30 : pl.tn <= 64 ? 40 : pl.tn <= 96 ? 42 : 50;
  const int64_t here = (tiles * splits + slots - 1) / slots * ((nkb + splits - 1) / splits * a_block + 350);
  const int64_t pair_tiles = (m + 255) / 256 * ((n + 255) / 256), pairs = n_sms / 2;
  const int64_t there = (pair_tiles + pairs - 1) / pairs * (nkb + (nkb & 1)) * 46 + 500;
  pl.pairs = there < here || passes > 65535;
  pl.passes = (int)std::min<int64_t>(passes, 65535);
  return pl;
}

}  // namespace vvs
