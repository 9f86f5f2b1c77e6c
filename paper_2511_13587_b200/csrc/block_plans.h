// How a product of 8-bit rows and weights is cut up (host arithmetic only): which of the two kernels, and the first one's tiles.
#pragma once

#include <algorithm>
#include <cstdint>

namespace vvs {

// Tiles of 128 weights; of each tile and pass the blocks of K are dealt to `splits` CTAs, a cluster.
struct BlockMatmulPart {
  int64_t first, count;
  int splits;
};
struct BlockMatmulPlan {
  bool pairs;        // block_matmul_pair.cu; the rest is of block_matmul.cu
  int tn;            // rows of a pass
  int passes;
  BlockMatmulPart part[2];                                        // the second may have no tiles
};

constexpr int kMatmulMaxSplits = 8, kMatmulMaxStages = 8;
constexpr int kMatmulTileBytes = 128 * 128;                       // 128 rows of a block of K

// Places of a block's sums in tensor memory.  The summing warps wait for them on their stage's barrier, by its parity: no more places than stages,
// or a stage could be filled and done again before its first sums are taken.
template <int TN>
constexpr int kMatmulPlaces = TN <= 32 ? 4 : 2;
inline int matmul_places(int tn) { return tn <= 32 ? kMatmulPlaces<32> : kMatmulPlaces<64>; }

// Columns of tensor memory of a CTA.  No kernel of the library takes a larger share of an SM's tensor memory than of its shared memory, so that
// whatever lies on an SM together fits; a CTA of the pairs' kernel has all columns and leaves room for nothing that wants some.
template <int TN>
constexpr int kMatmulColumns = TN <= 64 ? 128 : 256;
inline int matmul_columns(int tn) { return tn <= 64 ? kMatmulColumns<64> : kMatmulColumns<128>; }
constexpr int kMatmulPairSmem = 226 * 1024;

// Rows of a pass: the fewest that hold what a pass has.  36 rows through passes of 48 / 64: of 4096 through 22016 weights 19.1 / 19.7 us, 11008 through
// 4096 13.7 / 14.5, 1280 through 1280 4.0 / 4.2.
inline int matmul_rows(int64_t m) {
  const int64_t passes = (m + 127) / 128, each = (m + passes - 1) / passes;
  return each <= 16 ? 16 : each <= 32 ? 32 : each <= 48 ? 48 : each <= 64 ? 64 : each <= 96 ? 96 : 128;
}
// The two parts of a plan go in one launch: clusters of the second part's size, in the first of which each CTA has a tile of the first part.
inline bool matmul_in_one_launch(int tn) { return tn <= 64; }
// Shared memory: blocks of K under way and, of a cluster, the sums that a CTA is sent, 128 weights of its share of the rows in fours.  Two CTAs
// fit an SM up to 64 rows, beside their factors (64 bytes a row) and barriers.
inline int matmul_stage_bytes(int tn) { return kMatmulTileBytes + tn * 128; }
inline int matmul_recv_bytes(int tn, int splits) { return splits > 1 ? splits * ((tn / 4 + splits - 1) / splits) * 128 * 16 : 0; }
inline int matmul_room(int tn) { return (tn <= 32 ? 108 : tn <= 64 ? 107 : 200) * 1024; }
inline int matmul_stages(int tn, int splits) {
  return std::min(kMatmulMaxStages, (matmul_room(tn) - matmul_recv_bytes(tn, splits)) / matmul_stage_bytes(tn));
}
// (with what brings the first stage to a multiple of 1024)
inline int matmul_smem(int tn, int splits) { return matmul_stages(tn, splits) * matmul_stage_bytes(tn) + matmul_recv_bytes(tn, splits) + 1024; }

// clusters: how many clusters of 1 .. 8 CTAs the device holds at once where each CTA has an SM (148, 74, 45, 33, 26, 22, 15, 15).
inline BlockMatmulPlan plan_block_matmul(int64_t m, int64_t n, int64_t k, int n_sms, const int* clusters) {
  BlockMatmulPlan pl{};
  const int64_t nkb = (k + 127) / 128;
  pl.tn = matmul_rows(m);
  const int64_t passes = (m + pl.tn - 1) / pl.tn, tiles = (n + 127) / 128;
  pl.passes = (int)std::min<int64_t>(passes, 65535);
  // Microseconds x 100: blocks of K of the busiest SM (where two CTAs share it, one's loads fill the other's waits), and what a cluster's
  // exchange costs.
  const int64_t a_block = pl.tn <= 32 ? 24 : pl.tn <= 48 ? 28 : pl.tn <= 64 ? 32 : pl.tn <= 96 ? 42 : 50;
  const int per_sm = pl.tn <= 64 ? 2 : 1;
  auto cost = [&](int64_t count, int s) {
    const int64_t each = (count * s + n_sms - 1) / n_sms, rounds = (each + per_sm - 1) / per_sm, blocks = (nkb + s - 1) / s;
    return (each < per_sm ? blocks * a_block * 3 / 2 : each * blocks * a_block) + rounds * 350 + (s > 1 ? 80 + 20 * s : 0);
  };
  // Clusters all fit at once, or some wait for others' end; a CTA has two blocks at least.  288 rows of 3456 through 1280 weights, 30 tiles by
  // 1 / 2 / 4 / 8 CTAs: 12.5 / 9.4 / 7.4 / 12.3 us; 18 rows of 4096 through 4096, 32 tiles: 11.2 / 8.1 / 6.5 / 6.0 (30 of eight fit: here two that
  // wait would do no harm).  Numbers between are slower where all SMs have work already (96 tiles of 32 blocks, 2 / 3: 12.4 / 15.5).
  auto splits_of = [&](int64_t count, bool beside) {              // beside others: a CTA an SM, any number
    int best = 1;
    for (int s = 2; s <= kMatmulMaxSplits && 2 * s <= nkb && count <= (int64_t)clusters[s] * (beside ? 1 : per_sm); s += beside ? 1 : s)
      if (cost(count, s) < cost(count, best)) best = s;
    return best;
  };
  const int whole_splits = splits_of(tiles * passes, false);
  pl.part[0] = {0, tiles, whole_splits};
  int64_t whole = cost(tiles * passes, whole_splits);
  // Tiles that are left over where all SMs have as many as the others: dealt to all SMs, up to 48 rows beside the first ones in the same launch
  // (two CTAs fit an SM), with more than 64 in a launch behind it.  4096 columns through 22016 weights, 172 tiles: 18 rows 18.4 to 18.8 us alike,
  // 17.7 as 148 and 24 by five (21.9 in two launches, of which the second waits for the first); 36 rows 18.1 / 19.0, of 1280 columns 9.0 / 8.9; 64
  // rows, whose sums take longer, 20.9 / 21.2; 72 rows 29.1 / 23.6, 128 rows 33.0 / 26.1.  In the same launch only where an SM has one of the first
  // tiles: with more its clusters do not all fit at once (18 rows of 1280 columns, 297 tiles 12.9 / 14.0, 470 16.8 / 18.3, 600 20.2 / 22.3).
  const int64_t full = tiles / n_sms * n_sms, left = tiles - full;
  if ((pl.tn <= 48 ? full == n_sms : pl.tn > 64 && full > 0) && passes == 1 && left > 0) {
    const int s = splits_of(left, true);
    const int64_t blocks = full / n_sms * nkb + (left * s + n_sms - 1) / n_sms * ((nkb + s - 1) / s);
    const int64_t both = blocks * a_block + 530 + 20 * s + (per_sm == 1 ? full / n_sms * 350 : 0);
    if (both < whole) {
      whole = both;
      pl.part[0] = {0, full, 1};
      pl.part[1] = {full, left, s};
    }
  }
  // The pairs' kernel: rounds of pairs x blocks of K.  Measured at 12 x 8 sizes from 65 to 2048 rows, the smaller of the two numbers is the faster
  // kernel or one within 4 %: 128 rows of 4096 through 22016 weights 26.3 us here, 33.2 on pairs; 256 49.7 / 33.7; 1024 163 / 80; 1024 rows of 1280
  // through 1280 8.0 / 8.3, 2048 15.8 / 9.1.
  const int64_t pair_tiles = (m + 255) / 256 * ((n + 255) / 256), pairs = n_sms / 2;
  const int64_t there = (pair_tiles + pairs - 1) / pairs * (nkb + (nkb & 1)) * 46 + 500;
  pl.pairs = there < whole || passes > 65535;
  return pl;
}

}  // namespace vvs
