// Attention of a block's rows over the 8-bit cache, and the weight that every cached key got.
//
// With codes c, scales K_b, V_b of the key's block and w_j = 2^(a_j - m), a_j = log2(e) scale q.k_j + log2 V_b, m a running maximum of a:
//   out = (sum_j w_j cv_j) / (sum_j w_j / V_b),   lse = ln 2 (m + log2 sum_j w_j / V_b)
// so a value's scale costs one addition per score, and what goes into the second product is at most 2^kShift whatever the blocks' scales
// are: halves hold it with 11 bits.  Queries are halves too, each row times a power of two that brings its largest element near 2^14:
// bf16 elements lose nothing but what is 2^-28 of the row's largest.  e4m3 codes are halves exactly.  Float32 contexts split a query
// into three halves and a weight into two (33 and 22 bits).
//
// One pass over the cache.  A (sequence, cached head, tile of rows) is an item of a cluster of CTAs, of four warps or of as many as an SM
// holds, each of them with a share of the keys; a warp has slices of 16 keys of its own, brought by 16-byte asynchronous copies into a ring
// of its own, so no barrier is met before the warps' sums are joined: in shared memory first, then over the cluster through distributed
// shared memory, in rank order.
// Query rows (rows x query heads of the cached head) are the M side of mma.sync m16n8k16.  The order of a head's elements along K of the
// first product, and of the output's columns, is the one in which a lane's codes lie side by side in memory: a 16-byte load of a
// lane is four (keys) or eight (values) operands.
//
// The weights' sums need the whole row's maximum and sum: from the scores, kept in shared memory, where those of the CTA's keys fit, else by a
// second walk over the CTA's keys (from L2).
//
// 32 sequences of nine rows behind 900 to 2380 keys, 32 heads of 128: 119 us, 3.8 TB/s, 59 % of a copy's rate.  Every key is turned to halves
// by the warp that multiplies it, for 16 rows of which nine are there: a slice takes a warp 3400 cycles beside eleven others on its SM,
// conversions, the two products and the weights in one chain.  Left out, measured: slices of 32 keys (116 where 16 took 107), rings of two, four
// and five slices (108 and more), eight warps a CTA (138), keys as 8-bit operands of mma.sync (131).  One token of a float32 context: 7.1 us, a
// call that does next to nothing 4.1; nine rows behind 311 keys, weights summed: 9.4.
#include <type_traits>

#include "quant_cache.cuh"
#include "tc_common.cuh"

namespace vvs {

namespace {

// The reference m of a row moves only when a score passes it by more than kSlack: weights are 2^kShift at the reference, 2^15 at most, and
// halves keep 11 bits down to 2^-21 of the reference's.  After a row's first slices its sums are hardly ever scaled again, and no lane
// has to ask the others for their largest score.
constexpr float kShift = 7.f, kSlack = 8.f;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 bytes from an address and a constant offset; or `bytes` of them, the rest zeros
template <int TO, int FROM>
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0 + %2], [%1 + %3], 16;" ::"r"(dst), "l"(src), "n"(TO), "n"(FROM) : "memory");
}
__device__ __forceinline__ void copy16_some(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
template <int OFF>
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4 + %5];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at), "n"(OFF) : "memory");
  return v;
}
template <int OFF>
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2 + %3];" : "=r"(v.x), "=r"(v.y) : "r"(at), "n"(OFF) : "memory");
  return v;
}
template <int OFF>
__device__ __forceinline__ float lds32(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1 + %2];" : "=f"(v) : "r"(at), "n"(OFF) : "memory");
  return v;
}

template <int HD, int MT, bool F32, bool WIDE>
struct Layout {
  static constexpr int kRows = 16 * MT;
  static constexpr int kSteps = HD / 16;                                    // k-steps of the first product
  static constexpr int kQ = F32 ? 3 : 1;                                    // halves a query element is split into
  static constexpr int kP = F32 ? 2 : 1;                                    // ... a weight
  static constexpr int kTile = 16 * HD;                                     // bytes of 16 keys
  static constexpr int kDepth = MT == 2 ? 4 : 3;                            // slices of a warp's ring
  static constexpr int kSlot = 2 * kTile + 16;                              // keys, values, two scales
  static constexpr int kRing = kDepth * kSlot;
  static constexpr int kQBytes = kQ * MT * kSteps * 512;                    // fragments [piece][tile][step][lane] of 16 bytes
  static constexpr int kPartBytes = kRows * HD * 4;                         // a warp's sums, over its own ring
  static_assert(kPartBytes <= kRing, "a warp's sums take the place of its ring");
  static constexpr int kQAt = 0;
  // CTAs an SM holds by registers: 64 sums of a lane for heads of 128, twice as many for two tiles of rows.  A wide CTA has all of their warps.
  static constexpr int kFit = MT * HD == 256 ? 2 : MT * HD == 128 ? (F32 ? 2 : 3) : 4;
  static constexpr int kWarps = WIDE ? 4 * kFit : 4, kThreads = 32 * kWarps, kCtas = WIDE ? 1 : kFit;
  static constexpr int kScoreBytes = (WIDE ? 56 : 40) * 1024;               // at most, for scores of rows whose weights are summed
  static constexpr int kRingAt = kQBytes;
  static constexpr int kMlAt = kRingAt + kWarps * kRing;                    // [kWarps][kRows][2] warps' maxima and sums
  static constexpr int kTotAt = kMlAt + kWarps * kRows * 8;                 // [kRows][2] the CTA's
  static constexpr int kLseAt = kTotAt + kRows * 8;                         // [kRows] log2 of the row's sum
  static constexpr int kFacAt = kLseAt + kRows * 4;                         // [kRows] what a row's queries were divided by
  static constexpr int kScoreAt = kFacAt + kRows * 4;                       // [rows that are summed][keys of the CTA] log2 scores
  static constexpr int kBytes = kScoreAt;
  // query fragments stay in registers where they are at most 32 of them
  static constexpr bool kQRegs = kQ * MT * kSteps * 4 <= 32;
  static_assert(kCtas * (kBytes + 1024) <= 228 * 1024 && kBytes + kScoreBytes <= 227 * 1024, "shared memory");
};

// where 16 bytes `chunk` of key `row` lie in a slice's tile, so that what the eight lanes of a quarter warp load lies in different banks
template <int HD>
__device__ __forceinline__ uint32_t key_at(int row, int chunk) {
  return HD == 128 ? row * 128 + ((chunk ^ ((row & 1) << 2)) << 4) : row * 64 + (chunk << 4);
}
template <int HD>
__device__ __forceinline__ uint32_t value_at(int row, int chunk) {
  if (HD == 128) return row * 128 + ((chunk ^ (row & 6)) << 4);
  return (row >> 1) * 128 + (((((row & 1) << 2) | chunk) ^ (row & 6)) << 4);
}

template <typename T, int HD, int MT, bool WIDE>
__global__ void __launch_bounds__(Layout<HD, MT, sizeof(T) == 4, WIDE>::kThreads, Layout<HD, MT, sizeof(T) == 4, WIDE>::kCtas)
quant_attend_kernel(QAttendArgs a, int tiles_each, int score_bytes) {
  constexpr bool F32 = sizeof(T) == 4;
  using L = Layout<HD, MT, F32, WIDE>;
  constexpr int kDepth = L::kDepth, kWarps = L::kWarps, kThreads = L::kThreads;
  extern __shared__ __align__(128) uint8_t smem[];
  const uint32_t sbase = tc::smem_u32(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  const int ranks = gridDim.x, rank = blockIdx.x, head = blockIdx.y % a.c.n_heads, group = blockIdx.y / a.c.n_heads, seq = blockIdx.z;
  grid_dep_launch();
  grid_dep_wait();

  const int share = a.n_heads / a.c.n_heads, rows = a.n_rows * share;
  int len = a.cache_len[seq], n = a.row_count ? a.row_count[seq] : a.n_rows, first = a.first_slot ? a.first_slot[seq] : 0;
  uint32_t bits = 0;
  if (n < 0 || n > a.n_rows) { bits |= VVS_DEV_BAD_ARG; n = 0; }
  if (len < 0 || len > a.c.cap - n) { bits |= VVS_DEV_CACHE_OVERFLOW; len = 0; n = 0; }
  if (first < 0 || first > len) { bits |= VVS_DEV_BAD_ARG; first = first < 0 ? 0 : len; }
  if (bits && rank == 0 && blockIdx.y == 0 && tid == 0) atomicOr(a.status, bits);
  const int end = len + n;

  const size_t item = (size_t)seq * a.c.n_heads + head;
  const uint8_t* keys = a.c.k + item * a.c.cap * HD;
  const uint8_t* values = a.c.v + item * a.c.cap * HD;
  const float* k_scale = a.c.k_scale + item * (a.c.cap >> a.c.block_log2);
  const float* v_scale = a.c.v_scale + item * (a.c.cap >> a.c.block_log2);
  // slices of 16 keys: this CTA's are s0 .. s1 - 1, this warp's every kWarps-th of them
  const int all0 = first >> 4, all1 = (end + 15) >> 4, each = (all1 - all0 + ranks - 1) / ranks;
  const int s0 = min(all1, all0 + rank * each), s1 = min(all1, s0 + each);
  const uint32_t ring = sbase + L::kRingAt + warp * L::kRing;

  // a slice is 16 HD bytes side by side; of each 512 of them a lane copies 16
  const uint32_t key_to = ring + key_at<HD>(lane / (HD / 16), lane % (HD / 16));
  const uint32_t value_to = ring + L::kTile + value_at<HD>(lane / (HD / 16), lane % (HD / 16));
  // of heads of 128, 512 bytes are four rows: every other four have their pieces in another order
  const uint32_t value_odd = HD == 128 ? ring + L::kTile + value_at<HD>(lane / 8 + 4, lane % 8) - 512 : value_to;
  const uint8_t *keys_at = keys + lane * 16, *values_at = values + lane * 16;
  const float* scale_at = lane ? v_scale : k_scale;
  auto request = [&](int slice, uint32_t at, bool with_values) {
    const size_t from = (size_t)slice * (16 * HD);
    const int left = end - (slice << 4);
    if (left >= 16 && (slice << 4) >= first) {
      copy16<0, 0>(key_to + at, keys_at + from);
      copy16<512, 512>(key_to + at, keys_at + from);
      if (HD == 128) {
        copy16<1024, 1024>(key_to + at, keys_at + from);
        copy16<1536, 1536>(key_to + at, keys_at + from);
      }
      if (with_values) {
        copy16<0, 0>(value_to + at, values_at + from);
        copy16<512, 512>(value_odd + at, values_at + from);
        if (HD == 128) {
          copy16<1024, 1024>(value_to + at, values_at + from);
          copy16<1536, 1536>(value_odd + at, values_at + from);
        }
      }
    } else {                                                              // zeros in the place of slots that no row sees
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) {
        const int row = i * (512 / HD) + lane / (HD / 16);
        const bool there = row < left && (slice << 4) + row >= first;
        const size_t off = there ? from + i * 512 : from;
        copy16_some(key_to + at + i * 512, keys_at + off, there ? 16 : 0);
        if (with_values) copy16_some((i & 1 ? value_odd : value_to) + at + i * 512, values_at + off, there ? 16 : 0);
      }
    }
    if (lane < 2) copy4(ring + at + 2 * L::kTile + 4 * lane, scale_at + (slice >> (a.c.block_log2 - 4)));
  };
  // where this lane's operands lie in a slice: keys g and 8 + g, pieces c and 4 + c; values 2c, 2c + 1, 8 + 2c, 9 + 2c, piece g
  const uint32_t k_lane[2] = {ring + key_at<HD>(g, c), HD == 128 ? ring + key_at<HD>(g, 4 + c) : 0u};
  const uint32_t v_lane = ring + L::kTile + (HD == 128 ? value_at<HD>(2 * c, g) : value_at<HD>(2 * c, g >> 1) + (g & 1) * 8);
  const uint32_t v_next = HD == 128 ? v_lane + 128 : ring + L::kTile + value_at<HD>(2 * c + 1, g >> 1) + (g & 1) * 8;

  // scores of the rows whose weights are summed stay in shared memory, if those of all of the CTA's keys fit
  const int score_ld = quant_score_ld((s1 - s0) * 16);

  for (int tile = group * tiles_each; tile < min((group + 1) * tiles_each, (rows + L::kRows - 1) / L::kRows); ++tile) {
    const int r0 = tile * L::kRows, summed = min(L::kRows, min(a.mass_rows, n) * share - r0);      // rows 0 .. summed - 1 of the tile
    const bool keep_scores = summed > 0 && quant_score_bytes(summed, (s1 - s0) * 16) <= score_bytes;
    float* held = reinterpret_cast<float*>(smem + L::kScoreAt);
    // requests of the first slices travel while the queries are laid out
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d) {
      if (s0 + warp + d * kWarps < s1) request(s0 + warp + d * kWarps, d * L::kSlot, true);
      tc::cp_async_commit();
    }

    // ---- queries: scaled rows as A fragments -------------------------------------------------------------------------------------
    for (int r = warp; r < L::kRows; r += kWarps) {
      const int row = r0 + r, t = row / share, h = head * share + row % share;
      const bool live = row < rows && t < n;
      constexpr int kEach = HD / 32;                         // elements of a lane: kEach * lane ..
      float x[kEach];
      float top = 0.f;
      const T* src = static_cast<const T*>(a.q.data) + seq * a.q.seq + (int64_t)t * a.q.row + h * a.q.head;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        x[e] = live ? static_cast<float>(src[kEach * lane + e]) : 0.f;
        top = fmaxf(top, fabsf(x[e]));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      // a power of two (its biased exponent) that brings the largest element to [2^13, 2^14)
      const int e_top = (int)(__float_as_uint(top) >> 23);
      const int up = top > 0.f && e_top < 255 ? min(max(127 + 13 + 127 - e_top, 1), 253) : 127;
      const float mul = __uint_as_float((uint32_t)up << 23);
      if (lane == 0) reinterpret_cast<float*>(smem + L::kFacAt)[r] = __uint_as_float((uint32_t)(254 - up) << 23);
      // element d = 64 h' + 16 c' + 4 s' + e is k-step 4 h' + s', lane column c', register pair e / 2, half e % 2
#pragma unroll
      for (int e = 0; e < kEach; e += 2) {
        const int d = kEach * lane + e, step = (d >> 6) * 4 + ((d >> 2) & 3), col = (d >> 4) & 3, pair = (d >> 1) & 1;
        const int reg = ((r >> 3) & 1) + 2 * pair, to_lane = (r & 7) * 4 + col;
        float lo = x[e] * mul, hi = x[e + 1] * mul;
#pragma unroll
        for (int piece = 0; piece < L::kQ; ++piece) {
          const uint32_t w = pack_f16(lo, hi);
          reinterpret_cast<uint32_t*>(smem + L::kQAt)[(((piece * MT + (r >> 4)) * L::kSteps + step) * 32 + to_lane) * 4 + reg] = w;
          const float2 f = halves_to_float2(w);
          lo -= f.x;
          hi -= f.y;
        }
      }
    }
    __syncthreads();
    float fac[MT][2];                       // log2(e) scale / what the row was multiplied by
    int t_of[MT][2];
    uint32_t sees[MT][2];                   // rows of the block that a row sees, where they are named
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = mt * 16 + g + 8 * i, row = r0 + r, t = row / share;
        fac[mt][i] = reinterpret_cast<const float*>(smem + L::kFacAt)[r] * a.scale * kLog2e;
        t_of[mt][i] = row < rows && t < n ? t : -1;
        sees[mt][i] = a.visible && t_of[mt][i] >= 0 ? a.visible[(size_t)seq * a.n_rows + t] : 0u;
      }
    auto visible = [&](int mt, int i, int slot) {
      const int j = slot - len, t = t_of[mt][i];
      if (j < 0) return slot >= first && t >= 0;
      if (j >= n || t < 0) return false;
      return a.visible ? ((sees[mt][i] >> j) & 1u) != 0u : j <= t;
    };
    uint32_t q_held[L::kQRegs ? MT * L::kSteps : 1][4];
    if (L::kQRegs) {
#pragma unroll
      for (int i = 0; i < MT * L::kSteps; ++i) {
        const uint4 t = lds128<0>(sbase + L::kQAt + i * 512 + lane * 16);
        q_held[L::kQRegs ? i : 0][0] = t.x; q_held[L::kQRegs ? i : 0][1] = t.y;
        q_held[L::kQRegs ? i : 0][2] = t.z; q_held[L::kQRegs ? i : 0][3] = t.w;
      }
    }
    // scores of a slice, unscaled; s[mt][nt]: keys 8 nt + 2c, + 1 of rows g, g + 8
    auto scores = [&](uint32_t slot, float (&s)[MT][2][4]) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[mt][nt][e] = 0.f;
#pragma unroll
      for (int h = 0; h < HD / 64; ++h) {
        const uint4 k4[2] = {lds128<0>(k_lane[h] + slot), lds128<8 * HD>(k_lane[h] + slot)};
#pragma unroll
        for (int st = 0; st < 4; ++st) {
          uint32_t b[2][2];
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) {
            const uint32_t w = st == 0 ? k4[nt].x : st == 1 ? k4[nt].y : st == 2 ? k4[nt].z : k4[nt].w;
            b[nt][0] = from_e4m3x2(w);
            b[nt][1] = from_e4m3x2(w >> 16);
          }
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int piece = L::kQ - 1; piece >= 0; --piece) {
              uint32_t q[4];
              if (L::kQRegs) {
#pragma unroll
                for (int e = 0; e < 4; ++e) q[e] = q_held[L::kQRegs ? mt * L::kSteps + 4 * h + st : 0][e];
              } else {
                const uint4 t = lds128<0>(sbase + L::kQAt + ((piece * MT + mt) * L::kSteps + 4 * h + st) * 512 + lane * 16);
                q[0] = t.x; q[1] = t.y; q[2] = t.z; q[3] = t.w;
              }
#pragma unroll
              for (int nt = 0; nt < 2; ++nt) mma_f16(s[mt][nt], q, b[nt][0], b[nt][1]);
            }
        }
      }
    };

    // ---- the cache, once -------------------------------------------------------------------------------------------------------------
    float m[MT][2], l[MT][2], o[MT][HD / 8][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int i = 0; i < 2; ++i) { m[mt][i] = -CUDART_INF_F; l[mt][i] = 0.f; }
#pragma unroll
      for (int j = 0; j < HD / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[mt][j][e] = 0.f;
    }
    // the weights of a slice's scores, in place of them; MASKED: some row does not see some key; apart: weights may vanish that count
    auto weights = [&](auto masked, bool apart, int slice, float ks, float lv, float inv_vs, float (&s)[MT][2][4], uint32_t (&p)[L::kP][MT][4]) {
      constexpr bool MASKED = decltype(masked)::value;
      const int slot0 = slice << 4;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if (keep_scores) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (mt * 16 + g + 8 * i >= summed) continue;
            const float f = fac[mt][i] * ks;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
              float x[2] = {s[mt][nt][2 * i] * f, s[mt][nt][2 * i + 1] * f};
              if (MASKED) {
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  if (!visible(mt, i, slot0 + 8 * nt + 2 * c + e)) x[e] = -CUDART_INF_F;
              }
              *reinterpret_cast<float2*>(held + (mt * 16 + g + 8 * i) * score_ld + (slice - s0) * 16 + 8 * nt + 2 * c) = make_float2(x[0], x[1]);
            }
          }
        }
        // log2 of the weights at the row's reference; a row that sees nothing yet has none
        bool passes = false;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float f = fac[mt][i] * ks, by = lv + kShift - (m[mt][i] == -CUDART_INF_F ? 0.f : m[mt][i]);
          float top = -CUDART_INF_F;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float& v = s[mt][e >> 1][2 * i + (e & 1)];
            v = fmaf(v, f, by);
            if (MASKED && !visible(mt, i, slot0 + 8 * (e >> 1) + 2 * c + (e & 1))) v = -CUDART_INF_F;
            top = fmaxf(top, v);
          }
          passes = passes || top > kShift + kSlack || (m[mt][i] == -CUDART_INF_F && top > -CUDART_INF_F);
        }
        if (__any_sync(0xffffffffu, passes || apart)) {      // some row's reference moves up to the slice's largest score
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float top = fmaxf(fmaxf(s[mt][0][2 * i], s[mt][0][2 * i + 1]), fmaxf(s[mt][1][2 * i], s[mt][1][2 * i + 1]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const bool none = m[mt][i] == -CUDART_INF_F;
            const float up = none ? top - kShift : fmaxf(top - kShift, 0.f);       // what the reference rises by (from 0 where there was none)
            if (up == -CUDART_INF_F) continue;
            const float alpha = none ? 0.f : ex2(-up);
            m[mt][i] = none ? up : m[mt][i] + up;
            l[mt][i] = none ? 0.f : times_ex2(l[mt][i], -up);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[mt][e >> 1][2 * i + (e & 1)] -= up;
#pragma unroll
            for (int j = 0; j < HD / 8; ++j) {
              o[mt][j][2 * i] *= alpha;
              o[mt][j][2 * i + 1] *= alpha;
            }
            if (apart) {
              const float gone = (gone_weight(s[mt][0][2 * i]) + gone_weight(s[mt][0][2 * i + 1])) +
                                 (gone_weight(s[mt][1][2 * i]) + gone_weight(s[mt][1][2 * i + 1]));
              l[mt][i] = fmaf(gone, inv_vs * kGoneDown, l[mt][i]);
            }
          }
          __syncwarp();
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = ex2(s[mt][e >> 1][2 * i + (e & 1)]);
          l[mt][i] = fmaf((v[0] + v[1]) + (v[2] + v[3]), inv_vs, l[mt][i]);
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) {
            p[0][mt][i + 2 * nt] = pack_f16(v[2 * nt], v[2 * nt + 1]);
            if (F32) {
              const float2 hi = halves_to_float2(p[0][mt][i + 2 * nt]);
              p[L::kP - 1][mt][i + 2 * nt] = pack_f16(v[2 * nt] - hi.x, v[2 * nt + 1] - hi.y);
            }
          }
        }
      }
    };
    bool apart = false;                     // a scale was met that is not an ordinary one
    uint32_t at = 0, ahead = (kDepth - 1) * L::kSlot;
    for (int slice = s0 + warp; slice < s1; slice += kWarps) {
      tc::cp_async_wait<kDepth - 2>();
      __syncwarp();
      const float ks = lds32<2 * L::kTile>(ring + at), vs = lds32<2 * L::kTile + 4>(ring + at);
      float s[MT][2][4];
      scores(at, s);
      const float lv = __log2f(vs), inv_vs = __frcp_rn(vs);
      apart = apart || odd_scale(vs);
      uint32_t p[L::kP][MT][4];
      if ((slice << 4) >= first && (slice << 4) + 16 <= len)
        weights(std::false_type{}, apart, slice, ks, lv, inv_vs, s, p);
      else
        weights(std::true_type{}, apart, slice, ks, lv, inv_vs, s, p);
      // values: this lane's keys are 2c, 2c + 1, 8 + 2c, 9 + 2c, its columns g * HD / 8 ..
      uint32_t w[4][HD / 32];
      if (HD == 128) {
        const uint4 t[4] = {lds128<0>(v_lane + at), lds128<0>(v_next + at), lds128<8 * HD>(v_lane + at), lds128<8 * HD>(v_next + at)};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          w[kk][0] = t[kk].x; w[kk][1] = t[kk].y; w[kk][HD / 32 - 2] = t[kk].z; w[kk][HD / 32 - 1] = t[kk].w;
        }
      } else {
        const uint2 t[4] = {lds64<0>(v_lane + at), lds64<0>(v_next + at), lds64<8 * HD>(v_lane + at), lds64<8 * HD>(v_next + at)};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) { w[kk][0] = t[kk].x; w[kk][1] = t[kk].y; }
      }
#pragma unroll
      for (int wi = 0; wi < HD / 32; ++wi) {
        uint32_t b[2][4];
#pragma unroll
        for (int kp = 0; kp < 2; ++kp) {
          const uint32_t x = __byte_perm(w[2 * kp][wi], w[2 * kp + 1][wi], 0x5140), y = __byte_perm(w[2 * kp][wi], w[2 * kp + 1][wi], 0x7362);
          b[kp][0] = from_e4m3x2(x);
          b[kp][1] = from_e4m3x2(x >> 16);
          b[kp][2] = from_e4m3x2(y);
          b[kp][3] = from_e4m3x2(y >> 16);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int piece = L::kP - 1; piece >= 0; --piece) mma_f16(o[mt][4 * wi + j], p[piece][mt], b[0][j], b[1][j]);
      }
      __syncwarp();
      if (slice + (kDepth - 1) * kWarps < s1) request(slice + (kDepth - 1) * kWarps, ahead, true);
      tc::cp_async_commit();
      ahead = at;
      at = at == (kDepth - 1) * L::kSlot ? 0u : at + L::kSlot;
    }
    tc::cp_async_wait<0>();
    __syncwarp();

    // ---- the warps' sums, then the ranks' -----------------------------------------------------------------------------------------------
    float* part = reinterpret_cast<float*>(smem + L::kRingAt + warp * L::kRing);
    float* ml = reinterpret_cast<float*>(smem + L::kMlAt);
    float* tot = reinterpret_cast<float*>(smem + L::kTotAt);
    float* lse2 = reinterpret_cast<float*>(smem + L::kLseAt);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        l[mt][i] += __shfl_xor_sync(0xffffffffu, l[mt][i], 1);
        l[mt][i] += __shfl_xor_sync(0xffffffffu, l[mt][i], 2);
        const int r = mt * 16 + g + 8 * i;
        if (c == 0) {
          ml[(warp * L::kRows + r) * 2] = m[mt][i];
          ml[(warp * L::kRows + r) * 2 + 1] = l[mt][i];
        }
        // columns c * HD / 4 + 0 .. HD / 8 - 1 (elements 0 and 2), + HD / 8 .. (elements 1 and 3)
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int j = 0; j < HD / 8; j += 4)
            *reinterpret_cast<float4*>(part + r * HD + c * (HD / 4) + half * (HD / 8) + j) =
                make_float4(o[mt][j][2 * i + half], o[mt][j + 1][2 * i + half], o[mt][j + 2][2 * i + half], o[mt][j + 3][2 * i + half]);
      }
    __syncthreads();
    constexpr int kVecs = L::kRows * HD / 4;
    for (int v = tid; v < kVecs; v += kThreads) {
      const int r = v / (HD / 4);
      float top = -CUDART_INF_F;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml[(w * L::kRows + r) * 2]);
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      float total = 0.f, low = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float mw = ml[(w * L::kRows + r) * 2], f = mw == -CUDART_INF_F ? 0.f : ex2(mw - top);
        const float4 x = reinterpret_cast<const float4*>(smem + L::kRingAt + w * L::kRing)[v];
        sum.x = fmaf(x.x, f, sum.x); sum.y = fmaf(x.y, f, sum.y); sum.z = fmaf(x.z, f, sum.z); sum.w = fmaf(x.w, f, sum.w);
        total = fmaf(ml[(w * L::kRows + r) * 2 + 1], f, total);
        low = fminf(low, mw == -CUDART_INF_F ? 0.f : mw - top);
      }
      if (low < -100.f) {
        total = 0.f;
#pragma unroll 1
        for (int w = 0; w < kWarps; ++w) {
          const float mw = ml[(w * L::kRows + r) * 2];
          total = add_times_ex2(total, ml[(w * L::kRows + r) * 2 + 1], mw == -CUDART_INF_F ? 0.f : mw - top);
        }
      }
      reinterpret_cast<float4*>(smem + L::kRingAt)[v] = sum;              // (of warp 0's sums this thread reads no other)
      if (v % (HD / 4) == 0) { tot[2 * r] = top; tot[2 * r + 1] = total; }
    }
    if (ranks > 1) tc::cluster_sync(); else __syncthreads();
    const uint32_t tot_at = sbase + L::kTotAt, sum_at = sbase + L::kRingAt;
    for (int v = rank * kThreads + tid; v < kVecs; v += ranks * kThreads) {
      const int r = v / (HD / 4), row = r0 + r;
      if (row >= rows) break;
      const int t = row / share, h = head * share + row % share;
      float top = -CUDART_INF_F;
      for (int k = 0; k < ranks; ++k) top = fmaxf(top, tc::ld_cluster_f32(tot_at + 8 * r, k));
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      float total = 0.f;
      for (int k = 0; k < ranks; ++k) {
        const float mk = tc::ld_cluster_f32(tot_at + 8 * r, k), f = mk == -CUDART_INF_F ? 0.f : ex2(mk - top);
        const float4 x = tc::ld_cluster_f4(sum_at + 16 * v, k);
        sum.x = fmaf(x.x, f, sum.x); sum.y = fmaf(x.y, f, sum.y); sum.z = fmaf(x.z, f, sum.z); sum.w = fmaf(x.w, f, sum.w);
        const float lk = tc::ld_cluster_f32(tot_at + 8 * r + 4, k);
        total = mk == -CUDART_INF_F || mk - top > -100.f ? fmaf(lk, f, total) : add_times_ex2(total, lk, mk - top);
      }
      const bool some = t < n && !(total == 0.f);            // (a NaN among the queries is an answer of NaN)
      const float inv = some ? 1.f / total : 0.f;
      float x[4] = {sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv};
      if (!some) x[0] = x[1] = x[2] = x[3] = 0.f;
      store4(static_cast<T*>(a.out.data) + seq * a.out.seq + (int64_t)t * a.out.row + h * a.out.head + v % (HD / 4) * 4, x);
      if (a.lse && v % (HD / 4) == 0)
        a.lse[((size_t)seq * a.n_rows + t) * a.n_heads + h] = some ? (top - kShift + log2f(total)) / kLog2e : -CUDART_INF_F;
    }

    // ---- weights of this CTA's keys ---------------------------------------------------------------------------------------------------
    if (a.mass_rows > 0) {
      if (tid < L::kRows) {
        float top = -CUDART_INF_F, total = 0.f;
        for (int k = 0; k < ranks; ++k) top = fmaxf(top, tc::ld_cluster_f32(tot_at + 8 * tid, k));
        for (int k = 0; k < ranks; ++k) {
          const float mk = tc::ld_cluster_f32(tot_at + 8 * tid, k);
          const float lk = tc::ld_cluster_f32(tot_at + 8 * tid + 4, k);
          total = add_times_ex2(total, lk, mk == -CUDART_INF_F ? 0.f : mk - top);
        }
        lse2[tid] = total == 0.f ? CUDART_INF_F : top - kShift + log2f(total);
      }
    }
    if (ranks > 1) tc::cluster_sync(); else __syncthreads();              // the other ranks have read this one's sums
    if (a.mass_rows > 0) {
      const bool begin = tile == 0;
      float* mass = a.c.mass + item * a.c.cap;
      // slots before the first that is seen only lose
      if (begin && a.mass_decay != 1.f)
        for (int slot = rank * kThreads + tid; slot < all0 * 16 && slot < end; slot += ranks * kThreads)
          mass[slot] = a.mass_decay == 0.f ? 0.f : a.mass_decay * mass[slot];
      const float decay = begin ? a.mass_decay : 1.f;
      if (keep_scores || summed <= 0) {
        const int n_keys = begin || summed > 0 ? min((s1 - s0) * 16, end - s0 * 16) : 0;
        constexpr int kTogether = 8;                                      // keys of a thread whose weights so far travel together
        for (int key0 = tid; key0 < n_keys; key0 += kTogether * kThreads) {
          float was[kTogether], sum[kTogether];
#pragma unroll
          for (int j = 0; j < kTogether; ++j) {
            const int key = key0 + j * kThreads;
            was[j] = decay != 0.f && key < n_keys ? mass[s0 * 16 + key] : 0.f;
            sum[j] = 0.f;
          }
          for (int r = 0; r < summed; ++r) {
            const float by = lse2[r];
            if (by == CUDART_INF_F) continue;
#pragma unroll
            for (int j = 0; j < kTogether; ++j)
              if (key0 + j * kThreads < n_keys) sum[j] += ex2(held[r * score_ld + key0 + j * kThreads] - by);
          }
#pragma unroll
          for (int j = 0; j < kTogether; ++j)
            if (key0 + j * kThreads < n_keys) mass[s0 * 16 + key0 + j * kThreads] = decay == 0.f ? sum[j] : fmaf(decay, was[j], sum[j]);
        }
        __syncthreads();
        continue;
      }
      float sub[MT][2];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 2; ++i) sub[mt][i] = t_of[mt][i] >= 0 && t_of[mt][i] < a.mass_rows ? lse2[mt * 16 + g + 8 * i] : CUDART_INF_F;
#pragma unroll
      for (int d = 0; d < kDepth - 1; ++d) {
        if (s0 + warp + d * kWarps < s1) request(s0 + warp + d * kWarps, d * L::kSlot, false);
        tc::cp_async_commit();
      }
      at = 0;
      ahead = (kDepth - 1) * L::kSlot;
      for (int slice = s0 + warp; slice < s1; slice += kWarps) {
        tc::cp_async_wait<kDepth - 2>();
        __syncwarp();
        const float ks = lds32<2 * L::kTile>(ring + at);
        float s[MT][2][4];
        scores(at, s);
        const int slot0 = slice << 4;
        const bool whole = slot0 >= first && slot0 + 16 <= len;
        float sum[4] = {0.f, 0.f, 0.f, 0.f}, was[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = slot0 + 8 * (e >> 1) + 2 * c + (e & 1);
          was[e] = lane < 4 && key < end && decay != 0.f ? mass[key] : 0.f;
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float f = fac[mt][i] * ks;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float w = ex2(fmaf(s[mt][e >> 1][2 * i + (e & 1)], f, -sub[mt][i]));
              if (sub[mt][i] != CUDART_INF_F && (whole || visible(mt, i, slot0 + 8 * (e >> 1) + 2 * c + (e & 1)))) sum[e] += w;
            }
          }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 4);
          sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 8);
          sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 16);
        }
        if (lane < 4) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = slot0 + 8 * (e >> 1) + 2 * c + (e & 1);
            if (key < end) mass[key] = decay == 0.f ? sum[e] : fmaf(decay, was[e], sum[e]);
          }
        }
        __syncwarp();
        if (slice + (kDepth - 1) * kWarps < s1) request(slice + (kDepth - 1) * kWarps, ahead, false);
        tc::cp_async_commit();
        ahead = at;
        at = at == (kDepth - 1) * L::kSlot ? 0u : at + L::kSlot;
      }
      tc::cp_async_wait<0>();
      __syncthreads();
    }
  }
}

template <typename T, int HD, int MT, bool WIDE>
int launch_kernel_of(const QAttendArgs& a, int tiles_each, int groups, int ranks, int slices, cudaStream_t s) {
  using L = Layout<HD, MT, sizeof(T) == 4, WIDE>;
  // Shared memory for the scores of summed rows, where all of a CTA's keys fit (a call that says less of its lengths than they are walks
  // the keys again).  More ranks than the device has room for, to make them fit, cost more than the second walk: 32 sequences of nine
  // rows behind 900 to 2380 keys 179 us so, 347 with sixteen ranks in the place of one.
  const int mass_rows = a.mass_rows < a.n_rows ? a.mass_rows : a.n_rows, share = a.n_heads / a.c.n_heads;
  const int summed = (long long)mass_rows * share < L::kRows ? mass_rows * share : L::kRows;
  const long long want = quant_score_bytes(summed, (slices + ranks - 1) / ranks * 16);
  const int score_bytes = want <= L::kScoreBytes ? (int)want : 0;
  auto kernel = quant_attend_kernel<T, HD, MT, WIDE>;
  if (ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), L::kBytes + L::kScoreBytes) != cudaSuccess) return VVS_ERR_CUDA;
  if (ranks > 8 && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return VVS_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ranks, a.c.n_heads * groups, a.c.n_seqs);
  cfg.blockDim = dim3(L::kThreads);
  cfg.dynamicSmemBytes = L::kBytes + score_bytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ranks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, a, tiles_each, score_bytes) == cudaSuccess ? VVS_OK : VVS_ERR_CUDA;
}

template <typename T, int HD, int MT>
int launch_tiles(const QAttendArgs& a, cudaStream_t s) {
  using L = Layout<HD, MT, sizeof(T) == 4, false>;
  using W = Layout<HD, MT, sizeof(T) == 4, true>;
  const int rows = a.n_rows * (a.n_heads / a.c.n_heads), tiles = (rows + L::kRows - 1) / L::kRows;
  // the weights' sums of a key are added by one thread: a CTA goes through all tiles of rows then
  const int tiles_each = a.mass_rows > 0 ? tiles : 1, groups = (tiles + tiles_each - 1) / tiles_each;
  const long long items = (long long)a.c.n_seqs * a.c.n_heads * groups;
  const int slices = ((a.max_len > 0 && a.max_len < a.c.cap ? a.max_len : a.c.cap) + 15) / 16;
  int ranks = 1;
  while (ranks < 16 && items * ranks * 2 <= 2LL * a.n_sms && slices >= 2 * ranks * L::kWarps) ranks *= 2;
  // Items that the device holds at once: CTAs that fill an SM, as many for an item as lets all items be there together, where an item gets as
  // many warps so.  A token behind 31K keys: 8 cached heads of 128 43.4 -> 30.0 us, 4 of 64 29.0 -> 13.8; 40 of 64 behind 3K keys 16.3 -> 10.1,
  // nine rows behind 311 11.4 -> 9.5 (the same number of warps, no cluster).  A slice is enough for a warp: with two at least, a token behind
  // 900 keys of 16 cached heads of 128 takes 12.1 instead of 10.7.
  if (items <= a.n_sms && slices >= W::kWarps) {
    auto kernel = quant_attend_kernel<T, HD, MT, true>;
    if (ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), W::kBytes + W::kScoreBytes) != cudaSuccess) return VVS_ERR_CUDA;
    const int* there = resident_clusters(reinterpret_cast<const void*>(kernel), W::kThreads, W::kBytes + W::kScoreBytes);
    if (!there) return VVS_ERR_CUDA;
    int wide = 0;
    for (int c = 1; c <= kMaxCluster && slices >= c * W::kWarps; ++c)
      if (there[c] >= items) wide = c;
    if (wide > 0 && wide * W::kWarps >= ranks * L::kWarps) return launch_kernel_of<T, HD, MT, true>(a, tiles_each, groups, wide, slices, s);
  }
  return launch_kernel_of<T, HD, MT, false>(a, tiles_each, groups, ranks, slices, s);
}

template <typename T, int HD>
int launch_hd(const QAttendArgs& a, cudaStream_t s) {
  const int rows = a.n_rows * (a.n_heads / a.c.n_heads);
  // Many rows of bf16 contexts: the kernel with 128 of them a tile.  Two trees of 27 rows x 4 heads behind 31K keys 79 us against 158 here (four
  // tiles of 32 rows turn every key four times), with their first rows' weights summed 163 against 447; 36 rows 75 against 101.  Up to 32 rows
  // only where its items are on the device at once and no weights are summed: 20 rows, 300 to 500 keys, 140 items 13.0 us against 15.2,
  // 160 items 20.6 against 18.2; 100 items behind 300 keys, weights summed, 17.8 against 13.5.  Summed rows have to lie in its first
  // tile.  (Rows by 2^32 / share: exact up to 2^20 rows of 4096 heads.)
  const long long items = (long long)a.c.n_seqs * a.c.n_heads, share = rows / a.n_rows;
  const long long summed = (a.mass_rows < a.n_rows ? a.mass_rows : a.n_rows) * share;
  if (sizeof(T) == 2 && summed <= 128 && share <= 4096 && (rows > 32 || (rows > 16 && items <= a.n_sms && a.mass_rows == 0)))
    return launch_quant_attend_rows(a, s);
  return rows <= 16 ? launch_tiles<T, HD, 1>(a, s) : launch_tiles<T, HD, 2>(a, s);
}

}  // namespace

template <typename T>
int launch_quant_attend(const QAttendArgs& a, cudaStream_t s) {
  return a.c.hd == 64 ? launch_hd<T, 64>(a, s) : launch_hd<T, 128>(a, s);
}
template int launch_quant_attend<float>(const QAttendArgs&, cudaStream_t);
template int launch_quant_attend<__nv_bfloat16>(const QAttendArgs&, cudaStream_t);

}  // namespace vvs
