// Attention over the 8-bit cache for many query rows of a cached head (bf16 contexts): both products on tcgen05.
//
// The mathematics is that of the kernel for few rows: out = (sum_j w_j cv_j) / (sum_j w_j / V_b), w_j = 2^(a_j - m), queries as halves
// times a power of two, weights as halves.  A row's reference m moves only when its weights of a tile add up to more than kMost, so that
// none of them is beyond it: a sum costs less than a maximum beside it.
//
// A stream has a tile of 128 rows and a share of the keys, 64 at a time.  Codes arrive by bulk copies.  Two warps turn the keys' into halves,
// two the values', in the 128-byte swizzled layout of the operands (keys K-major; values, as the same rows, MN-major), and issue
// S = Q K^T (twice 64 columns of tensor memory) and O += P V.  Four warps have a row per lane: its 64 scores come from tensor memory and
// its weights go back over them as halves, P is an operand there.  A row's sums need no other lane.  A CTA has two streams, each with
// its own keys and tensor memory, and one copy of the queries; a cluster's CTAs have more shares.  The shares' sums are joined
// through distributed shared memory, in their order.
//
// Weights summed for eviction (of rows of the first tile): with the rows' sums at hand the keys go through the first product once more, and
// the lanes' weights are added over the rows by shuffles.
//
// Two sequences, 27 rows x 4 heads over each of 8 cached heads of 128, 30K to 33K keys: 79 us, 350 TFLOP/s (bytes alone are 20 us, the products
// 16); 163 with the first rows' weights summed.  A stream needs 3000 cycles for 64 keys: the row's lane 1200 for its powers, sums and halves, the
// rest waits of one stage for another; an SM issues in 42 of 100 cycles, its tensor pipe is busy in 30.  Clusters of six CTAs with an SM each are
// what the device holds for 16 items at once: 96 of 148 SMs work (eight: 15 clusters, one waits for another to end, 124 us).  One CTA with one
// stream, twice on an SM, is packed on half of the SMs: 135 us.
#include <type_traits>

#include "quant_cache.cuh"
#include "tc_common.cuh"

namespace vvs {

namespace {

constexpr int kKeys = 64;                       // keys of a tile
constexpr int kRows = 128;
constexpr int kSoft = 4, kConv = 4;             // warps
constexpr int kStreams = 2;                     // of a CTA, with keys, tensor memory and eight warps each
constexpr int kThreads = 32 * kStreams * (kSoft + kConv);
constexpr int kMaxRanks = 16;
constexpr int kTilesEach = 2;                   // of a stream, at least, where several share the keys
constexpr float kShift = 7.f, kMost = 32768.f;   // log2 of a weight at the reference; the most a row's weights of a tile may add up to
constexpr float kLog2e = 1.4426950408889634f;

// two float32 at a time
__device__ __forceinline__ uint64_t pair_of(float x, float y) { return (uint64_t)__float_as_uint(x) | (uint64_t)__float_as_uint(y) << 32; }
__device__ __forceinline__ float low_of(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float high_of(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint4 halves_of(uint32_t a, uint32_t b) {
  return make_uint4(from_e4m3x2(a), from_e4m3x2(a >> 16), from_e4m3x2(b), from_e4m3x2(b >> 16));
}
// bytes side by side, 16-byte aligned, counted on a barrier
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(tc::smem_u32(bar)) : "memory");
}
// O (+)= P V for 64 keys, P in tensor memory (8 columns for 16 keys), V's rows of 128 bytes MN-major (16 keys are 2048 bytes).  Called by a
// converged warp, of which one lane issues.
__device__ __forceinline__ void mma_values(uint32_t d, uint32_t p, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred e, p, q;\n\t.reg .b64 b;\n\t.reg .b32 x, y;\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 q, %5, %5;\n\t"
      "mov.b64 b, {%2, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t"
      "add.u32 x, %1, 8;\n\tadd.u32 y, %2, 128;\n\tmov.b64 b, {y, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %3, q;\n\t"
      "add.u32 x, %1, 16;\n\tadd.u32 y, %2, 256;\n\tmov.b64 b, {y, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %3, q;\n\t"
      "add.u32 x, %1, 24;\n\tadd.u32 y, %2, 384;\n\tmov.b64 b, {y, %5};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %3, q;\n\t}"
      ::"r"(d), "r"(p), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(tc::kDescHiSw128) : "memory");
}
__device__ __forceinline__ float2 ld_cluster_f2(uint32_t local_addr, uint32_t rank) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(tc::mapa(local_addr, rank)) : "memory");
  return v;
}
// 32 columns of this lane's row; there after tmem_arrived
__device__ __forceinline__ void tmem_request32(uint32_t taddr, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
        "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
        "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
        "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr) : "memory");
}
template <int N>
__device__ __forceinline__ void tmem_arrived(float* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+f"(v[i]));
}
__device__ __forceinline__ void tmem_store16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <int HD>
struct Layout {
  static constexpr int kStages = HD == 128 ? 2 : 4;             // tiles of codes on their way
  static constexpr int kCodes = kKeys * HD;                     // bytes of a tile's keys, or values
  static constexpr int kHalves = 2 * kCodes;                    // ... as halves: HD / 64 slabs of [64][128 bytes]
  static constexpr int kSlab = kKeys * 128;
  static constexpr int kQAt = 0;                                // HD / 64 slabs of [128][128 bytes]
  // of each stream: keys and values as halves, codes; its sums [128][HD] in the place of all of them
  static constexpr int kStreamAt = kRows * HD * 2;
  static constexpr int kValueAt = kHalves, kCodeAt = 2 * kHalves;
  static constexpr int kStreamBytes = kCodeAt + kStages * 2 * kCodes;
  static constexpr int kTotAt = kStreamAt + kStreams * kStreamBytes;      // [stream][128][2] its rows' references and sums
  static constexpr int kFacAt = kTotAt + kStreams * kRows * 8;  // [128] what scores are multiplied by
  static constexpr int kPartAt = kFacAt + kRows * 4;            // [stream][2][4 warps][64] summed weights of a tile's keys
  static constexpr int kBarAt = kPartAt + kStreams * 2 * kSoft * kKeys * 4;
  static constexpr int kBars = 2 * kStages + 8;                 // of a stream; and one of the queries
  static constexpr int kNeed = kBarAt + (kStreams * kBars + 1) * 8 + 16 + 1024;       // (the base is brought to a multiple of 1024)
  // One CTA on an SM: it has all of the tensor memory, S twice 64 columns and O HD of them for each stream.  And none of another kernel that
  // multiplies there: two clusters that hold tensor memory on one SM each and wait for it on the other's would wait forever.  (Its 512 threads have
  // all registers of an SM beside that, 128 each.)
  static constexpr int kBytes = kNeed < 200 * 1024 ? 200 * 1024 : kNeed;
  static constexpr int kColumns = 512, kStreamColumns = 256, kOut = 2 * kKeys;
  static_assert(kStreamBytes >= kRows * HD * 4, "a stream's sums fit");
  static_assert(kBytes <= 227 * 1024, "shared memory");
};

// MASS: weights are summed, of rows of the first tile alone
template <int HD, bool MASS>
__global__ void __launch_bounds__(kThreads, 1) quant_attend_rows_kernel(QAttendArgs a, uint32_t share_inv) {
  using L = Layout<HD>;
  constexpr int kStages = L::kStages;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sbase = tc::smem_u32(smem);
  const int tid = threadIdx.x, lane = tid & 31, stream = tid / (32 * (kSoft + kConv)), warp = (tid >> 5) % (kSoft + kConv);     // (of the stream)
  float2* tot = reinterpret_cast<float2*>(smem + L::kTotAt) + stream * kRows;
  float* fac_of = reinterpret_cast<float*>(smem + L::kFacAt);
  uint64_t* all_bars = reinterpret_cast<uint64_t*>(smem + L::kBarAt);
  uint64_t *q_full = all_bars + kStreams * L::kBars, *bars = all_bars + stream * L::kBars;
  uint64_t* code_full = bars;                                   // [keys, values][stage]
  uint64_t *s_full = bars + 2 * kStages, *p_full = s_full + 2, *o_done = s_full + 4, *drained = s_full + 6;       // .., [keys, values]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(q_full + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const uint32_t stream_at = L::kStreamAt + stream * L::kStreamBytes;

  const int ranks = gridDim.x, rank = blockIdx.x, seq = blockIdx.z, head = blockIdx.y % a.c.n_heads, tile = blockIdx.y / a.c.n_heads;
  if (tid == 0) {
    for (int i = 0; i < kStreams * L::kBars; ++i) tc::mbar_init(&all_bars[i], (unsigned)(i % L::kBars - 2 * kStages - 2) < 2u ? kSoft : 1);
    tc::mbar_init(q_full, kThreads / 32);
    tc::fence_barrier_init();
    *abort_flag = 0;
  }
  if (tid < 32) {
    tc::tmem_alloc(tmem_slot, L::kColumns);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  grid_dep_launch();
  grid_dep_wait();

  const int share = a.n_heads / a.c.n_heads, rows = a.n_rows * share, r0 = tile * kRows;
  int len = a.cache_len[seq], n = a.row_count ? a.row_count[seq] : a.n_rows, first = a.first_slot ? a.first_slot[seq] : 0;
  uint32_t bits = 0;
  if (n < 0 || n > a.n_rows) { bits |= VVS_DEV_BAD_ARG; n = 0; }
  if (len < 0 || len > a.c.cap - n) { bits |= VVS_DEV_CACHE_OVERFLOW; len = 0; n = 0; }
  if (first < 0 || first > len) { bits |= VVS_DEV_BAD_ARG; first = first < 0 ? 0 : len; }
  if (bits && rank == 0 && blockIdx.y == 0 && tid == 0) atomicOr(a.status, bits);
  const int end = len + n;
  // tiles from the slice of 16 slots that holds the first one; this stream's are t0 .. t0 + nt - 1
  const int shares = ranks * kStreams, from = first & ~15, tiles = (end - from + kKeys - 1) / kKeys, each = (tiles + shares - 1) / shares;
  const int t0 = min(tiles, (rank * kStreams + stream) * each), nt = min(tiles, t0 + each) - t0;
  const size_t item = (size_t)seq * a.c.n_heads + head;
  const uint32_t tmem = *tmem_slot + stream * L::kStreamColumns, t_out = tmem + L::kOut;
  // row of the item -> row of the block (share_inv: 2^32 / share, rounded up; rows are far below 2^32 / share)
  auto t_row = [&](int row) { return share == 1 ? row : (int)__umulhi((uint32_t)row, share_inv); };

  // codes: keys by the first two of the warps that turn them, values by the others.  The first tiles' travel while the queries are laid out.
  const bool converts = warp >= kSoft, of_keys = warp < kSoft + kConv / 2;
  constexpr int kTurn = 16 * kConv;                             // threads of a kind
  const int at = tid % (2 * kTurn) % kTurn;                     // .. of them
  const uint8_t* codes = (of_keys ? a.c.k : a.c.v) + item * a.c.cap * HD;
  uint64_t* full = code_full + (of_keys ? 0 : kStages);
  const uint32_t code_at = stream_at + L::kCodeAt + (of_keys ? 0 : kStages * L::kCodes);
  auto request = [&](int i) {
    const int slot0 = from + (t0 + (MASS && i >= nt ? i - nt : i)) * kKeys, st = i % kStages;       // (i >= nt: the keys once more)
    const uint32_t bytes = min(kKeys, a.c.cap - slot0) * HD;
    tc::mbar_expect_tx(&full[st], bytes);
    bulk_load(sbase + code_at + st * L::kCodes, codes + (size_t)slot0 * HD, bytes, &full[st]);
  };
  if (converts && at == 0)
    for (int i = 0; i < min(nt, kStages); ++i) request(i);

  // Barriers by tile i: s_full, p_full and o_done have one for even and one for odd tiles.  A wait for tile i comes when tile i - 2 is known
  // to have passed and tile i + 2 cannot have: S of i is made after O of i - 2 was added, P of i needs S of i, O of i needs P of i.
  bool ok = true;

  // ---- queries: rows times a power of two, as halves; every warp has eight ---------------------------------------------------------
  {
    constexpr int kEach = HD / 32, kWarps = kThreads / 32, kBatch = kRows / kWarps;     // elements of a lane; rows of a warp
    uint32_t raw[kBatch][kEach / 2];
#pragma unroll
    for (int m = 0; m < kBatch; ++m) {
      const int row = r0 + (tid >> 5) + m * kWarps, t = t_row(row), h = head * share + row - t * share;
#pragma unroll
      for (int e = 0; e < kEach / 2; ++e) raw[m][e] = 0u;
      if (row < rows && t < n) {
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q.data) + seq * a.q.seq + (int64_t)t * a.q.row + h * a.q.head + kEach * lane;
        if (kEach == 4) {
          const uint2 w = *reinterpret_cast<const uint2*>(src);
          raw[m][0] = w.x;
          raw[m][kEach / 2 - 1] = w.y;
        } else {
          raw[m][0] = *reinterpret_cast<const uint32_t*>(src);
        }
      }
    }
    float top[kBatch];
#pragma unroll
    for (int m = 0; m < kBatch; ++m) {
      top[m] = 0.f;
#pragma unroll
      for (int e = 0; e < kEach / 2; ++e)
        top[m] = fmaxf(top[m], fmaxf(fabsf(__uint_as_float(raw[m][e] << 16)), fabsf(__uint_as_float(raw[m][e] & 0xffff0000u))));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int m = 0; m < kBatch; ++m) top[m] = fmaxf(top[m], __shfl_xor_sync(0xffffffffu, top[m], o));
#pragma unroll
    for (int m = 0; m < kBatch; ++m) {
      const int r = (tid >> 5) + m * kWarps;
      // a power of two (its biased exponent) that brings the largest element to [2^13, 2^14)
      const int e_top = (int)(__float_as_uint(top[m]) >> 23);
      const int up = top[m] > 0.f && e_top < 255 ? min(max(127 + 13 + 127 - e_top, 1), 253) : 127;
      const float mul = __uint_as_float((uint32_t)up << 23);
      if (lane == 0) fac_of[r] = __uint_as_float((uint32_t)(254 - up) << 23) * a.scale * kLog2e;
      uint32_t w[kEach / 2];
#pragma unroll
      for (int e = 0; e < kEach / 2; ++e) w[e] = pack_f16(__uint_as_float(raw[m][e] << 16) * mul, __uint_as_float(raw[m][e] & 0xffff0000u) * mul);
      const int d = kEach * lane;
      uint8_t* at = smem + L::kQAt + (d >> 6) * (kRows * 128) + r * 128 + ((((d & 63) >> 3) ^ (r & 7)) << 4) + (d & 7) * 2;
      if (kEach == 4) *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[kEach / 2 - 1]);
      else *reinterpret_cast<uint32_t*>(at) = w[0];
    }
    tc::fence_proxy_async();
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(q_full);
  }

  // This thread's 16 codes (piece of a row) of each kRowsEach rows.  Eight lanes side by side read 16-byte words of eight different groups of
  // banks and write such: two rows, four pieces each, for heads of 128 of different slabs.
  constexpr int kPieces = HD / 16, kTimes = kKeys * kPieces / kTurn, kRowsEach = kTurn / kPieces;
  const int c_row = HD == 128 ? at / 16 * 2 + ((at >> 2) & 1) : at / kPieces;
  const int c_piece = HD == 128 ? (((at >> 2) ^ (at >> 3)) & 1) * 4 + (at & 3) : at % kPieces;
  uint8_t* to = smem + stream_at + (of_keys ? 0 : L::kValueAt) + (c_piece >> 2) * L::kSlab + c_row * 128;
  // (kRowsEach is a multiple of 8)
  uint8_t *to_lo = to + (((2 * (c_piece & 3)) ^ (c_row & 7)) << 4), *to_hi = to + (((2 * (c_piece & 3) + 1) ^ (c_row & 7)) << 4);
  const bool issues = warp == (of_keys ? kSoft : kSoft + kConv / 2);
  // Keys or values of tile i; the next ones' codes are asked for up to tile last - 1.  Both warps of a kind have the same answer, whether to go on:
  // one that gave up comes to the barrier all the same.
  auto turn_codes = [&](int i, int last) {
    const int slot0 = from + (t0 + i) * kKeys, st = i % kStages;
    ok = ok && tc::warp_wait_or_abort(&full[st], (i / kStages) & 1, abort_flag);
    uint4 w[kTimes];
#pragma unroll
    for (int x = 0; x < kTimes; ++x)
      w[x] = *reinterpret_cast<const uint4*>(smem + code_at + st * L::kCodes + (x * kRowsEach + c_row) * HD + c_piece * 16);
    if (!of_keys && (slot0 < first || slot0 + kKeys > end)) {
      // values of slots that no row sees are zeros, whatever lies there
#pragma unroll
      for (int x = 0; x < kTimes; ++x) {
        const int slot = slot0 + c_row + x * kRowsEach;
        if (slot < first || slot >= end) w[x] = make_uint4(0, 0, 0, 0);
      }
    }
    // the halves before these have been read: by S, by O of the tile before
    if (i > 0)
      ok = ok && (of_keys ? tc::warp_wait_or_abort(&s_full[(i - 1) & 1], ((i - 1) >> 1) & 1, abort_flag)
                          : tc::warp_wait_or_abort(&o_done[(i - 1) & 1], ((i - 1) >> 1) & 1, abort_flag));
#pragma unroll
    for (int x = 0; x < kTimes; ++x) {
      *reinterpret_cast<uint4*>(to_lo + x * kRowsEach * 128) = halves_of(w[x].x, w[x].y);
      *reinterpret_cast<uint4*>(to_hi + x * kRowsEach * 128) = halves_of(w[x].z, w[x].w);
    }
    tc::fence_proxy_async();
    ok = tc::named_bar_all(1 + 2 * stream + (of_keys ? 0 : 1), kTurn, ok);
    if (ok && at == 0 && i + kStages < last) request(i + kStages);
    return ok;
  };
  auto multiply_keys = [&](int i) {
    tc::tc_fence_after();
    constexpr uint32_t idesc = (1u << 4) | ((kKeys >> 3) << 17) | ((kRows >> 4) << 24);
#pragma unroll
    for (int h = 0; h < HD / 64; ++h)
      tc::mma_bf16_k64(tmem + (i & 1) * kKeys, tc::desc_lo_sw128(sbase + L::kQAt + h * (kRows * 128)),
                       tc::desc_lo_sw128(sbase + stream_at + h * L::kSlab), idesc, h);      // (the descriptor's types are halves)
    tc::mma_commit_elect(&s_full[i & 1]);
  };
  // products and copies under way, of tiles i and behind, still read and write
  auto give_up = [&](int i, int last) {
    *abort_flag = 1;
    if (issues) {
      tc::mma_commit_elect(&drained[of_keys ? 0 : 1]);
      tc::mbar_wait(&drained[of_keys ? 0 : 1], 0);
    }
    if (at == 0)
      for (int x = i; x < min(last, i + kStages); ++x) tc::mbar_wait(&full[x % kStages], (x / kStages) & 1);
    __syncwarp();
  };

  // a row's lane: what it sees, and the tiles' scales
  const int mine = (warp % kSoft) * 32 + lane, my_t = t_row(r0 + mine);
  const bool live = r0 + mine < rows && my_t < n;
  // rows of the block that this one sees: a bit of each, or those up to itself
  const uint32_t sees = !converts && a.visible && live ? a.visible[(size_t)seq * a.n_rows + my_t] & (n < 32 ? (1u << n) - 1u : 0xffffffffu) : 0u;
  const int upto = !live ? first : a.visible ? len : len + my_t + 1;
  // the slots that it sees of 64 from slot0 on: first .. upto - 1, and of the block's those of `sees`
  auto seen = [&](int slot0) {
    const int lo = min(max(first - slot0, 0), 64), hi = min(max(upto - slot0, 0), 64), by = len - slot0;
    uint64_t bits = (hi < 64 ? (1ULL << hi) - 1ULL : ~0ULL) & (lo < 64 ? ~0ULL << lo : 0ULL);
    if (by > -32 && by < 64) bits |= by >= 0 ? (uint64_t)sees << by : (uint64_t)(sees >> -by);
    return bits;
  };
  const uint32_t t_lane = (uint32_t)((warp % kSoft) * 32) << 16;
  const float* scale_at = (lane & 4 ? a.c.v_scale : a.c.k_scale) + item * (a.c.cap >> a.c.block_log2);
  // lanes 0 to 3 have the scales of the keys of a tile's four slices, lanes 4 to 7 those of their values
  auto scale_of_tile = [&](int i) { return scale_at[min(from + (t0 + i) * kKeys + 16 * (lane & 3), end - 1) >> a.c.block_log2]; };
  auto scores = [&](uint32_t from_at, float (&s)[kKeys]) {
    tmem_request32(from_at, s);
    tmem_request32(from_at + 32, s + 32);
    tmem_arrived<kKeys>(s);
  };

  if (converts) {                                               // ---- codes to halves, products: two warps for keys and S, two for values and O
    int i = 0;
#pragma unroll 1
    for (; i < nt; ++i) {
      if (!turn_codes(i, nt)) break;
      if (!issues) continue;
      if (of_keys) {                                            // S of tile i, where P of tile i - 2 was
        if (i == 0) ok = tc::warp_wait_or_abort(q_full, 0, abort_flag);
        if (i > 1) ok = tc::warp_wait_or_abort(&o_done[i & 1], ((i - 2) >> 1) & 1, abort_flag);
        if (ok) multiply_keys(i);
      } else {
        ok = tc::warp_wait_or_abort(&p_full[i & 1], (i >> 1) & 1, abort_flag);
        if (!ok) continue;
        tc::tc_fence_after();
        constexpr uint32_t idesc = (1u << 4) | (1u << 16) | ((HD >> 3) << 17) | ((kRows >> 4) << 24);       // B is MN-major
        mma_values(t_out, tmem + (i & 1) * kKeys, (((sbase + stream_at + L::kValueAt) >> 4) & 0x3FFFu) | ((uint32_t)(L::kSlab >> 4) << 16), idesc, i > 0);
        tc::mma_commit_elect(&o_done[i & 1]);
      }
    }
    if (!ok) give_up(i, nt);
  } else {                                                      // ---- scores to weights, sums
    float next_scale = nt > 0 ? scale_of_tile(0) : 1.f;
    bool odd = false;                                           // this lane has met a scale of values that is not an ordinary one
    float m = -CUDART_INF_F, l = 0.f;                           // (a row that is not there has neither)
    if (nt > 0) ok = tc::warp_wait_or_abort(q_full, 0, abort_flag);
    const float fac = fac_of[mine];
    // log2 of the weights in the place of a tile's scores; MASKED: some row does not see some key
    auto logs = [&](auto masked, int i, float ks, float lv, float (&s)[kKeys]) {
      const uint64_t bits = decltype(masked)::value ? seen(from + (t0 + i) * kKeys) : 0ULL;
      const float base = kShift - (m == -CUDART_INF_F ? 0.f : m);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float f = fac * __shfl_sync(0xffffffffu, ks, q), by = base + __shfl_sync(0xffffffffu, lv, 4 + q);
        const uint64_t f2 = pair_of(f, f), by2 = pair_of(by, by);
#pragma unroll
        for (int e = 16 * q; e < 16 * q + 16; e += 2) {
          const uint64_t v = fma2(pair_of(s[e], s[e + 1]), f2, by2);
          s[e] = low_of(v);
          s[e + 1] = high_of(v);
          if (decltype(masked)::value) {
            if (!(bits >> e & 1)) s[e] = -CUDART_INF_F;
            if (!(bits >> e & 2)) s[e + 1] = -CUDART_INF_F;
          }
        }
      }
    };
    // the weights; returned is their sum, in by_value that of weights over the values' scales
    auto powers = [&](float inv_vs, float (&s)[kKeys], float& by_value) {
      float all = 0.f;
      by_value = 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint64_t x = 0, y = 0;
#pragma unroll
        for (int e = 16 * q; e < 16 * q + 16; e += 4) {
#pragma unroll
          for (int j = 0; j < 4; ++j) s[e + j] = ex2(s[e + j]);
          x = add2(x, pair_of(s[e], s[e + 1]));
          y = add2(y, pair_of(s[e + 2], s[e + 3]));
        }
        x = add2(x, y);
        const float part = low_of(x) + high_of(x);
        all += part;
        by_value = fmaf(part, __shfl_sync(0xffffffffu, inv_vs, 4 + q), by_value);
      }
      return all;
    };
#pragma unroll 1
    for (int i = 0; i < nt && ok; ++i) {
      const float scale = next_scale, lv = __log2f(scale), inv_vs = __frcp_rn(scale);
      if (i + 1 < nt) next_scale = scale_of_tile(i + 1);
      ok = tc::warp_wait_or_abort(&s_full[i & 1], (i >> 1) & 1, abort_flag);
      if (!ok) break;
      tc::tc_fence_after();
      const uint32_t at = tmem + t_lane + (i & 1) * kKeys;
      float s[kKeys], by_value;
      const int slot0 = from + (t0 + i) * kKeys;
      const bool whole = slot0 >= first && slot0 + kKeys <= len;
      auto tile_logs = [&]() {
        scores(at, s);
        if (whole) logs(std::false_type{}, i, scale, lv, s);
        else logs(std::true_type{}, i, scale, lv, s);
      };
      tile_logs();
      // A sum of at most kMost has no weight beyond it.  Else, and where a row has no reference yet, rows' references move up to their largest
      // score of the tile, which lies in tensor memory still.  And where scales of values lie far apart.
      const bool none = live && m == -CUDART_INF_F;
      odd = odd || ((lane & 4) && odd_scale(scale));
      bool moves = __any_sync(0xffffffffu, none || odd);
      if (!moves) {
        const float all = powers(inv_vs, s, by_value);
        moves = __any_sync(0xffffffffu, live && !(all <= kMost));
        if (moves) tile_logs();
      }
      if (moves) {
        float top = -CUDART_INF_F;
#pragma unroll
        for (int e = 0; e < kKeys; e += 2) top = fmaxf(top, fmaxf(s[e], s[e + 1]));
        float up = none ? top - kShift : fmaxf(top - kShift, 0.f), alpha = 1.f;
        if (up != -CUDART_INF_F && live) {
          alpha = none ? 0.f : ex2(-up);
          m = none ? up : m + up;
          l = none ? 0.f : times_ex2(l, -up);
        } else {
          up = 0.f;
        }
#pragma unroll
        for (int e = 0; e < kKeys; ++e) s[e] -= up;
        if (__any_sync(0xffffffffu, odd)) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float inv = __shfl_sync(0xffffffffu, inv_vs, 4 + q) * kGoneDown;
            float gone = 0.f;
#pragma unroll
            for (int e = 16 * q; e < 16 * q + 16; ++e) gone += gone_weight(s[e]);
            l = fmaf(gone, inv, l);
          }
        }
        if (i > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
          ok = tc::warp_wait_or_abort(&o_done[(i - 1) & 1], ((i - 1) >> 1) & 1, abort_flag);
          if (!ok) break;
          tc::tc_fence_after();
#pragma unroll 1
          for (int j = 0; j < HD; j += 16) {
            float o[16];
            tc::tmem_ld16(t_out + t_lane + j, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] *= alpha;
            tmem_store16(t_out + t_lane + j, reinterpret_cast<const uint32_t*>(o));
          }
          tmem_stored();
        }
        powers(inv_vs, s, by_value);
      }
      l += by_value;
      uint32_t p[16];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = pack_f16(s[32 * half + 2 * e], s[32 * half + 2 * e + 1]);
        tmem_store16(at + 16 * half, p);
      }
      tmem_stored();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&p_full[i & 1]);
    }
    if (nt > 0) ok = ok && tc::warp_wait_or_abort(&o_done[(nt - 1) & 1], ((nt - 1) >> 1) & 1, abort_flag);
    tc::tc_fence_after();
    // the stream's sums: 16-byte pieces of row r in places that differ by r % 8
    float4* sum = reinterpret_cast<float4*>(smem + stream_at) + mine * (HD / 4);
    tot[mine] = make_float2(m, l);
    if (!ok) *abort_flag = 1;
    if (ok) {
#pragma unroll 1
      for (int j = 0; j < HD && nt > 0; j += 32) {
        float o[32];
        tmem_request32(t_out + t_lane + j, o);
        tmem_arrived<32>(o);
#pragma unroll
        for (int e = 0; e < 32; e += 4) sum[((j + e) / 4) ^ (mine & 7)] = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
      }
    }
    tc::tc_fence_before();
  }
  __syncwarp();
  if (ranks > 1) tc::cluster_sync(); else __syncthreads();
  tc::tc_fence_after();
  const bool failed = *abort_flag != 0;
  if (failed && tid == 0) atomicOr(a.status, VVS_DEV_TIMEOUT);

  // ---- the shares' sums, in their order; what a thread reads of the other CTAs travels together -------------------------------------------------
  const uint32_t tot_at = sbase + L::kTotAt, sum_at = sbase + L::kStreamAt;
#pragma unroll 1
  for (int v = rank * kThreads + tid; v < kRows * (HD / 4) && !failed; v += ranks * kThreads) {
    const int r = v / (HD / 4), piece = v % (HD / 4), row = r0 + r;
    if (row >= rows) break;
    const int t = t_row(row), h = head * share + row - t * share;
    constexpr int kTogether = 4;
    float2 ml[kMaxRanks][kStreams];
    float top = -CUDART_INF_F;
#pragma unroll
    for (int k = 0; k < kMaxRanks; ++k)
#pragma unroll
      for (int st = 0; st < kStreams; ++st) {
        ml[k][st] = make_float2(-CUDART_INF_F, 0.f);
        if (k < ranks) ml[k][st] = ld_cluster_f2(tot_at + (st * kRows + r) * 8, k);
      }
#pragma unroll
    for (int k = 0; k < kMaxRanks; ++k)
#pragma unroll
      for (int st = 0; st < kStreams; ++st) top = fmaxf(top, ml[k][st].x);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    float total = 0.f, low = 0.f;
#pragma unroll
    for (int k0 = 0; k0 < kMaxRanks; k0 += kTogether) {
      if (k0 >= ranks) break;
      float4 x[kTogether][kStreams];
#pragma unroll
      for (int k = 0; k < kTogether; ++k)
#pragma unroll
        for (int st = 0; st < kStreams; ++st) {
          x[k][st] = make_float4(0.f, 0.f, 0.f, 0.f);
          // (a share without keys has written no sums)
          if (ml[k0 + k][st].y != 0.f) x[k][st] = tc::ld_cluster_f4(sum_at + st * L::kStreamBytes + 16 * (r * (HD / 4) + (piece ^ (r & 7))), k0 + k);
        }
#pragma unroll
      for (int k = 0; k < kTogether; ++k)
#pragma unroll
        for (int st = 0; st < kStreams; ++st) {
          const float2 m = ml[k0 + k][st];
          const float f = m.x == -CUDART_INF_F ? 0.f : ex2(m.x - top);
          const float4 y = x[k][st];
          sum.x = fmaf(y.x, f, sum.x); sum.y = fmaf(y.y, f, sum.y); sum.z = fmaf(y.z, f, sum.z); sum.w = fmaf(y.w, f, sum.w);
          total = fmaf(m.y, f, total);
          low = fminf(low, m.x == -CUDART_INF_F ? 0.f : m.x - top);
        }
    }
    if (low < -100.f) {
      total = 0.f;
#pragma unroll
      for (int k = 0; k < kMaxRanks; ++k)
#pragma unroll
        for (int st = 0; st < kStreams; ++st) total = add_times_ex2(total, ml[k][st].y, ml[k][st].x == -CUDART_INF_F ? 0.f : ml[k][st].x - top);
    }
    const bool some = t < n && !(total == 0.f);                // (a NaN among the queries is an answer of NaN)
    const float inv = some ? 1.f / total : 0.f;
    float x[4] = {sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv};
    if (!some) x[0] = x[1] = x[2] = x[3] = 0.f;
    store4(static_cast<__nv_bfloat16*>(a.out.data) + seq * a.out.seq + (int64_t)t * a.out.row + h * a.out.head + piece * 4, x);
    if (a.lse && piece == 0) a.lse[((size_t)seq * a.n_rows + t) * a.n_heads + h] = some ? (top - kShift + log2f(total)) / kLog2e : -CUDART_INF_F;
  }
  // log2 of a summed row's sum; of other rows, and of one that sees nothing, infinity
  const int summed = MASS && tile == 0 ? min(kRows, min(a.mass_rows, n) * share) : 0;
  float sub = CUDART_INF_F;
  if (MASS && !converts && mine < summed) {
    float2 ml[kMaxRanks][kStreams];
    float top = -CUDART_INF_F, total = 0.f;
#pragma unroll
    for (int k = 0; k < kMaxRanks; ++k)
#pragma unroll
      for (int st = 0; st < kStreams; ++st) {
        ml[k][st] = make_float2(-CUDART_INF_F, 0.f);
        if (k < ranks) ml[k][st] = ld_cluster_f2(tot_at + (st * kRows + mine) * 8, k);
        top = fmaxf(top, ml[k][st].x);
      }
#pragma unroll
    for (int k = 0; k < kMaxRanks; ++k)
#pragma unroll
      for (int st = 0; st < kStreams; ++st)
        total = add_times_ex2(total, ml[k][st].y, ml[k][st].x == -CUDART_INF_F ? 0.f : ml[k][st].x - top);
    if (!(total == 0.f)) sub = top - kShift + log2f(total);
  }
  if (MASS) tc::fence_proxy_async();                            // codes come where the sums were
  __syncwarp();
  if (ranks > 1) tc::cluster_sync(); else __syncthreads();      // the other ranks have read this one's sums

  // ---- weights of the keys: the keys once more, by the CTAs of the first rows --------------------------------------------------------------------
  if (MASS && tile == 0 && !failed) {
    float* mass = a.c.mass + item * a.c.cap;
    const float decay = a.mass_decay;
    // slots before the first tile only lose; where no row is summed, all do
    for (int slot = rank * kThreads + tid; slot < (summed > 0 ? min(from, end) : end); slot += ranks * kThreads)
      if (decay != 1.f) mass[slot] = decay == 0.f ? 0.f : decay * mass[slot];
    if (summed > 0) {
      const int last = 2 * nt;
      if (converts) {
        if (of_keys) {
          if (at == 0)
            for (int i = nt; i < min(last, nt + kStages); ++i) request(i);
          int i = nt;
#pragma unroll 1
          for (; i < last; ++i) {
            if (!turn_codes(i, last)) break;
            if (!issues) continue;
            if (i >= nt + 2) ok = tc::warp_wait_or_abort(&p_full[i & 1], ((i - 2) >> 1) & 1, abort_flag);      // S of tile i - 2 has been read
            if (ok) multiply_keys(i);
          }
          if (!ok) give_up(i, last);
        }
      } else {
        const int warps = (summed + 31) / 32;                   // that have summed rows
        const float fac = fac_of[mine];
        float* part = reinterpret_cast<float*>(smem + L::kPartAt) + stream * 2 * kSoft * kKeys;
        float next_scale = nt > 0 ? scale_of_tile(0) : 1.f;
#pragma unroll 1
        for (int j = 0; j < nt; ++j) {
          const int i = nt + j, slot0 = from + (t0 + j) * kKeys;
          const float scale = next_scale;
          if (j + 1 < nt) next_scale = scale_of_tile(j + 1);
          float was[2] = {0.f, 0.f};
          if (warp == 0 && decay != 0.f)
#pragma unroll
            for (int x = 0; x < 2; ++x)
              if (slot0 + x * 32 + lane < end) was[x] = mass[slot0 + x * 32 + lane];
          ok = ok && tc::warp_wait_or_abort(&s_full[i & 1], (i >> 1) & 1, abort_flag);
          tc::tc_fence_after();
          if (warp < warps) {
            float s[kKeys];
            scores(tmem + t_lane + (i & 1) * kKeys, s);
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&p_full[i & 1]);
            const uint64_t bits = sub == CUDART_INF_F ? 0ULL : seen(slot0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const float f = fac * __shfl_sync(0xffffffffu, scale, q);
              float v[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] = (bits >> (16 * q + e)) & 1 ? ex2(fmaf(s[16 * q + e], f, -sub)) : 0.f;
              tc::warp_sums<16>(v, lane);
              if (!(lane & 1)) part[((i & 1) * kSoft + warp) * kKeys + 16 * q + tc::warp_sums_index<16>(lane)] = v[0];
            }
            // (of the part's two buffers, this one's were read before the barrier of the tile before)
            if (warps > 1) tc::named_bar_sync(5 + stream, 32 * warps);
            else __syncwarp();
            if (warp == 0) {
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                const int key = x * 32 + lane;
                float sum = 0.f;
                for (int w = 0; w < warps; ++w) sum += part[((i & 1) * kSoft + w) * kKeys + key];
                if (slot0 + key < end && ok) mass[slot0 + key] = decay == 0.f ? sum : fmaf(decay, was[x], sum);
              }
              __syncwarp();
            }
          } else if (lane == 0) {
            tc::mbar_arrive(&p_full[i & 1]);
          }
          __syncwarp();
        }
        if (!ok) *abort_flag = 1;
      }
    }
    __syncthreads();
    tc::tc_fence_after();
    if (tid == 0 && *abort_flag) atomicOr(a.status, VVS_DEV_TIMEOUT);
  }
  if (tid < 32) tc::tmem_dealloc(*tmem_slot, L::kColumns);
}

template <int HD, bool MASS>
int launch_hd(const QAttendArgs& a, cudaStream_t s) {
  using L = Layout<HD>;
  const int rows = a.n_rows * (a.n_heads / a.c.n_heads), row_tiles = (rows + kRows - 1) / kRows;
  const long long items = (long long)a.c.n_seqs * a.c.n_heads * row_tiles;
  const int tiles = ((a.max_len > 0 && a.max_len < a.c.cap ? a.max_len : a.c.cap) + kKeys - 1) / kKeys;
  const int share = a.n_heads / a.c.n_heads;
  const uint32_t share_inv = share == 1 ? 0u : (uint32_t)(((1ULL << 32) + share - 1) / share);
  auto kernel = quant_attend_rows_kernel<HD, MASS>;
  if (ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), L::kBytes) != cudaSuccess) return VVS_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = L::kBytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  const int* there = resident_clusters(reinterpret_cast<const void*>(kernel), kThreads, L::kBytes);
  if (!there) return VVS_ERR_CUDA;
  // the most CTAs for an item by which all items are there at once: a cluster more than that waits until another one has ended
  int ranks = 1;
  for (int c = 2; c <= kMaxRanks && tiles >= kTilesEach * kStreams * c; ++c)
    if (there[c] >= items) ranks = c;
  attr[0].val.clusterDim.x = ranks;
  cfg.numAttrs = 2;
  cfg.gridDim = dim3(ranks, a.c.n_heads * row_tiles, a.c.n_seqs);
  return cudaLaunchKernelEx(&cfg, kernel, a, share_inv) == cudaSuccess ? VVS_OK : VVS_ERR_CUDA;
}

}  // namespace

int launch_quant_attend_rows(const QAttendArgs& a, cudaStream_t s) {
  if (a.mass_rows > 0) return a.c.hd == 64 ? launch_hd<64, true>(a, s) : launch_hd<128, true>(a, s);
  return a.c.hd == 64 ? launch_hd<64, false>(a, s) : launch_hd<128, false>(a, s);
}

}  // namespace vvs
