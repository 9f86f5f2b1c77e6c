// The 8-bit product (block_matmul.cu has the formula) of many rows: pairs of CTAs (tcgen05.mma.cta_group::2, M = 256), tiles of 256 rows and
// 256 weights one after the other.
//
// Rows of the call lie on the M side here, so that a summing thread has one of them and weights of one block: its factor is one number
// a block of K, and a packed multiply-add takes two elements.  Each CTA stages its 128 rows and half of the tile's weights, 32 KB a block
// of K.  A block's sums go to tensor memory in two halves of 128 weights, twice each: sixteen warps take them from there and add them, times
// their factor, to 128 x 256 float32 sums in registers (64 of each thread's), one half while the tensor cores form the others.  Two warps
// bring the factors to shared memory some blocks ahead.  A tile's result leaves by bulk copies, while the next tile's sums begin.
//
// Bound by the summing warps: 690 cycles a block of K, where its MMAs take 512 and shared memory's fill from L2 575 (32 KB).  Four of them share a
// scheduler, whose slots are 60 % taken; a warp's own chain (wait, factor, eight loads of eight columns with four multiply-adds each, signal) is
// what lasts.  5460 rows of 4096 through 12288 weights: 284 us, 1.94 PFLOP/s, at the power cap (987 W, 1.3 GHz), 252 us before it is reached.
#include "block_matmul.cuh"
#include "block_plans.h"

namespace vvs {

using namespace bmm;

namespace {

constexpr int kSumWarps = 16, kThreads = 128 + kSumWarps * 32, kStages = 4, kTile = 256, kCols = 64;   // kCols: weights of a summing thread
constexpr int kBatch = 4, kBatches = 4;            // blocks whose factors are told of together; batches that lie in shared memory
constexpr uint32_t kStageBytes = 2 * kTileBytes, kHalfBytes = kTileBytes / 2, kOutBytes = 32 * 128;      // kOutBytes: of a summing warp
constexpr int kFactors = 2 * 128;                  // of a block: both halves, all rows
// (more than it needs: two clusters that hold tensor memory on one SM each and wait for it on the other's would wait forever)
constexpr int kSmemBytes = kMatmulPairSmem;
static_assert(kStages * kStageBytes + kSumWarps * kOutBytes + kBatches * kBatch * kFactors * 4 + 1024 <= kSmemBytes, "shared memory");
constexpr int kBand = 8;                           // tiles of rows that go through the weights together

// An arrival in another CTA, relaxed: what it tells of has been read from tensor memory, which tcgen05's fences order, or is told of by another
// barrier.  A release to the cluster waits for everything that the warp has under way, 1000 to 1600 cycles.
__device__ __forceinline__ void mbar_arrive_at(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ float ld_shared(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
// two sums, as the packed multiply-add takes them
typedef unsigned long long Two;
__device__ __forceinline__ Two two(float a, float b) {
  Two t;
  asm("mov.b64 %0, {%1, %2};" : "=l"(t) : "f"(a), "f"(b));
  return t;
}
__device__ __forceinline__ void one_and_one(Two t, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(t)); }
// Eight columns of the warp's lanes are added to their sums.  (Of sixteen at once the compiler moves a half of every pair to where the packed
// multiply-add finds it, on the pipe that it takes itself; of eight it does not.)
__device__ __forceinline__ void add_columns8(uint32_t taddr, Two* acc, Two ff) {
  asm volatile(
      "{\n\t.reg .b32 t<8>;\n\t.reg .b64 x;\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {t0,t1,t2,t3,t4,t5,t6,t7}, [%4];\n\t"
      "tcgen05.wait::ld.sync.aligned;\n\t"
      "mov.b64 x, {t0,t1};\n\tfma.rn.f32x2 %0, x, %5, %0;\n\tmov.b64 x, {t2,t3};\n\tfma.rn.f32x2 %1, x, %5, %1;\n\t"
      "mov.b64 x, {t4,t5};\n\tfma.rn.f32x2 %2, x, %5, %2;\n\tmov.b64 x, {t6,t7};\n\tfma.rn.f32x2 %3, x, %5, %3;\n\t}"
      : "+l"(acc[0]), "+l"(acc[1]), "+l"(acc[2]), "+l"(acc[3]) : "r"(taddr), "l"(ff) : "memory");
}
// sixteen bytes of a row
__device__ __forceinline__ void put_piece(uint8_t* to, const float (&y)[8]) {
  *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}
__device__ __forceinline__ void put_piece(uint8_t* to, const float (&y)[4]) { *reinterpret_cast<float4*>(to) = make_float4(y[0], y[1], y[2], y[3]); }
// shared -> global, 128 bytes of 32 rows
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* m, const void* src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];\n\tcp.async.bulk.commit_group;"
               ::"l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(src)), "r"(x), "r"(y) : "memory");
}

struct Tiles {
  int rows, outs;                                  // tiles of either
  __device__ __forceinline__ void place(int id, int& mt, int& nt) const {
    const int band = id / (kBand * outs), in = id - band * kBand * outs, high = min(kBand, rows - band * kBand);
    nt = in / high;
    mt = band * kBand + in - nt * high;
  }
};
// a place in a ring and the parity of the phase that is waited for there
template <int N>
struct Ring {
  uint32_t at = 0, par;
  __device__ explicit Ring(uint32_t parity) : par(parity) {}
  __device__ __forceinline__ void next() {
    if (++at == N) { at = 0; par ^= 1; }
  }
};

template <typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
block_matmul_pair_kernel(const __grid_constant__ MatmulParams p, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_a,
                         const __grid_constant__ CUtensorMap tm_out, Tiles tiles) {
  extern __shared__ uint8_t smem_raw[];
  // full: a stage of both CTAs, and their factors (in the first CTA).  done: its MMAs.  sum: a half's sums are there, free: they have been taken
  // (by both CTAs, in the first one).  ready: this CTA's factors of a batch
  __shared__ __align__(8) uint64_t full_bar[kStages], done_bar[kStages], sum_bar[2][2], free_bar[2][2], ready_bar[kBatches];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int s_abort;

  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* factors = reinterpret_cast<float*>(smem + kStages * kStageBytes + kSumWarps * kOutBytes);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int rank = (int)(blockIdx.x & 1), first = (int)(blockIdx.x >> 1), step = (int)(gridDim.x >> 1), n_tiles = tiles.rows * tiles.outs;
  // Blocks go in twos, for two places of sums that the code knows: behind an odd number comes one of zeros (the copies' fill, factors of nothing).
  const int nkb = (p.nkb + 1) & ~1;

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&full_bar[i], 1 + 4);              // the producer, two warps of either CTA with factors
      mbar_init(&done_bar[i], 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&sum_bar[0][i], 1);
      mbar_init(&free_bar[0][i], kSumWarps);       // half of either CTA's
    }
    for (int i = 0; i < kBatches; ++i) mbar_init(&ready_bar[i], 2);
    s_abort = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tm_w);
    tma_prefetch_desc(&tm_a);
    tma_prefetch_desc(&tm_out);
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  cluster_sync();                                  // both CTAs' barriers are ready
  const uint32_t tmem = tmem_slot;
  pdl_launch_dependents();
  pdl_wait();

  bool ok = true;                                  // (a wait that ran out is reported, and its warp does nothing more)
  if (warp == 0) {
    // ---- producer: this CTA's rows and its share of the weights, counted on the first CTA's barrier -----------------------------------
    Ring<kStages> st(1);
    int issued = 0;
    for (int id = first; id < n_tiles && ok; id += step) {
      int mt, nt;
      tiles.place(id, mt, nt);
      const int m0 = mt * kTile + rank * 128, n0 = nt * kTile + rank * 64;
      for (int kb = 0; kb < nkb; ++kb, ++issued) {
        if (issued >= kStages && !(ok = warp_wait_or_abort(&done_bar[st.at], st.par, &s_abort))) break;
        __syncwarp();
        if (elect_one()) {
          const uint32_t bar0 = mapa(smem_u32(&full_bar[st.at]), 0);
          uint8_t* to = smem + st.at * kStageBytes;
          if (rank == 0) mbar_expect_tx(&full_bar[st.at], 2 * kStageBytes);
          tma_load_pair_2d(to, &tm_a, bar0, kb * kQBlock, m0);
          tma_load_pair_2d(to + kTileBytes, &tm_w, bar0, kb * kQBlock, n0);
          tma_load_pair_2d(to + kTileBytes + kHalfBytes, &tm_w, bar0, kb * kQBlock, n0 + 128);
        }
        st.next();
      }
    }
    // The last stages' MMAs signal both CTAs too, and nobody else waits for that: no CTA leaves before it was told of them.
    for (int i = max(issued - kStages, 0); i < issued && ok; ++i) ok = warp_wait_or_abort(&done_bar[i % kStages], (i / kStages) & 1, &s_abort);
    if (!ok && rank == 0) {                        // nothing may be in flight when the pair leaves (bounded)
      for (int i = issued > kStages ? issued - kStages : 0; i < issued; ++i) mbar_wait(&full_bar[i % kStages], (i / kStages) & 1);
      __syncwarp();
    }
  } else if (warp == 1) {
    if (rank == 0) {
      // ---- MMA issuer of the pair -----------------------------------------------------------------------------------------------
      const uint32_t idesc = idesc_e4m3_f32(256, 128), lo0 = desc_lo_sw128(smem_u32(smem));
      Ring<kStages> st(0);
      uint32_t buf = 0, bpar = 1;
      int i = 0;
      for (int id = first; id < n_tiles && ok; id += step)
        for (int kb = 0; kb < nkb; ++kb, ++i) {
          ok = warp_wait_or_abort(&full_bar[st.at], st.par, &s_abort);
          const uint32_t a_lo = lo0 + st.at * (kStageBytes >> 4);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            ok = ok && (i < 2 || warp_wait_or_abort(&free_bar[h][buf], bpar, &s_abort));
            if (!ok) break;
            tc_fence_after();
            mma_e4m3_block<2>(tmem + buf * kTile + h * 128, a_lo, a_lo + ((kTileBytes + h * kHalfBytes) >> 4), idesc);
            commit_pair(&sum_bar[h][buf]);
          }
          if (!ok) break;
          commit_pair(&done_bar[st.at]);
          st.next();
          buf ^= 1;
          bpar ^= buf ^ 1;
        }
    }
  } else if (warp < 4) {
    // ---- factors: a thread has two rows, and both halves' weights ------------------------------------------------------------------
    // A second producer: no block's MMAs begin without its factors.  Their place is that of eight blocks before at least (a tile's last batch may
    // have two): the MMAs of four blocks before are done, which waited for the sums of six before to be taken.
    const int r0 = (warp - 2) * 32 + lane;
    Ring<kStages> st(1);
    int count = 0, batch = 0;
    for (int id = first; id < n_tiles && ok; id += step) {
      int mt, nt;
      tiles.place(id, mt, nt);
      const int row = mt * kTile + rank * 128 + r0;
      const bool there[2] = {row < p.m, row + 64 < p.m}, second = nt * kTile + 128 < p.n;
      const float* as[2] = {p.a_scale + (size_t)(there[0] ? row : 0) * p.nkb, p.a_scale + (size_t)(there[1] ? row + 64 : 0) * p.nkb};
      const float* ws[2] = {p.w_scale + (size_t)(2 * nt) * p.nkb, p.w_scale + (size_t)(2 * nt + second) * p.nkb};
      float a[2][kBatch], w[2][kBatch];
      auto request = [&](int kb) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            a[h][j] = there[h] && kb + j < p.nkb ? __ldg(as[h] + kb + j) : 0.f;     // rows that are not there: factors of nothing
            w[h][j] = kb + j < p.nkb ? __ldg(ws[h] + kb + j) : 0.f;
          }
      };
      request(0);
      for (int kb = 0; kb < nkb && ok; kb += kBatch) {
        float f[kBatch][4];
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
#pragma unroll
          for (int h = 0; h < 4; ++h) f[j][h] = a[h & 1][j] * w[h >> 1][j];
        request(kb + kBatch);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          if (kb + j >= nkb || !ok) break;
          if (count >= kStages && !(ok = warp_wait_or_abort(&done_bar[st.at], st.par, &s_abort))) break;
          float* to = factors + ((batch % kBatches) * kBatch + j) * kFactors + r0;
#pragma unroll
          for (int h = 0; h < 4; ++h) to[(h >> 1) * 128 + (h & 1) * 64] = f[j][h];
          __syncwarp();
          if (lane == 0) mbar_arrive_at(mapa(smem_u32(&full_bar[st.at]), 0));
          st.next();
          ++count;
        }
        if (!ok) break;
        if (lane == 0) mbar_arrive(&ready_bar[batch % kBatches]);
        ++batch;
      }
    }
  } else {
    // ---- sums: a thread has a row and 64 weights -------------------------------------------------------------------------------------
    const int group = (warp - 4) >> 2, half = group >> 1, quad = warp & 3;
    const uint32_t t_row = tmem + ((uint32_t)(quad * 32) << 16) + group * kCols;
    const uint32_t my_factor = smem_u32(factors) + (uint32_t)(half * 128 + quad * 32 + lane) * 4;
    const uint32_t ready0 = smem_u32(&ready_bar[0]), sum0 = smem_u32(&sum_bar[half][0]), free0 = mapa(smem_u32(&free_bar[half][0]), 0);
    uint32_t turn = 0, batch = 0;                  // pairs of blocks so far, and batches of factors
    for (int id = first; id < n_tiles && ok; id += step) {
      Two acc[kCols / 2];
#pragma unroll
      for (int j = 0; j < kCols / 2; ++j) acc[j] = 0;
#pragma unroll 1
      for (int kb = 0; kb < nkb; kb += 2, ++turn) {
        if (kb % kBatch == 0) {
          if (!(ok = warp_wait_lean(ready0 + batch % kBatches * 8, batch / kBatches & 1, &s_abort))) break;
          ++batch;
        }
        const uint32_t factor_at = my_factor + ((batch - 1) % kBatches * kBatch + kb % kBatch) * (kFactors * 4);
#pragma unroll
        for (int buf = 0; buf < 2; ++buf) {
          if (!(ok = warp_wait_lean(sum0 + buf * 8, turn & 1, &s_abort))) break;
          const float f = ld_shared(factor_at + buf * (kFactors * 4));
          tc_fence_after();
          const Two ff = two(f, f);
#pragma unroll
          for (int c = 0; c < kCols; c += 8) add_columns8(t_row + buf * kTile + c, acc + c / 2, ff);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_at(free0 + buf * 8);
        }
        if (!ok) break;
      }
      if (!ok) break;
      // ---- out: 128 bytes of each of the warp's rows at a time, swizzled as the bulk copy takes them -----------------------------------
      int mt, nt;
      tiles.place(id, mt, nt);
      const int row0 = mt * kTile + rank * 128 + quad * 32, n0 = nt * kTile + group * kCols;
      constexpr int kPiece = 16 / sizeof(T), kWide = 8 * kPiece;
      uint8_t* stage_out = smem + kStages * kStageBytes + (warp - 4) * kOutBytes;
#pragma unroll
      for (int c0 = 0; c0 < kCols; c0 += kWide) {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");     // the copy before has read what lies here
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float y[kPiece];
#pragma unroll
          for (int j = 0; j < kPiece; j += 2) one_and_one(acc[(c0 + i * kPiece + j) / 2], y[j], y[j + 1]);
          put_piece(stage_out + lane * 128 + ((i ^ (lane & 7)) << 4), y);
        }
        if (p.wide) {
          fence_proxy_async();
          __syncwarp();
          if (lane == 0 && row0 < p.m && n0 + c0 < p.n) tma_store_2d(&tm_out, stage_out, (n0 + c0) * (int)sizeof(T), row0);
        } else {                                   // rows that begin anywhere: element by element
          __syncwarp();
          for (int r = 0; r < 32 && row0 + r < p.m; ++r)
            for (int j = lane; j < kWide && n0 + c0 + j < p.n; j += 32) {
              const int piece = j / kPiece, in = j % kPiece;
              static_cast<T*>(p.out)[(size_t)(row0 + r) * p.out_row + n0 + c0 + j] =
                  reinterpret_cast<const T*>(stage_out + r * 128 + ((piece ^ (r & 7)) << 4))[in];
            }
          __syncwarp();
        }
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  if (!ok) {
    if (lane == 0) atomicOr(p.status, VVS_DEV_TIMEOUT);
    s_abort = 1;
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();                                  // no CTA leaves while the other one's signals may still reach it
  tc_fence_after();
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

}  // namespace

int launch_block_matmul_pair(const BlockMatmulArgs& g, cudaStream_t s) {
  const int es = g.f32 ? 4 : 2;
  MatmulParams p{};
  p.a_scale = g.a_scale; p.w_scale = g.w_scale; p.out = g.out; p.out_row = g.out_row; p.m = g.m; p.n = g.n; p.nkb = qblocks(g.k);
  p.wide = g.out_row * es % 16 == 0 && (int64_t)g.n * es % 16 == 0 && g.out_row * es < (int64_t)1 << 40;    // (a bulk copy writes 16 bytes at a time)
  p.status = g.status;
  const long long rows = ((long long)g.m + kTile - 1) / kTile, outs = ((long long)g.n + kTile - 1) / kTile;
  if (rows * outs > 0x3fffffff) return VVS_ERR_SHAPE;
  const Tiles tiles{(int)rows, (int)outs};
  CUtensorMap tm_w, tm_a, tm_out;
  int rc = make_tmap_e4m3(&tm_w, g.w, g.n, g.k, g.w_row, 64);
  if (rc == VVS_OK) rc = make_tmap_e4m3(&tm_a, g.a, g.m, g.k, g.a_row, 128);
  if (rc == VVS_OK && p.wide) rc = make_tmap_bytes_2d(&tm_out, g.out, (uint64_t)g.m, (uint64_t)g.n * es, (uint64_t)g.out_row * es, 128, 32);
  if (rc != VVS_OK) return rc;
  if (!p.wide) tm_out = tm_a;                      // (not used)
  auto* fn = g.f32 ? block_matmul_pair_kernel<float> : block_matmul_pair_kernel<__nv_bfloat16>;
  if (ensure_dynamic_smem(reinterpret_cast<const void*>(fn), kSmemBytes) != cudaSuccess) return VVS_ERR_CUDA;
  const int pairs = (int)std::min<long long>(rows * outs, g.n_sms / 2);
  return launch_kernel(fn, dim3(2 * pairs), dim3(kThreads), kSmemBytes, true, s, p, tm_w, tm_a, tm_out, tiles) == cudaSuccess ? VVS_OK : VVS_ERR_CUDA;
}

}  // namespace vvs
