// Product of rows and weights in e4m3 with scales of blocks of 128, for few to some hundred rows.
//
//   out[m, n] = sum_b a_scale[m, b] * w_scale[n / 128, b] * sum_{k in b} a[m, k] * w[n, k]
//
// Weights lie on the tensor cores' M side (128 of them a tile, one scale a block), the rows on its N side, so that few rows cost few
// columns.  A block of K is one sum in tensor memory; while the next blocks' are under way, eight warps take it from there and add it, times
// the two scales, to float32 sums in registers: a thread has a weight's row and half of the pass's rows.  The blocks of K of a tile are
// dealt to the CTAs of a cluster where tiles are few; each CTA is sent the others' sums of its share of the rows and adds them in rank order.
//
// Bound by the weights' way from HBM, small ones by their chain of round trips (wait for what precedes, first loads, sums, exchange: a
// microsecond each).  Rows of 4096 through 22016 weights: 18 in 18.5 us, 4.9 TB/s (76 % of a copy's rate; 94 % through 88064 weights), 128 in 26.7;
// 288 of 3456 through 1280 7.0, one of 1280 through 1280 4.2 (2.9 in a graph).
#include <atomic>

#include "block_matmul.cuh"
#include "block_plans.h"

namespace vvs {

using namespace bmm;

namespace {

constexpr int kThreads = 384, kSumWarps = 8;
constexpr int kMaxStages = kMatmulMaxStages, kMaxSplits = kMatmulMaxSplits, kChunk = 8;     // kChunk: blocks whose factors lie in shared memory together

constexpr int kFourBytes = 128 * 16;               // sums of four rows of the call with a tile of weights
static_assert(kTileBytes == kMatmulTileBytes, "what the plans count with");

__device__ __forceinline__ void put_one(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put_one(float* p, float v) { *p = v; }

// CPT: columns (rows of the call) of a summing thread; a pass has 2 CPT of them
template <int CPT, typename T>
__global__ void __launch_bounds__(kThreads, CPT <= 32 ? 2 : 1)
block_matmul_kernel(const __grid_constant__ MatmulParams p, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_a, int stages) {
  constexpr int TN = 2 * CPT, kBufs = kMatmulPlaces<TN>, kCols = CPT <= 16 ? 32 : CPT <= 32 ? 64 : 128, kTmem = kMatmulColumns<TN>;
  static_assert(kBufs * kCols <= kTmem, "columns of tensor memory, a power of two; two CTAs fit an SM");
  constexpr uint32_t kStageBytes = kTileBytes + TN * kQBlock;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[kMaxStages], done_bar[kMaxStages], free_bar[kBufs], recv_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int s_abort;
  __shared__ __align__(16) float s_factor[2][2][kChunk][CPT];     // of a half, of even or odd chunks

  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  // (of a product in two parts the first clusters have a tile of the first part in each CTA, the others a tile of the second part together)
  const bool alone = (int)blockIdx.y < p.alone;
  const int splits = alone ? 1 : (int)gridDim.x, rank = alone ? 0 : (int)blockIdx.x, tok0 = (int)blockIdx.z * TN;
  const int tile = alone ? (int)(blockIdx.y * gridDim.x + blockIdx.x) : p.first + (int)blockIdx.y - p.alone;
  if (alone && tile >= p.first) return;
  const int kb0 = (int)((long long)p.nkb * rank / splits), kb1 = (int)((long long)p.nkb * (rank + 1) / splits), n_kb = kb1 - kb0;

  // Rows of the call go in fours to the CTAs of a cluster, in turns: that is whose sums a CTA gets.  [CTA][four rows][weight][row] behind the stages
  const int toks = min(TN, p.m - tok0), fours = (toks + 3) / 4, each = (TN / 4 + splits - 1) / splits;
  uint8_t* recv = smem + stages * kStageBytes;

  if (tid == 0) {
    for (int i = 0; i < stages; ++i) {
      mbar_init(&full_bar[i], 1);
      mbar_init(&done_bar[i], 1);
    }
    for (int i = 0; i < kBufs; ++i) mbar_init(&free_bar[i], kSumWarps);
    s_abort = 0;
    mbar_init(&recv_bar, 1);
    fence_barrier_init();
    mbar_expect_tx(&recv_bar, (uint32_t)((splits - 1) * ((fours - rank + splits - 1) / splits) * kFourBytes));
  }
  if (warp == 2) {
    tmem_alloc(&tmem_slot, kTmem);
    tmem_relinquish();
  }
  if (warp == 0 && elect_one()) {
    tma_prefetch_desc(&tm_w);
    tma_prefetch_desc(&tm_a);
    // Weights go as far as L2 before the wait, not into shared memory: what precedes this kernel may be what writes them.
    for (int i = 0; i < min(n_kb, stages); ++i) tma_prefetch_2d(&tm_w, (kb0 + i) * kQBlock, tile * 128);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (splits > 1) cluster_arrive_relaxed();        // this CTA's barrier is ready for the others' sums (fence_barrier_init above)
  const uint32_t tmem = tmem_slot;
  // (Of two launches the second waits for the first, of which it needs nothing: only behind a wait of its own does a launch see what those
  // before it wrote.)
  pdl_launch_dependents();
  pdl_wait();

  if (warp == 0) {
    // ---- producer -------------------------------------------------------------------------------------------------------
    uint32_t stage = 0, par = 1;                   // parity of the stage's previous release
    int issued = 0;
    bool ok = true;
    for (int i = 0; i < n_kb; ++i, ++issued) {
      if (i >= stages && !(ok = warp_wait_or_abort(&done_bar[stage], par, &s_abort))) break;
      __syncwarp();
      if (elect_one()) {
        uint8_t* st = smem + stage * kStageBytes;
        mbar_expect_tx(&full_bar[stage], kStageBytes);
        tma_load_2d(st, &tm_w, &full_bar[stage], (kb0 + i) * kQBlock, tile * 128);
        tma_load_2d(st + kTileBytes, &tm_a, &full_bar[stage], (kb0 + i) * kQBlock, tok0);
      }
      if (++stage == (uint32_t)stages) { stage = 0; par ^= 1; }
    }
    if (!ok) {
      if (lane == 0) atomicOr(p.status, VVS_DEV_TIMEOUT);
      s_abort = 1;
    }
    // Nothing may be in flight when the CTA leaves, also where it is another warp that gives up (bounded)
    for (int i = max(issued - stages, 0); i < issued; ++i) mbar_wait(&full_bar[i % stages], (i / stages) & 1);
    __syncwarp();
  } else if (warp == 1) {
    // ---- MMA issuer (a wait that ran out is reported, and nothing more is issued) -------------------------------------------
    const uint32_t idesc = idesc_e4m3_f32(128, TN), lo0 = desc_lo_sw128(smem_u32(smem));
    uint32_t stage = 0, par = 0, buf = 0, bpar = 1;
    for (int i = 0; i < n_kb; ++i) {
      const bool ok = (i < kBufs || warp_wait_or_abort(&free_bar[buf], bpar, &s_abort)) && warp_wait_or_abort(&full_bar[stage], par, &s_abort);
      __syncwarp();
      if (!ok) {
        if (lane == 0) atomicOr(p.status, VVS_DEV_TIMEOUT);
        s_abort = 1;
        break;
      }
      tc_fence_after();
      const uint32_t a_lo = lo0 + stage * (kStageBytes >> 4);
      mma_e4m3_block<1>(tmem + buf * kCols, a_lo, a_lo + (kTileBytes >> 4), idesc);
      mma_commit_elect(&done_bar[stage]);          // the sum is there, and its stage may be filled again
      if (++stage == (uint32_t)stages) { stage = 0; par ^= 1; }
      if (++buf == kBufs) { buf = 0; bpar ^= 1; }
    }
  } else if (warp >= 4) {
    // ---- sums -----------------------------------------------------------------------------------------------------------
    const int half = (warp - 4) >> 2, t = tid & 127;                  // t: of the 128 threads of a half
    const uint32_t t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16) + half * CPT;
    const int n_chunks = (n_kb + kChunk - 1) / kChunk;
    // factors a_scale * w_scale of a chunk: eight neighbouring blocks of a row by eight neighbouring threads
    constexpr int kLoads = (CPT * kChunk + 127) / 128;
    float next_a[kLoads], next_w[kLoads];         // (multiplied where they are put down: a product here would wait for the loads)
    auto request = [&](int chunk) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int at = j * 128 + t, b = chunk * kChunk + (at & (kChunk - 1)), tok = tok0 + half * CPT + at / kChunk;
        const bool in = at < CPT * kChunk && b < n_kb && tok < p.m;
        next_a[j] = in ? p.a_scale[(size_t)tok * p.nkb + kb0 + b] : 0.f;
        next_w[j] = in ? p.w_scale[(size_t)tile * p.nkb + kb0 + b] : 0.f;
      }
    };
    auto put = [&](int chunk) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int at = j * 128 + t;
        if (at < CPT * kChunk) s_factor[half][chunk & 1][at & (kChunk - 1)][at / kChunk] = next_a[j] * next_w[j];
      }
    };
    float acc[CPT];
#pragma unroll
    for (int j = 0; j < CPT; ++j) acc[j] = 0.f;
    uint32_t buf = 0, stage = 0, par = 0;
    bool ok = true;
    request(0);
    for (int c = 0; c < n_chunks; ++c) {
      put(c);
      if (c + 1 < n_chunks) request(c + 1);
      named_bar_sync(1 + half, 128);               // (a chunk's place was last read two chunks ago, before the barrier between)
      const int blocks = min(kChunk, n_kb - c * kChunk);
#pragma unroll 1
      for (int b = 0; b < blocks; ++b) {
        ok = ok && warp_wait_lean(smem_u32(&done_bar[stage]), par, &s_abort);
        if (ok) {
          tc_fence_after();
          const float4* f = reinterpret_cast<const float4*>(&s_factor[half][c & 1][b][0]);
          constexpr int kLd = CPT % 16 ? 8 : 16, kPieces = CPT / kLd;
          float part[kPieces > 1 ? 2 : 1][kLd];
          tmem_request(t_row + buf * kCols, part[0]);
#pragma unroll
          for (int c = 0; c < kPieces; ++c) {
            float (&now)[kLd] = part[kPieces > 1 ? c & 1 : 0];
            tmem_wait(now);
            if (c + 1 < kPieces) tmem_request(t_row + buf * kCols + (c + 1) * kLd, part[(c + 1) & 1]);
#pragma unroll
            for (int j = 0; j < kLd; j += 4) {
              const float4 g = f[(c * kLd + j) / 4];
              acc[c * kLd + j] = fmaf(now[j], g.x, acc[c * kLd + j]);
              acc[c * kLd + j + 1] = fmaf(now[j + 1], g.y, acc[c * kLd + j + 1]);
              acc[c * kLd + j + 2] = fmaf(now[j + 2], g.z, acc[c * kLd + j + 2]);
              acc[c * kLd + j + 3] = fmaf(now[j + 3], g.w, acc[c * kLd + j + 3]);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&free_bar[buf]);
        }
        if (++buf == kBufs) buf = 0;
        if (++stage == (uint32_t)stages) { stage = 0; par ^= 1; }
      }
    }
    if (!ok) {
      if (lane == 0) atomicOr(p.status, VVS_DEV_TIMEOUT);
      s_abort = 1;
    }
    const int w_row = (warp & 3) * 32 + lane;
    if (splits > 1) {
      __syncwarp();
      cluster_wait();
      if (ok) {
        int owner = half * (CPT / 4) % splits, at = half * (CPT / 4) / splits;
#pragma unroll
        for (int q = 0; q < CPT / 4; ++q) {
          if (half * (CPT / 4) + q < fours) {
            uint8_t* to = recv + ((rank * each + at) * 128 + w_row) * 16;
            if (owner == rank) st_shared4(smem_u32(to), &acc[4 * q]);
            else st_async4(mapa(smem_u32(to), owner), mapa(smem_u32(&recv_bar), owner), &acc[4 * q]);
          }
          if (++owner == splits) owner = 0, ++at;
        }
      }
    } else if (ok) {
      // the stages have drained: the last sum is behind every MMA.  [row of the call][weight]
      float* red = reinterpret_cast<float*>(smem);
#pragma unroll
      for (int j = 0; j < CPT; ++j) red[(half * CPT + j) * 128 + w_row] = acc[j];
    }
  }
  __syncwarp();
  if (splits > 1 && warp < 4) cluster_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (splits > 1) {
    // ---- out, of a cluster: four rows of one weight a thread, sums in rank order -----------------------------------------------------
    bool got = false;
    for (uint32_t k = 0; k < kSpinLimit && !got; ++k) got = mbar_try_wait_cluster(&recv_bar, 0) || ((k & 1023u) == 1023u && s_abort);
    if (!got) {
      atomicOr(p.status, VVS_DEV_TIMEOUT);
      s_abort = 1;
    }
    __syncwarp();
    cluster_arrive_relaxed();                      // what was sent has come, here; waited for at the end: no CTA leaves while it may be sent to
    const int n = tile * 128 + (tid & 127);
    if (!s_abort && n < p.n) {
      for (int i = tid >> 7; rank + i * splits < fours; i += kThreads / 128) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < kMaxSplits; ++s)
          if (s < splits) {
            const float4 x = *reinterpret_cast<const float4*>(recv + ((s * each + i) * 128 + (tid & 127)) * 16);
            v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
          }
        const int r = (rank + i * splits) * 4;
        T* o = static_cast<T*>(p.out) + (size_t)(tok0 + r) * p.out_row + n;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (r + j < toks) put_one(o + (size_t)j * p.out_row, v[j]);
      }
    }
    __syncwarp();
    cluster_wait();
  } else if (!s_abort) {
    // ---- out: four weights of a row a thread ---------------------------------------------------------------------------------------
    const int n0 = tile * 128 + (tid & 31) * 4;
    const float* red = reinterpret_cast<const float*>(smem) + (tid & 31) * 4;
    if (n0 < p.n)
      for (int r = tid >> 5; r < toks; r += kThreads / 32) {
        const float4 x = *reinterpret_cast<const float4*>(red + r * 128);
        const float v[4] = {x.x, x.y, x.z, x.w};
        T* o = static_cast<T*>(p.out) + (size_t)(tok0 + r) * p.out_row + n0;
        if (p.wide && n0 + 4 <= p.n) {
          store4(o, v);
        } else {
          for (int j = 0; j < 4 && n0 + j < p.n; ++j) put_one(o + j, v[j]);
        }
      }
  }
  __syncwarp();
  if (warp == 2) tmem_dealloc(tmem, kTmem);
}

// The kernel set up on the current device, and how many of its clusters the device holds; asked once (a look into both tables is a tenth of what a
// small call costs the host).
template <int CPT, typename T>
const int* clusters_of() {
  constexpr int TN = 2 * CPT, kDevices = 64;
  static std::atomic<const int*> known[kDevices] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return nullptr;
  if (dev < kDevices)
    if (const int* there = known[dev].load(std::memory_order_acquire)) return there;
  const void* fn = reinterpret_cast<const void*>(block_matmul_kernel<CPT, T>);
  if (ensure_dynamic_smem(fn, matmul_room(TN) + 1024) != cudaSuccess) return nullptr;
  const int* there = resident_clusters(fn, kThreads, matmul_smem(TN, 1));
  if (there && dev < kDevices) known[dev].store(there, std::memory_order_release);
  return there;
}

template <int CPT, typename T>
int launch_cpt(const BlockMatmulArgs& g, MatmulParams p, cudaStream_t s) {
  constexpr int TN = 2 * CPT;
  auto* fn = block_matmul_kernel<CPT, T>;
  const int* clusters = clusters_of<CPT, T>();
  if (!clusters) return VVS_ERR_CUDA;
  const BlockMatmulPlan pl = plan_block_matmul(g.m, g.n, g.k, g.n_sms, clusters);
  if (pl.pairs) return launch_block_matmul_pair(g, s);
  CUtensorMap tm_w, tm_a;
  int rc = make_tmap_e4m3(&tm_w, g.w, g.n, g.k, g.w_row, 128);
  if (rc == VVS_OK) rc = make_tmap_e4m3(&tm_a, g.a, g.m, g.k, g.a_row, TN);
  if (rc != VVS_OK) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  auto launch = [&](int splits, int64_t rows) {
    cfg.gridDim = dim3(splits, (unsigned)rows, pl.passes);
    cfg.dynamicSmemBytes = matmul_smem(TN, splits);
    attr[1].val.clusterDim.x = splits;
    cfg.numAttrs = splits > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, fn, p, tm_w, tm_a, matmul_stages(TN, splits)) == cudaSuccess;
  };
  const BlockMatmulPart &main = pl.part[0], &rest = pl.part[1];
  if (rest.count && matmul_in_one_launch(TN)) {
    p.first = (int)rest.first;
    p.alone = (int)((main.count + rest.splits - 1) / rest.splits);
    return launch(rest.splits, p.alone + rest.count) ? VVS_OK : VVS_ERR_CUDA;
  }
  if (!launch(main.splits, main.count)) return VVS_ERR_CUDA;
  p.first = (int)rest.first;
  if (rest.count && !launch(rest.splits, rest.count)) return VVS_ERR_CUDA;
  return VVS_OK;
}

template <typename T>
int launch_rows(const BlockMatmulArgs& g, const MatmulParams& p, cudaStream_t s) {
  switch (matmul_rows(g.m)) {
    case 16: return launch_cpt<8, T>(g, p, s);
    case 32: return launch_cpt<16, T>(g, p, s);
    case 48: return launch_cpt<24, T>(g, p, s);
    case 64: return launch_cpt<32, T>(g, p, s);
    case 96: return launch_cpt<48, T>(g, p, s);
    default: return launch_cpt<64, T>(g, p, s);
  }
}

}  // namespace

namespace bmm {
int make_tmap_e4m3(CUtensorMap* out, const void* base, int64_t rows, int64_t cols, int64_t row_bytes, uint32_t box_rows) {
  return make_tmap_bytes_2d(out, base, (uint64_t)rows, (uint64_t)cols, (uint64_t)row_bytes, kQBlock, box_rows);
}
}  // namespace bmm

int launch_block_matmul(const BlockMatmulArgs& g, cudaStream_t s) try {
  MatmulParams p{};
  p.a_scale = g.a_scale; p.w_scale = g.w_scale; p.out = g.out; p.out_row = g.out_row; p.m = g.m; p.n = g.n; p.nkb = qblocks(g.k);
  p.wide = g.out_row % 4 == 0;
  p.status = g.status;
  return g.f32 ? launch_rows<float>(g, p, s) : launch_rows<__nv_bfloat16>(g, p, s);
} catch (...) {
  return VVS_ERR_NOMEM;
}

}  // namespace vvs
