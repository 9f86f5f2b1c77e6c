// Eviction from the 8-bit cache by accumulated attention weight: selection of what stays, then the moves.
//
// Selection: the keep-th largest of a head's weights is found digit by digit (four histograms of 256 over order-preserving 32-bit keys; a
// guarded token's key is above every weight's); a bitmap of what stays follows, with the lower slots first among equals.
// Moves: what stays in slots behind `keep` goes, in order, into the slots below that became free.  Sources and targets never overlap, so
// the moves need no order among themselves, and only what fills a hole is read and written.  A cluster of CTAs has a head: every rank
// selects by itself (the weights come from L2), and has a share of the target blocks.
#include "quant_cache.cuh"
#include "tc_common.cuh"

namespace vvs {

namespace {

constexpr int kMaxCap = 131072;

// larger key, larger weight; a NaN below everything
__device__ __forceinline__ uint32_t key_of(float w) {
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w + 0.f);               // (-0 counts as 0)
  return b >> 31 ? ~b : b | 0x80000000u;
}

// exclusive sums of v over the threads of a CTA; *total = the whole
__device__ __forceinline__ int scan_exclusive(int v, int* warp_sums, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int w = lane < n_warps ? warp_sums[lane] : 0, t = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, t, o);
      if (lane >= o) t += y;
    }
    warp_sums[lane] = t - w;
    if (lane == 31) warp_sums[32] = t;
  }
  __syncthreads();
  const int r = x - v + warp_sums[warp];
  *total = warp_sums[32];
  __syncthreads();
  return r;
}

__global__ void __launch_bounds__(1024) quant_evict_kernel(QEvictArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int hist[256], warp_sums[33];
  __shared__ int digit_found, left_found;
  grid_dep_launch();
  grid_dep_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
  const int ranks = gridDim.x, rank = blockIdx.x, head = blockIdx.y, seq = blockIdx.z;
  const int cap = a.c.cap, keep = a.keep, len = a.cache_len[seq];
  if (len < 0 || len > cap) {                                  // (the same for every rank)
    if (rank == 0 && head == 0 && tid == 0) atomicOr(a.status, VVS_DEV_CACHE_OVERFLOW);
    return;
  }
  const int end_age = a.next_age ? a.next_age[seq] : len;
  const size_t item = (size_t)seq * a.c.n_heads + head;
  const float* mass = a.c.mass + item * cap;
  const int32_t* age = a.c.age ? a.c.age + item * cap : nullptr;
  float* mass_out = a.mass_out + item * cap;
  int32_t* age_out = a.age_out ? a.age_out + item * cap : nullptr;
  int32_t* kept = a.kept + item * keep;
  const int new_len = min(len, keep);
  if (rank == 0 && head == 0 && tid == 0) a.new_len[seq] = new_len;
  for (int i = rank * blockDim.x + tid; new_len + i < len; i += ranks * blockDim.x) {
    mass_out[new_len + i] = 0.f;
    if (age_out) age_out[new_len + i] = -1;
  }
  if (len <= keep) {
    for (int i = rank * blockDim.x + tid; i < keep; i += ranks * blockDim.x) {
      kept[i] = i < len ? i : -1;
      if (i >= len) continue;
      mass_out[i] = mass[i];
      if (age_out) age_out[i] = age ? age[i] : i;
    }
    return;
  }
  auto key_at = [&](int slot) {
    const int t = age ? age[slot] : slot;
    return t < a.n_sink || t >= end_age - a.n_recent ? 0xffffffffu : key_of(mass[slot]);
  };

  // ---- the smallest key that stays, and how many of its equals do --------------------------------------------------------------
  uint32_t prefix = 0;
  int left = keep;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += blockDim.x) hist[i] = 0;
    __syncthreads();
    for (int slot = tid; slot < len; slot += blockDim.x) {
      const uint32_t k = key_at(slot);
      if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1);
    }
    __syncthreads();
    if (warp == 0) {                           // lane i has the bins 255 - 8i .. 248 - 8i, from the largest down
      int mine = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) mine += hist[255 - 8 * lane - j];
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      int before = upto - mine;
      if (before < left && upto >= left) {
        for (int j = 0; j < 8; ++j) {
          const int n = hist[255 - 8 * lane - j];
          if (before + n >= left) {
            digit_found = 255 - 8 * lane - j;
            left_found = left - before;
            break;
          }
          before += n;
        }
      }
    }
    __syncthreads();
    prefix |= (uint32_t)digit_found << shift;
    left = left_found;
    __syncthreads();
  }

  // ---- a bitmap of what stays; free slots below `keep` and movers behind it, counted word by word ---------------------------------
  const int words = (len + 31) / 32;
  uint32_t* stays = reinterpret_cast<uint32_t*>(smem);
  int* movers_before = reinterpret_cast<int*>(stays + words);  // of the words from keep / 32 on
  int* holes_before = movers_before + words + 1;
  for (int w = warp; w < words; w += n_warps) {
    const int slot = w * 32 + lane;
    const uint32_t k = slot < len ? key_at(slot) : 0u;
    const uint32_t more = __ballot_sync(0xffffffffu, slot < len && k > prefix), equal = __ballot_sync(0xffffffffu, slot < len && k == prefix);
    if (lane == 0) {
      stays[w] = more;
      holes_before[w] = (int)equal;
    }
  }
  __syncthreads();
  int run = 0;
  for (int w0 = 0; w0 < words; w0 += blockDim.x) {
    const int w = w0 + tid;
    uint32_t equal = w < words ? (uint32_t)holes_before[w] : 0u;
    int total;
    int take = left - (run + scan_exclusive(__popc(equal), warp_sums, &total));
    run += total;
    if (w < words) {
      uint32_t bits = 0;
      for (; take > 0 && equal; --take) {
        bits |= equal & (0u - equal);
        equal &= equal - 1u;
      }
      stays[w] |= bits;
    }
  }
  __syncthreads();
  const int keep_word = keep / 32;
  const uint32_t below = (1u << (keep & 31)) - 1u;             // of the word that keep lies in
  int holes = 0, movers = 0;
  for (int w0 = 0; w0 < words; w0 += blockDim.x) {
    const int w = w0 + tid;
    const uint32_t s = w < words ? stays[w] : 0u;
    const uint32_t free_bits = w < keep_word ? ~s : w == keep_word ? ~s & below : 0u;
    const uint32_t move_bits = w > keep_word ? s : w == keep_word ? s & ~below : 0u;
    int total;
    const int h = scan_exclusive(__popc(free_bits), warp_sums, &total) + holes;
    holes += total;
    const int m = scan_exclusive(__popc(move_bits), warp_sums, &total) + movers;
    movers += total;
    if (w < words) {
      holes_before[w] = h;
      movers_before[w] = m;
    }
  }
  __syncthreads();

  // ---- this rank's target blocks: where each slot's row comes from ------------------------------------------------------------------
  const int blk_log2 = a.c.block_log2, blk = 1 << blk_log2;
  const int blocks = (keep + blk - 1) >> blk_log2, per = (blocks + ranks - 1) / ranks;
  const int b0 = min(blocks, rank * per), b1 = min(blocks, b0 + per);
  float* now = reinterpret_cast<float*>(holes_before + words + 1);      // [per][2] new scales
  for (int d = (b0 << blk_log2) + tid; d < min(keep, b1 << blk_log2); d += blockDim.x) {
    int from = d;
    if (!((stays[d >> 5] >> (d & 31)) & 1u)) {
      const int r = holes_before[d >> 5] + __popc(~stays[d >> 5] & ((1u << (d & 31)) - 1u));
      int lo = keep_word, hi = words - 1;                     // the last word with at most r movers before it
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (movers_before[mid] <= r) lo = mid; else hi = mid - 1;
      }
      uint32_t s = lo == keep_word ? stays[lo] & ~below : stays[lo];
      for (int j = r - movers_before[lo]; j > 0; --j) s &= s - 1u;
      from = lo * 32 + __ffs(s) - 1;
    }
    kept[d] = from;
    mass_out[d] = mass[from];
    if (age_out) age_out[d] = age ? age[from] : from;
  }
  __syncthreads();

  // ---- new scales, from the old ones ---------------------------------------------------------------------------------------------------
  const size_t scale_row = item * (cap >> blk_log2);
  for (int b = b0 + warp; b < b1; b += n_warps) {
    float ks = 0.f, vs = 0.f;
    for (int i = lane; i < blk; i += 32) {
      const int d = (b << blk_log2) + i;
      if (d >= keep) break;
      const int from = kept[d];
      if (from == d) continue;
      ks = fmaxf(ks, a.c.k_scale[scale_row + (from >> blk_log2)]);
      vs = fmaxf(vs, a.c.v_scale[scale_row + (from >> blk_log2)]);
    }
    __syncwarp();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      ks = fmaxf(ks, __shfl_xor_sync(0xffffffffu, ks, o));
      vs = fmaxf(vs, __shfl_xor_sync(0xffffffffu, vs, o));
    }
    if (lane == 0) {
      now[2 * (b - b0)] = fmaxf(ks, a.c.k_scale[scale_row + b]);
      now[2 * (b - b0) + 1] = fmaxf(vs, a.c.v_scale[scale_row + b]);
    }
  }
  __syncthreads();

  // ---- the moves, 16 bytes a thread; rows that stay in a block whose scale grows are rounded again --------------------------------------
  const int chunks = a.c.hd / 16;
  auto rescaled = [](uint4 v, float f) {
    return make_uint4(rescale_e4m3x4(v.x, f), rescale_e4m3x4(v.y, f), rescale_e4m3x4(v.z, f), rescale_e4m3x4(v.w, f));
  };
  for (int i = tid; i < ((b1 - b0) << blk_log2) * chunks; i += blockDim.x) {
    const int d = (b0 << blk_log2) + i / chunks, cc = i % chunks;
    if (d >= keep) continue;
    const int from = kept[d], b = d >> blk_log2;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      uint4* rows = reinterpret_cast<uint4*>((kv ? a.c.v : a.c.k) + item * cap * a.c.hd);
      const float was = (kv ? a.c.v_scale : a.c.k_scale)[scale_row + (from >> blk_log2)], f = was / now[2 * (b - b0) + kv];
      if (from == d && f == 1.f) continue;
      const uint4 v = rows[(size_t)from * chunks + cc];
      rows[(size_t)d * chunks + cc] = f == 1.f ? v : rescaled(v, f);
    }
  }
  if (ranks > 1) tc::cluster_sync(); else __syncthreads();     // every rank has read the old scales and its sources
  if (rank == (blocks - 1) / per && (keep & (blk - 1))) {      // the block that keep lies in: the rows behind it go with its scale
    const int b = blocks - 1;
    for (int i = tid; i < ((blocks << blk_log2) - keep) * chunks; i += blockDim.x)
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        uint4* rows = reinterpret_cast<uint4*>((kv ? a.c.v : a.c.k) + item * cap * a.c.hd) + (size_t)keep * chunks;
        const float f = (kv ? a.c.v_scale : a.c.k_scale)[scale_row + b] / now[2 * (b - b0) + kv];
        if (f != 1.f) rows[i] = rescaled(rows[i], f);
      }
  }
  __syncthreads();
  for (int b = b0 + tid; b < b1; b += blockDim.x) {
    a.c.k_scale[scale_row + b] = now[2 * (b - b0)];
    a.c.v_scale[scale_row + b] = now[2 * (b - b0) + 1];
  }
}

}  // namespace

int launch_quant_evict(const QEvictArgs& a, cudaStream_t s) {
  if (a.c.cap > kMaxCap) return VVS_ERR_SHAPE;
  const int blocks = (a.keep + (1 << a.c.block_log2) - 1) >> a.c.block_log2, words = (a.c.cap + 31) / 32;
  const long long items = (long long)a.c.n_seqs * a.c.n_heads;
  int ranks = 1;
  while (ranks < 8 && items * ranks * 2 <= a.n_sms && blocks >= 4 * ranks) ranks *= 2;
  const size_t smem = (size_t)(3 * words + 2) * 4 + (size_t)((blocks + ranks - 1) / ranks) * 8;
  if (ensure_dynamic_smem(reinterpret_cast<const void*>(quant_evict_kernel), (int)smem) != cudaSuccess) return VVS_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ranks, a.c.n_heads, a.c.n_seqs);
  cfg.blockDim = dim3(a.c.cap <= 2048 ? 256 : 1024);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ranks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, quant_evict_kernel, a) == cudaSuccess ? VVS_OK : VVS_ERR_CUDA;
}

}  // namespace vvs
