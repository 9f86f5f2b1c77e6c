// Eviction from the 8-bit cache by accumulated attention weight: selection of what stays, then the moves.
//
// Selection, a cluster of CTAs for a head, each with a range of its slots: order-preserving 32-bit keys of the weights in shared memory (a
// guarded token's key is above every weight's); the keep-th largest digit by digit, histograms summed over the ranks; a bitmap of what
// stays, the lower slots first among equals; free slots below `keep` and movers behind it counted, and matched through a list.
// Moves: what stays in slots behind `keep` goes, in order, into the slots below that became free.
// Sources and targets never overlap, so only what fills a hole is read and written; the one block that holds both, where `keep` lies, is
// left to a last launch.
//
// 32 heads of 128, 32K slots of which 24.6K stay, scales that grow no more: 67 us for 98 MB of rows that fill holes (15 us at a copy's rate).  The
// selection is 32 of them: three passes over 8192 keys in shared memory, and the barriers of four ranks between them.  The moves, 128 slots a
// CTA, are a chain of four round trips each.  With a CTA for a block, keys and values in turn, 82, and 214 where blocks are of 16 slots
// (68 now).  40 heads of 640 slots: 10 us, two launches of some round trips each.
#include "quant_cache.cuh"
#include "tc_common.cuh"

namespace vvs {

namespace {

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

constexpr int kMaxRanks = 8;
constexpr int kTogether = 4;                                   // slots of a thread whose weights travel together

// FEW threads: one CTA, digits of 8 bits, four histograms.  Otherwise 1024 threads of one or several CTAs and digits of 11 bits, three
// histograms: of 8 bits, so many threads would add to the handful of bins that weights' exponents are that the adding costs more.
template <bool FEW>
__global__ void __launch_bounds__(1024) quant_select_kernel(QEvictArgs a, int slots_each) {
  constexpr int BITS = FEW ? 8 : 11, kBins = 1 << BITS, kTurns = FEW ? 4 : 3;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int hist[2][kBins], warp_sums[33], counts[3];     // counts: equals, holes, movers of this rank
  __shared__ int digit_found, left_found;
  grid_dep_launch();
  grid_dep_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = blockDim.x >> 5;
  const int ranks = FEW ? 1 : gridDim.x, rank = FEW ? 0 : blockIdx.x, head = blockIdx.y, seq = blockIdx.z;
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
  auto all_sync = [&]() {
    if (ranks > 1) tc::cluster_sync();
    else __syncthreads();
  };
  // this rank's slots s0 .. s1 - 1 and their keys
  const int s0 = min(len, rank * slots_each), s1 = min(len, s0 + slots_each), n = s1 - s0, words = (n + 31) / 32;
  uint32_t* keys = reinterpret_cast<uint32_t*>(smem);
  uint32_t* stays = keys + slots_each;                         // [words]
  int* before = reinterpret_cast<int*>(stays + slots_each / 32);       // [words] equals, then holes or movers before a word, in this rank
  for (int i = tid; i < kBins; i += blockDim.x) hist[0][i] = hist[1][i] = 0;
  __syncthreads();
  for (int i0 = tid; i0 < n; i0 += kTogether * blockDim.x) {
    float w[kTogether];
    int t[kTogether];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      const int i = min(i0 + j * (int)blockDim.x, n - 1);
      w[j] = mass[s0 + i];
      t[j] = age ? age[s0 + i] : s0 + i;
    }
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      const int i = i0 + j * blockDim.x;
      if (i >= n) break;
      const uint32_t k = t[j] < a.n_sink || t[j] >= end_age - a.n_recent ? 0xffffffffu : key_of(w[j]);
      keys[i] = k;
      atomicAdd(&hist[0][k >> (32 - BITS)], 1);
    }
  }

  // ---- the smallest key that stays, and how many of its equals do --------------------------------------------------------------
  uint32_t prefix = 0;
  int left = keep;
#pragma unroll 1
  for (int turn = 0, above_bit = 32; turn < kTurns; ++turn, above_bit -= BITS) {
    const int shift = max(0, above_bit - BITS);
    int* bins = hist[turn & 1];
    if (turn > 0) {
      for (int i = tid; i < n; i += blockDim.x) {
        const uint32_t k = keys[i];
        if ((k >> above_bit) == (prefix >> above_bit)) atomicAdd(&bins[(k >> shift) & ((1 << (above_bit - shift)) - 1)], 1);
      }
    }
    all_sync();
    if (FEW) {                                 // a warp's sums, bins 255 - 8 lane and down; the others clear the next turn's
      if (warp == 0) {
        int bin[8], mine = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          bin[j] = bins[255 - 8 * lane - j];
          mine += bin[j];
        }
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += y;
        }
        int above = upto - mine;
        if (above < left && upto >= left) {
          int j = 0;
#pragma unroll
          for (int q = 0; q < 7; ++q)
            if (j == q && above + bin[q] < left) {
              above += bin[q];
              ++j;
            }
          digit_found = 255 - 8 * lane - j;
          left_found = left - above;
        }
      } else {
        for (int i = tid - 32; i < kBins; i += blockDim.x - 32) hist[(turn & 1) ^ 1][i] = 0;
      }
    } else {                                   // bins 2047 - 2 tid and the one below, of all ranks
      const int at = 2046 - 2 * tid;
      int hi = 0, lo = 0, total;
      if (ranks == 1) {
        hi = bins[at + 1];
        lo = bins[at];
      } else {
        int c[2 * kMaxRanks];
#pragma unroll
        for (int k = 0; k < kMaxRanks; ++k) {
          c[2 * k] = k < ranks ? tc::ld_cluster_s32(&bins[at + 1], k) : 0;
          c[2 * k + 1] = k < ranks ? tc::ld_cluster_s32(&bins[at], k) : 0;
        }
#pragma unroll
        for (int k = 0; k < kMaxRanks; ++k) {
          hi += c[2 * k];
          lo += c[2 * k + 1];
        }
      }
      const int above = scan_exclusive(hi + lo, warp_sums, &total);
      if (above < left && above + hi + lo >= left) {
        digit_found = above + hi >= left ? at + 1 : at;
        left_found = left - above - (above + hi >= left ? 0 : hi);
      }
      for (int i = tid; i < kBins; i += blockDim.x) hist[(turn & 1) ^ 1][i] = 0;
    }
    __syncthreads();
    prefix |= (uint32_t)digit_found << shift;
    left = left_found;
    __syncthreads();
  }

  // ---- a bitmap of what stays; free slots below `keep` and movers behind it, counted word by word ---------------------------------
  for (int w = warp; w < words; w += n_warps) {
    const int i = w * 32 + lane;
    const uint32_t k = i < n ? keys[i] : 0u;
    const uint32_t more = __ballot_sync(0xffffffffu, i < n && k > prefix), equal = __ballot_sync(0xffffffffu, i < n && k == prefix);
    if (lane == 0) {
      stays[w] = more;
      before[w] = (int)equal;
    }
  }
  __syncthreads();
  int run = 0;
  if (ranks > 1) {                                             // equals of this rank, so that the ranks above know where theirs begin
    for (int w0 = 0; w0 < words; w0 += blockDim.x) {
      int total;
      scan_exclusive(w0 + tid < words ? __popc((uint32_t)before[w0 + tid]) : 0, warp_sums, &total);
      run += total;
    }
    if (tid == 0) counts[0] = run;
    tc::cluster_sync();
    run = 0;
    for (int k = 0; k < rank; ++k) run += tc::ld_cluster_s32(&counts[0], k);
  }
  for (int w0 = 0; w0 < words; w0 += blockDim.x) {
    const int w = w0 + tid;
    uint32_t equal = w < words ? (uint32_t)before[w] : 0u;
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
  // free slots and movers of a word of this rank
  auto free_bits = [&](int w) {
    const int at = keep - (s0 + w * 32);                       // slots of the word below keep
    const uint32_t below = at >= 32 ? 0xffffffffu : at <= 0 ? 0u : (1u << at) - 1u;
    return ~stays[w] & below;
  };
  auto move_bits = [&](int w) {
    const int at = keep - (s0 + w * 32);
    const uint32_t below = at >= 32 ? 0xffffffffu : at <= 0 ? 0u : (1u << at) - 1u;
    return stays[w] & ~below;
  };
  int holes = 0, movers = 0;
  for (int w0 = 0; w0 < words; w0 += blockDim.x) {             // (both counts in one sum: a rank has at most 2^14 slots)
    const int w = w0 + tid;
    int total;
    const int both = scan_exclusive(w < words ? __popc(free_bits(w)) << 16 | __popc(move_bits(w)) : 0, warp_sums, &total);
    // free slots or movers before the word, as it lies below keep or not; of the word of keep, free slots: its movers are the first
    if (w < words) before[w] = s0 + w * 32 < keep ? (both >> 16) + holes : (both & 0xffff) + movers;
    holes += total >> 16;
    movers += total & 0xffff;
  }
  // the movers' slots, in order: of one rank in the place of the keys, of several where the weights' new places will be
  int holes_lower = 0, movers_lower = 0;
  if (ranks > 1) {
    if (tid == 0) {
      counts[1] = holes;
      counts[2] = movers;
    }
    tc::cluster_sync();
    for (int k = 0; k < rank; ++k) {
      holes_lower += tc::ld_cluster_s32(&counts[1], k);
      movers_lower += tc::ld_cluster_s32(&counts[2], k);
    }
  }
  __syncthreads();
  int32_t* list = ranks > 1 ? reinterpret_cast<int32_t*>(mass_out) : reinterpret_cast<int32_t*>(keys);
  for (int w = warp; w < words; w += n_warps) {
    const uint32_t bits = move_bits(w);
    if (!bits) continue;
    const int base = movers_lower + (s0 + w * 32 < keep ? 0 : before[w]);
    if ((bits >> lane) & 1u) list[base + __popc(bits & ((1u << lane) - 1u))] = s0 + w * 32 + lane;
  }
  all_sync();
  auto source_of = [&](int d) {
    const int i = d - s0, w = i >> 5;
    const uint32_t bits = free_bits(w);
    return (bits >> (i & 31)) & 1u ? list[holes_lower + before[w] + __popc(bits & ((1u << (i & 31)) - 1u))] : d;
  };
  const int e1 = min(keep, s1);
  if (ranks > 1) {                                             // (the list has to be read before the weights' places are written)
    for (int d = s0 + tid; d < e1; d += blockDim.x) kept[d] = source_of(d);
    tc::cluster_sync();
  }
  for (int d0 = s0 + tid; d0 < e1; d0 += kTogether * blockDim.x) {
    int from[kTogether];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      const int d = min(d0 + j * (int)blockDim.x, e1 - 1);
      from[j] = ranks > 1 ? kept[d] : source_of(d);
    }
    float w[kTogether];
    int t[kTogether];
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      w[j] = mass[from[j]];
      t[j] = age ? age[from[j]] : from[j];
    }
#pragma unroll
    for (int j = 0; j < kTogether; ++j) {
      const int d = d0 + j * blockDim.x;
      if (d >= e1) break;
      if (ranks == 1) kept[d] = from[j];
      mass_out[d] = w[j];
      if (age_out) age_out[d] = t[j];
    }
  }
  if (ranks > 1) tc::cluster_sync();                           // (a rank's counts are read until here)
}

// The blocks of 128 target slots below `end`, their keys or their values: new scales from the old ones, rows that come in or are rounded again
// through a list, so that no thread is left without one, into registers, and back once all are read.  The block where `keep` lies
// has sources of its own rows too, and its rows behind keep go with its scale: it is done when all others are.
template <int HD>
__global__ void __launch_bounds__(256) quant_move_kernel(QEvictArgs a, int begin, int end) {
  constexpr int kChunks = HD / 16, kMine = 128 * kChunks / 256;              // 16-byte pieces of a row; of a thread
  __shared__ int from_of[128], list[128];
  __shared__ float factor_of[128], top[4];
  __shared__ uint32_t touched[4];
  grid_dep_launch();
  grid_dep_wait();
  const int tid = threadIdx.x, d0 = begin + 128 * (blockIdx.x / 2), head = blockIdx.y, seq = blockIdx.z;
  const int len = a.cache_len[seq], keep = a.keep, blk_log2 = a.c.block_log2, blk = 1 << blk_log2;
  if (len <= keep || len > a.c.cap) return;
  const bool keys = blockIdx.x % 2 == 0;
  const size_t item = (size_t)seq * a.c.n_heads + head;
  float* scales = (keys ? a.c.k_scale : a.c.v_scale) + item * (a.c.cap >> blk_log2);
  uint4* rows = reinterpret_cast<uint4*>((keys ? a.c.k : a.c.v) + item * a.c.cap * HD);
  // of each slot: where its row comes from, and the scale there
  const int d = d0 + tid;
  const bool mine = tid < 128 && d < end;
  int from = d;
  if (mine && d < keep) from = a.kept[item * keep + d];
  const bool moved = from != d;
  float old = 0.f, there = 0.f;
  if (mine) {
    old = scales[d >> blk_log2];
    if (moved) there = scales[from >> blk_log2];
  }
  float most = there;                                          // of the rows that come into the slot's block
  for (int o = blk < 32 ? blk >> 1 : 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  if (tid < 128 && tid % 32 == 0) top[tid / 32] = most;
  if (!__syncthreads_or(moved)) return;
  if (tid < 128) {
    for (int w = 0; w < 4; ++w)
      if (blk > 32 && ((w * 32) ^ tid) < blk) most = fmaxf(most, top[w]);
    const float now = fmaxf(most, old), grown = old / now;
    const uint32_t mask = __ballot_sync(0xffffffffu, mine && (moved || grown != 1.f));
    if (tid % 32 == 0) touched[tid / 32] = mask;
    from_of[tid] = from;
    factor_of[tid] = moved ? there / now : grown;
    if (mine && (tid & (blk - 1)) == 0) scales[d >> blk_log2] = now;
  }
  __syncthreads();
  int n = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t mask = touched[w];
    if (tid / 32 == w && (mask >> (tid % 32)) & 1u) list[n + __popc(mask & ((1u << (tid % 32)) - 1u))] = tid;
    n += __popc(mask);
  }
  __syncthreads();
  uint4 v[kMine];
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int i = tid + j * 256;
    if (i >= n * kChunks) break;
    v[j] = rows[(size_t)from_of[list[i / kChunks]] * kChunks + i % kChunks];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int i = tid + j * 256;
    if (i >= n * kChunks) break;
    const int r = list[i / kChunks];
    const float f = factor_of[r];
    uint4 x = v[j];
    if (f != 1.f) x = make_uint4(rescale_e4m3x4(x.x, f), rescale_e4m3x4(x.y, f), rescale_e4m3x4(x.z, f), rescale_e4m3x4(x.w, f));
    rows[(size_t)(d0 + r) * kChunks + i % kChunks] = x;
  }
}

}  // namespace

int launch_quant_evict(const QEvictArgs& a, cudaStream_t s) {
  if (a.c.cap > VVS_QCACHE_EVICT_CAP) return VVS_ERR_SHAPE;
  // a rank for every 4096 slots, while that does not leave more CTAs than SMs (32 heads of 32K slots: 81 us with four ranks, 140 with
  // eight, whose clusters do not fit all at once)
  const long long items = (long long)a.c.n_seqs * a.c.n_heads;
  int ranks = 1;
  while (ranks < kMaxRanks && (a.c.cap > 16384 * ranks || (items * ranks * 2 <= a.n_sms && a.c.cap >= 8192 * ranks))) ranks *= 2;
  const int slots = ((a.c.cap + ranks - 1) / ranks + 31) / 32 * 32;
  const size_t smem = (size_t)slots * 4 + (size_t)slots / 32 * 8;
  // Heads that have an SM each are selected by 1024 threads, more heads by CTAs of fewer threads, several on an SM: 40 heads of 640 slots 10.3
  // us against 13, 640 heads 52 against 28; 160 heads of 2048 slots 34 against 27, of 8192 slots 83 against 80.
  const bool few = ranks == 1 && items > a.n_sms && slots <= 8192;
  auto select = few ? quant_select_kernel<true> : quant_select_kernel<false>;
  if (ensure_dynamic_smem(reinterpret_cast<const void*>(select), (int)smem) != cudaSuccess) return VVS_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ranks, a.c.n_heads, a.c.n_seqs);
  cfg.blockDim = dim3(!few ? 1024 : slots <= 1024 && items > 2LL * a.n_sms ? 256 : 512);
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
  if (cudaLaunchKernelEx(&cfg, select, a, slots) != cudaSuccess) return VVS_ERR_CUDA;
  const int whole = a.keep >> a.c.block_log2 << a.c.block_log2, next = whole + (1 << a.c.block_log2);
  auto move = a.c.hd == 64 ? quant_move_kernel<64> : quant_move_kernel<128>;
  auto launch_move = [&](int begin, int end) {
    return launch_kernel(move, dim3(2 * ((end - begin + 127) / 128), a.c.n_heads, a.c.n_seqs), dim3(256), 0, true, s, a, begin, end) == cudaSuccess;
  };
  if (whole > 0 && !launch_move(0, whole)) return VVS_ERR_CUDA;
  if (a.keep > whole && !launch_move(whole, next)) return VVS_ERR_CUDA;
  return VVS_OK;
}

}  // namespace vvs
