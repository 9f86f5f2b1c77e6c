// Appends a block's keys and values to the 8-bit cache: rotation, one scale for each (block of slots, head), e4m3 codes; the query
// heads of the same rows are rotated too.  Every input is read once and every output written once: bound by HBM for prompts, by the
// launch and a few round trips for a step's rows.  A CTA has the rows that fall into one block of slots, and some of the heads;
// cosines and sines of its rows are computed once, into shared memory.  A head's rows stay in registers, as they are stored, between
// the maximum that fixes the scale and the rounding.
// Few rows: a warp has a head, so that nothing but the table of sines is waited for by a whole CTA, and queries are heads like others.
// Prompts: a CTA has a head.
//
// Eight prompts of 1301 rows, 32 + 2 x 8 heads of 128: 71.5 us for 235 MB, 51 % of a copy's rate: the queries' launch 29 of them, the keys' and
// values' 42, in which half of the issue slots turn, compare, scale and round (two passes over what a head's rows hold in registers).  32 blocks
// of 9 rows, 32 + 2 x 32 heads: 8.7 us; two of them of 3 x 20 heads of 64: 5.5, where a call that does next to nothing takes 4.1.
#include "quant_cache.cuh"

namespace vvs {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// rows of a pass of a warp and of a CTA: 4 and 32 of 64 elements, 2 and 16 of 128
template <int HD, bool WARP>
constexpr int kPassRows = (WARP ? 32 : kThreads) / (HD / 8);
constexpr int kFewPasses = 8;                  // of a warp: 32 rows of 64 elements, 16 of 128

// What a CTA works on: rows t0 .. t1 - 1 of the call, those of its k and v t0 .. tk - 1, behind `live` rows of the block of slots.
struct Chunk {
  int seq, block, live, t0, t1, tk;
};

// A thread's pieces of a head's rows, as they are stored; of keys and values the row index picks the rows.
template <typename T, int HD, int PASSES, bool WARP>
__device__ __forceinline__ void request_rows(const QAppendArgs& a, const HeadRows& src, const Chunk& ch, int head, int end, bool picked, bool split,
                                             Unit<T> (&raw)[PASSES]) {
  const int in = WARP ? threadIdx.x % 32 : threadIdx.x, u = in % (HD / 8), r = in / (HD / 8);
  const T* base = static_cast<const T*>(src.data) + ch.seq * src.seq + head * src.head;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int t = ch.t0 + p * kPassRows<HD, WARP> + r;
    if (t >= end) continue;
    const int from = picked ? a.row_index[(size_t)ch.seq * a.n_rows + t] : t;
    if (from >= 0 && from < a.n_rows) {
      raw[p] = load_unit(base + from * src.row + unit_at(u, split), split, a.rope.n_pairs);
    } else {
      raw[p] = Unit<T>{};
      atomicOr(a.status, VVS_DEV_BAD_ARG);
    }
  }
}

// Cosines and sines of a piece's four pairs, of a row.
template <int HD>
__device__ __forceinline__ void angles_of(const float2* table, int row, float (&c)[4], float (&s)[4]) {
  const float4* cs = reinterpret_cast<const float4*>(table + (size_t)row * (HD / 2) + 4 * (threadIdx.x % (HD / 8)));
  const float4 lo = cs[0], hi = cs[1];
  c[0] = lo.x; s[0] = lo.y; c[1] = lo.z; s[1] = lo.w;
  c[2] = hi.x; s[2] = hi.y; c[3] = hi.z; s[3] = hi.w;
}
// Whether a unit has any pair at all.
__device__ __forceinline__ bool unit_turns(const RopeAxes& r, int u) { return 4 * u < r.n_pairs; }
// A piece's values, turned by its row's angles if it is `mine`: all pairs, or (SOME) those that have any.
template <typename T, int HD, bool SOME>
__device__ __forceinline__ void values_of(const Unit<T>& raw, bool mine, bool split, const float2* table, int row, float (&x)[8]) {
  widen_unit(raw, x);
  if (!mine) return;
  float c[4], s[4];
  angles_of<HD>(table, row, c, s);
  if (SOME) turn_some(x, split, c, s, pairs_of(c));
  else turn_unit(x, split, c, s);
}
// One of a thread's pieces, by an index that is not known where the code is made.
template <typename T, int PASSES>
__device__ __forceinline__ Unit<T> piece_of(const Unit<T> (&raw)[PASSES], int p) {
  Unit<T> piece = raw[0];
#pragma unroll
  for (int j = 1; j < PASSES; ++j)
    if (j == p) piece = raw[j];
  return piece;
}

// A head's rows into the cache, by a warp or by the CTA.  They are turned twice, for the maximum and for the codes: that takes fewer registers
// than one turned copy (bf16 rows of long blocks: 80 of a thread in the place of 213).
template <typename T, int HD, int PASSES, bool WARP>
__device__ __forceinline__ void put_rows(const QAppendArgs& a, const Unit<T> (&raw)[PASSES], bool turned, uint8_t* codes, float* scales,
                                         const Chunk& ch, int head, const float2* table, float* red, bool& odd) {
  constexpr int kUnits = HD / 8, kRows = kPassRows<HD, WARP>;
  const int tid = WARP ? threadIdx.x % 32 : threadIdx.x, u = tid % kUnits, r = tid / kUnits, n_pairs = a.rope.n_pairs;
  const bool mine = turned && unit_turns(a.rope, u), split = turned && unit_split(a.rope, u);
  float* scale = scales + ((size_t)ch.seq * a.c.n_heads + head) * (a.c.cap >> a.c.block_log2) + ch.block;
  const float old = ch.live > 0 ? *scale : 0.f;
  float amax = 0.f, zero = 0.f;                // zero: NaN once an infinity or a NaN has been seen
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (ch.t0 + p * kRows + r >= ch.tk) continue;
    float x[8];
    values_of<T, HD, false>(raw[p], mine, split, table, p * kRows + r, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      amax = fmaxf(amax, fabsf(x[e]));
      zero = fmaf(x[e], 0.f, zero);
    }
  }
  const bool strange = zero != zero;           // an infinity becomes the largest code, a NaN zero; neither counts for the scale
  if (strange) {
    amax = 0.f;
#pragma unroll 1
    for (int p = 0; p < PASSES; ++p) {
      if (ch.t0 + p * kRows + r >= ch.tk) continue;
      float x[8];
      values_of<T, HD, true>(piece_of(raw, p), mine, split, table, p * kRows + r, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool fine = fabsf(x[e]) < CUDART_INF_F;
        if (fine) amax = fmaxf(amax, fabsf(x[e]));
        odd = odd || !fine;
      }
    }
  }
  __syncwarp();
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if (!WARP) {
    if (tid % 32 == 0) red[tid / 32] = amax;
    __syncthreads();
    amax = red[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) amax = fmaxf(amax, red[w]);
  }
  const float fresh = scale_of(amax), now = ch.live > 0 ? fmaxf(old, fresh) : fresh, inv = 1.f / now;
  uint8_t* rows = codes + (((size_t)ch.seq * a.c.n_heads + head) * a.c.cap + ((size_t)ch.block << a.c.block_log2)) * HD;
  auto put_codes = [&](int p, float (&x)[8]) {
    uint8_t* at = rows + (size_t)(ch.live + p * kRows + r) * HD;
    const uint32_t lo = to_e4m3x4(x[0], x[1], x[2], x[3]), hi = to_e4m3x4(x[4], x[5], x[6], x[7]);
    if (split) {
      *reinterpret_cast<uint32_t*>(at + 4 * u) = lo;
      *reinterpret_cast<uint32_t*>(at + n_pairs + 4 * u) = hi;
    } else {
      *reinterpret_cast<uint2*>(at + 8 * u) = make_uint2(lo, hi);
    }
  };
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (strange || ch.t0 + p * kRows + r >= ch.tk) continue;
    float x[8];
    values_of<T, HD, false>(raw[p], mine, split, table, p * kRows + r, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= inv;
    put_codes(p, x);
  }
  if (strange) {
#pragma unroll 1
    for (int p = 0; p < PASSES; ++p) {
      if (ch.t0 + p * kRows + r >= ch.tk) continue;
      float x[8];
      values_of<T, HD, true>(piece_of(raw, p), mine, split, table, p * kRows + r, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] == x[e] ? x[e] * inv : 0.f;
      put_codes(p, x);
    }
  }
  if (ch.live > 0 && now > old) {              // the rows before these are rounded again
    const float f = old / now;
    uint32_t* w = reinterpret_cast<uint32_t*>(rows);
    for (int i = tid; i < ch.live * (HD / 4); i += WARP ? 32 : kThreads) w[i] = rescale_e4m3x4(w[i], f);
  }
  __syncwarp();
  if (tid == 0) *scale = now;                  // (every thread has read the old one: by a warp in step, or before the barrier)
}

// FEW: a chunk's rows fit a warp's passes.
template <typename T, int HD, bool FEW>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 3 : 1) quant_append_kernel(QAppendArgs a, int items_each) {
  constexpr int PASSES = FEW ? kFewPasses : 128 / kPassRows<HD, false>;
  extern __shared__ __align__(16) uint8_t smem[];
  float2* table = reinterpret_cast<float2*>(smem);     // [rows of the chunk][HD / 2] cosine, sine
  __shared__ float red[2][kWarps];
  grid_dep_launch();
  grid_dep_wait();
  const int tid = threadIdx.x, blk = 1 << a.c.block_log2;
  Chunk ch;
  ch.seq = blockIdx.z;
  int base = a.cache_len[ch.seq], n = a.row_count ? a.row_count[ch.seq] : a.n_rows;
  const int age0 = a.next_age ? a.next_age[ch.seq] : base;
  uint32_t bits = 0;
  if (n < 0 || n > a.n_rows) { bits |= VVS_DEV_BAD_ARG; n = 0; }
  if (base < 0 || base > a.c.cap - n) { bits |= VVS_DEV_CACHE_OVERFLOW; base = 0; n = 0; }
  if (bits && blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) atomicOr(a.status, bits);
  // the rows whose slots lie in the blockIdx.x-th block that the call reaches
  const int in_block = base & (blk - 1), chunk = blockIdx.x;
  ch.t0 = max(0, chunk * blk - in_block);
  ch.t1 = min(a.n_rows, (chunk + 1) * blk - in_block);
  if (ch.t0 >= ch.t1) return;
  ch.tk = min(ch.t1, n);
  ch.block = (base >> a.c.block_log2) + chunk;
  ch.live = chunk == 0 ? in_block : 0;
  // items: keys of every head, queries of every head (few rows), values of every head
  const int kv = a.c.n_heads, qs = FEW ? a.n_heads : 0, i0 = blockIdx.y * items_each, i1 = min(2 * kv + qs, i0 + items_each);
  const int mine = FEW ? i0 + tid / 32 : i0, step = FEW ? kWarps : 1;
  const bool rope = a.rope.inv_freq != nullptr;
  const int u = tid % (HD / 8), r = (FEW ? tid % 32 : tid) / (HD / 8);
  auto is_query = [&](int i) { return FEW && i >= kv && i < kv + qs; };
  auto request = [&](int i, Unit<T> (&raw)[PASSES]) {
    if (i >= i1) return;
    const bool query = is_query(i), split = rope && i < kv + qs && unit_split(a.rope, u);
    request_rows<T, HD, PASSES, FEW>(a, query ? a.q : i < kv ? a.k : a.v, ch, query ? i - kv : i < kv ? i : i - kv - qs, query ? ch.t1 : ch.tk,
                                     !query && a.row_index, split, raw);
  };
  Unit<T> raw[PASSES];
  request(mine, raw);                          // travels beside the table
  if (rope && i0 < kv + qs) {
    // a thread has one pair of every kStep-th row; the positions of several rows travel together
    constexpr int kStep = kThreads / (HD / 2), kTogether = FEW ? 4 : 8;
    const int pair = tid % (HD / 2), rows = ch.t1 - ch.t0;
    const PairAxis pa = pair_axis(a.rope, pair, a.c.n_seqs, a.n_rows, a.status);
    for (int t0 = tid / (HD / 2); t0 < rows; t0 += kTogether * kStep) {
      int pos[kTogether];
#pragma unroll
      for (int j = 0; j < kTogether; ++j) {
        const int t = ch.t0 + min(t0 + j * kStep, rows - 1);
        int from = t;
        if (a.row_index && t < ch.tk) from = min(max(a.row_index[(size_t)ch.seq * a.n_rows + t], 0), a.n_rows - 1);
        pos[j] = pa.pos ? pa.pos[(size_t)ch.seq * a.n_rows + from] : 0;
      }
#pragma unroll
      for (int j = 0; j < kTogether; ++j) {
        const int t = t0 + j * kStep;
        if (t >= rows) break;
        float2 cs;
        sincosf(__fmul_rn((float)pos[j], pa.freq), &cs.y, &cs.x);
        if (!pa.pos) cs = make_float2(kStays, CUDART_NAN_F);       // (a piece with such a pair takes the way of the infinities)
        table[t * (HD / 2) + pair] = cs;
      }
    }
    __syncthreads();
  }
  // of queries: where this thread's pieces lie, and the pairs of them that are turned
  const bool apart = rope && unit_split(a.rope, u);
  uint32_t pairs = 0;
  if (FEW && rope && i0 < kv + qs && unit_turns(a.rope, u)) {
    float c[4], s[4];
    angles_of<HD>(table, 0, c, s);
    pairs = pairs_of(c);
  }
  bool odd = false;
  int use = 0;                                 // the maxima's room in turns: one barrier a head is enough
  for (int i = mine; i < i1; i += step) {
    if (is_query(i)) {
      auto put_query = [&](int p, const Unit<T>& piece, bool some) {
        const int in = p * kPassRows<HD, FEW> + r, t = ch.t0 + in;
        if (t >= ch.t1) return;
        Unit<T> out = piece;
        if (pairs) {
          float c[4], s[4];
          angles_of<HD>(table, in, c, s);
          out = some ? turned_some(piece, apart, c, s, pairs) : turned_unit(piece, apart, c, s);
        }
        store_unit(static_cast<T*>(a.q_out.data) + ch.seq * a.q_out.seq + (i - kv) * a.q_out.head + t * a.q_out.row +
                       unit_at(u, apart),
                   apart, a.rope.n_pairs, out);
      };
      if (!pairs || pairs == kAllPairs) {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) put_query(p, raw[p], false);
      } else {
#pragma unroll 1
        for (int p = 0; p < PASSES; ++p) put_query(p, piece_of(raw, p), true);
      }
    } else if (ch.t0 < ch.tk) {
      const bool key = i < kv;
      const int head = key ? i : i - kv - qs, at = FEW ? tid % 32 : tid;
      put_rows<T, HD, PASSES, FEW>(a, raw, key && rope, key ? a.c.k : a.c.v, key ? a.c.k_scale : a.c.v_scale, ch, head, table,
                                   red[use ^= 1], odd);
      if (key && at < ch.tk - ch.t0) {         // (few rows are at most 32)
        const size_t slot = ((size_t)ch.seq * kv + head) * a.c.cap + base + ch.t0 + at;
        if (a.c.mass) a.c.mass[slot] = 0.f;
        if (a.c.age) a.c.age[slot] = age0 + ch.t0 + at;
      }
    }
    __syncwarp();
    request(i + step, raw);
  }
  if (odd) atomicOr(a.status, VVS_DEV_NONFINITE);
}

template <typename T, int HD, bool FEW>
int launch_rows(const QAppendArgs& a, cudaStream_t s) {
  const int blk = 1 << a.c.block_log2, rows = a.n_rows < blk ? a.n_rows : blk;
  const int chunks = (a.n_rows + blk - 2) / blk + 1, items = 2 * a.c.n_heads + (FEW ? a.n_heads : 0);
  const size_t smem = a.rope.inv_freq ? (size_t)rows * (HD / 2) * sizeof(float2) : 0;
  // Heads of a CTA: few rows, one for each warp (fewer where that leaves SMs without work).  Prompts, as many as leave every SM six
  // CTAs (71.5 us; two 75.8, sixteen 70.4): the cosines and sines of the rows serve all of them.
  const long long each_head = (long long)chunks * a.c.n_seqs;
  int each;
  if (FEW) {
    each = kWarps;
    while (each > 1 && each_head * ((items + each - 1) / each) < a.n_sms) each /= 2;
  } else {
    long long groups = (6LL * a.n_sms + each_head - 1) / each_head;
    groups = groups > items ? items : groups;
    each = (int)((items + groups - 1) / groups);
  }
  auto kernel = quant_append_kernel<T, HD, FEW>;
  if (ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), (int)smem) != cudaSuccess) return VVS_ERR_CUDA;
  const cudaError_t e = launch_kernel(kernel, dim3(chunks, (items + each - 1) / each, a.c.n_seqs), dim3(kThreads), smem, true, s, a, each);
  return e == cudaSuccess ? VVS_OK : VVS_ERR_CUDA;
}

// A call of few rows, or of small blocks, is one launch: two blocks of 9 rows 5.5 us, a CTA for a head and the queries by themselves 7.2; 32
// blocks 8.6 against 25.0.  Of prompts the queries have a launch of their own, whose threads keep their
// angles in registers and have no block to wait for.
template <typename T, int HD>
int launch_hd(const QAppendArgs& a, cudaStream_t s) {
  const int blk = 1 << a.c.block_log2, rows = a.n_rows < blk ? a.n_rows : blk;
  if (rows <= kFewPasses * kPassRows<HD, true>) return launch_rows<T, HD, true>(a, s);
  if (a.n_heads > 0) {
    RotateArgs ra{};
    ra.rope = a.rope; ra.q = a.q; ra.q_out = a.q_out;
    ra.n_seqs = a.c.n_seqs; ra.n_rows = a.n_rows; ra.n_heads = a.n_heads; ra.hd = HD; ra.status = a.status; ra.n_sms = a.n_sms;
    const int rc = launch_rotate_axes<T>(ra, s);
    if (rc != VVS_OK) return rc;
  }
  return launch_rows<T, HD, false>(a, s);
}

}  // namespace

template <typename T>
int launch_quant_append(const QAppendArgs& a, cudaStream_t s) {
  return a.c.hd == 64 ? launch_hd<T, 64>(a, s) : launch_hd<T, 128>(a, s);
}
template int launch_quant_append<float>(const QAppendArgs&, cudaStream_t);
template int launch_quant_append<__nv_bfloat16>(const QAppendArgs&, cudaStream_t);

}  // namespace vvs
