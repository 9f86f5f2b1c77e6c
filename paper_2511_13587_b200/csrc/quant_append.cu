// Appends a block's keys and values to the 8-bit cache: rotation, one scale for each (block of slots, head), e4m3 codes; the query
// heads of the same rows are rotated in the same launch.  Every input is read once and every output written once: bound by HBM for
// prompts, by the launch and one round trip for a step's rows.  A CTA has the rows that fall into one block of slots, and some of the
// heads: a head's rows stay in registers between the maximum that fixes the scale and the rounding.  Cosines and sines of the CTA's rows
// are computed once, into shared memory, for all of its heads.
#include "quant_cache.cuh"

namespace vvs {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// rows of a pass: 32 of 64, 16 of 128 elements; a block has at most 128
template <int HD>
constexpr int kPassRows = kThreads / (HD / 8);

template <typename T, int HD, int PASSES>
__device__ __forceinline__ void put_rows(const QAppendArgs& a, const HeadRows& src, bool turned, uint8_t* codes, float* scales, int seq, int head,
                                         int block, int live, int t0, int t1, const float2* table, float* red, bool& odd) {
  constexpr int kUnits = HD / 8, kRows = kPassRows<HD>;
  const int tid = threadIdx.x, u = tid % kUnits, r = tid / kUnits, n_pairs = a.rope.n_pairs;
  const bool split = turned && unit_split(a.rope, u);
  const T* base = static_cast<const T*>(src.data) + seq * src.seq + head * src.head;
  float* scale = scales + ((size_t)seq * a.c.n_heads + head) * (a.c.cap >> a.c.block_log2) + block;
  const float old = live > 0 ? *scale : 0.f;
  // the rows as they are stored; they are turned twice, for the maximum and for the codes, which takes fewer registers than one turned
  // copy (bf16: half, and 80 of a thread in the place of 213)
  Unit<T> raw[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int t = t0 + p * kRows + r;
    if (t >= t1) continue;
    const int from = a.row_index ? a.row_index[(size_t)seq * a.n_rows + t] : t;
    if (from >= 0 && from < a.n_rows) {
      raw[p] = load_unit_raw(base + from * src.row, u, split, n_pairs);
    } else {
      raw[p] = Unit<T>{};
      atomicOr(a.status, VVS_DEV_BAD_ARG);
    }
  }
  const bool mine = turned && (split || !a.rope.halves);
  auto value = [&](int p, float (&x)[8]) {
    widen_unit(raw[p], x);
    if (mine) {
      const float2* cs = table + (size_t)(p * kRows + r) * (HD / 2) + 4 * u;
      float c[4], s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) { c[j] = cs[j].x; s[j] = cs[j].y; }
      turn_unit(x, split, c, s);
    }
  };
  float amax = 0.f;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (t0 + p * kRows + r >= t1) continue;
    float x[8];
    value(p, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float m = fabsf(x[e]);
      if (m < CUDART_INF_F) amax = fmaxf(amax, m);
      else odd = true;                         // an infinity becomes the largest code, a NaN zero
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if (tid % 32 == 0) red[tid / 32] = amax;
  __syncthreads();
  amax = red[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) amax = fmaxf(amax, red[w]);
  const float fresh = scale_of(amax), now = live > 0 ? fmaxf(old, fresh) : fresh, inv = 1.f / now;
  uint8_t* rows = codes + (((size_t)seq * a.c.n_heads + head) * a.c.cap + ((size_t)block << a.c.block_log2)) * HD;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int t = t0 + p * kRows + r;
    if (t >= t1) continue;
    uint8_t* at = rows + (size_t)(live + t - t0) * HD;
    float x[8];
    value(p, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] == x[e] ? x[e] * inv : 0.f;
    const uint32_t lo = to_e4m3x4(x[0], x[1], x[2], x[3]), hi = to_e4m3x4(x[4], x[5], x[6], x[7]);
    if (split) {
      *reinterpret_cast<uint32_t*>(at + 4 * u) = lo;
      *reinterpret_cast<uint32_t*>(at + n_pairs + 4 * u) = hi;
    } else {
      *reinterpret_cast<uint2*>(at + 8 * u) = make_uint2(lo, hi);
    }
  }
  if (live > 0 && now > old) {                 // the rows before these are rounded again
    const float f = old / now;
    uint32_t* w = reinterpret_cast<uint32_t*>(rows);
    for (int i = tid; i < live * (HD / 4); i += kThreads) w[i] = rescale_e4m3x4(w[i], f);
  }
  if (tid == 0) *scale = now;
}

template <typename T, int HD, int PASSES>
__global__ void __launch_bounds__(kThreads) quant_append_kernel(QAppendArgs a, int items_each) {
  extern __shared__ __align__(16) uint8_t smem[];
  float2* table = reinterpret_cast<float2*>(smem);     // [rows of the chunk][HD / 2] cosine, sine
  __shared__ float red[2][kWarps];
  grid_dep_launch();
  grid_dep_wait();
  const int seq = blockIdx.z, tid = threadIdx.x, blk = 1 << a.c.block_log2;
  int base = a.cache_len[seq], n = a.row_count ? a.row_count[seq] : a.n_rows;
  const int age0 = a.next_age ? a.next_age[seq] : base;
  uint32_t bits = 0;
  if (n < 0 || n > a.n_rows) { bits |= VVS_DEV_BAD_ARG; n = 0; }
  if (base < 0 || base > a.c.cap - n) { bits |= VVS_DEV_CACHE_OVERFLOW; base = 0; n = 0; }
  if (bits && blockIdx.x == 0 && blockIdx.y == 0 && tid == 0) atomicOr(a.status, bits);
  // rows t0 .. t1 - 1 of the call: those whose slots lie in the blockIdx.x-th block that the call reaches
  const int in_block = base & (blk - 1), chunk = blockIdx.x;
  const int t0 = max(0, chunk * blk - in_block), t1 = min(a.n_rows, (chunk + 1) * blk - in_block);
  if (t0 >= t1) return;
  const int block = (base >> a.c.block_log2) + chunk, live = chunk == 0 ? in_block : 0, tk = min(t1, n);
  const int kv = a.c.n_heads, i0 = blockIdx.y * items_each, i1 = min(2 * kv + a.n_heads, i0 + items_each);
  // items: keys of every head, queries of every head, values of every head
  const bool turned = a.rope.inv_freq != nullptr;
  if (turned && i0 < kv + a.n_heads) {
    for (int i = tid; i < (t1 - t0) * (HD / 2); i += kThreads) {
      const int t = t0 + i / (HD / 2);
      int from = t;
      if (a.row_index && t < tk) from = min(max(a.row_index[(size_t)seq * a.n_rows + t], 0), a.n_rows - 1);
      float c, s;
      pair_turn(a.rope, i % (HD / 2), seq, from, a.c.n_seqs, a.n_rows, a.status, c, s);
      table[i] = make_float2(c, s);
    }
    __syncthreads();
  }
  bool odd = false;
  int use = 0;                                 // the sums' room in turns: one barrier a head is enough
  for (int i = i0; i < i1; ++i) {
    if (i < kv || i >= kv + a.n_heads) {
      if (t0 >= tk) continue;
      const bool key = i < kv;
      const int head = key ? i : i - kv - a.n_heads;
      put_rows<T, HD, PASSES>(a, key ? a.k : a.v, key && turned, key ? a.c.k : a.c.v, key ? a.c.k_scale : a.c.v_scale, seq, head, block, live,
                              t0, tk, table, red[use ^= 1], odd);
      if (key && tid < tk - t0) {
        const size_t slot = ((size_t)seq * kv + head) * a.c.cap + base + t0 + tid;
        if (a.c.mass) a.c.mass[slot] = 0.f;
        if (a.c.age) a.c.age[slot] = age0 + t0 + tid;
      }
    } else {
      const int head = i - kv;
      const T* from = static_cast<const T*>(a.q.data) + seq * a.q.seq + head * a.q.head;
      T* to = static_cast<T*>(a.q_out.data) + seq * a.q_out.seq + head * a.q_out.head;
      constexpr int kUnits = HD / 8, kRows = kPassRows<HD>;
      const int u = tid % kUnits, r = tid / kUnits;
      const bool split = turned && unit_split(a.rope, u);
      const bool mine = turned && (split || !a.rope.halves);
      Unit<T> raw[PASSES];
#pragma unroll
      for (int p = 0; p < PASSES; ++p)
        if (t0 + p * kRows + r < t1) raw[p] = load_unit_raw(from + (t0 + p * kRows + r) * a.q.row, u, split, a.rope.n_pairs);
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int t = t0 + p * kRows + r;
        if (t >= t1) continue;
        float x[8];
        widen_unit(raw[p], x);
        if (mine) {
          const float2* cs = table + (size_t)(t - t0) * (HD / 2) + 4 * u;
          float c[4], s[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) { c[j] = cs[j].x; s[j] = cs[j].y; }
          turn_unit(x, split, c, s);
        }
        store_unit(to + t * a.q_out.row, u, split, a.rope.n_pairs, x);
      }
    }
  }
  if (odd) atomicOr(a.status, VVS_DEV_NONFINITE);
}

template <typename T, int HD, int PASSES>
int launch_passes(const QAppendArgs& a, cudaStream_t s) {
  const int blk = 1 << a.c.block_log2, rows = a.n_rows < blk ? a.n_rows : blk;
  const int chunks = (a.n_rows + blk - 2) / blk + 1, items = 2 * a.c.n_heads + a.n_heads;
  const size_t smem = a.rope.inv_freq ? (size_t)rows * (HD / 2) * sizeof(float2) : 0;
  // as many groups of heads as keep every SM busy with eight CTAs (four of long blocks, whose sines cost more than their elements'
  // traffic unless they serve several heads)
  const long long room = (rows > 32 ? 4LL : 8LL) * a.n_sms, each_head = (long long)chunks * a.c.n_seqs;
  long long groups = (room + each_head - 1) / each_head;
  groups = groups > items ? items : groups;
  const int each = (int)((items + groups - 1) / groups);
  auto kernel = quant_append_kernel<T, HD, PASSES>;
  if (ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), (int)smem) != cudaSuccess) return VVS_ERR_CUDA;
  const cudaError_t e = launch_kernel(kernel, dim3(chunks, (items + each - 1) / each, a.c.n_seqs), dim3(kThreads), smem, true, s, a, each);
  return e == cudaSuccess ? VVS_OK : VVS_ERR_CUDA;
}

// a call of few rows, or of small blocks, keeps fewer rows of a head in registers
template <typename T, int HD>
int launch_hd(const QAppendArgs& a, cudaStream_t s) {
  const int blk = 1 << a.c.block_log2, rows = a.n_rows < blk ? a.n_rows : blk;
  if (rows <= kPassRows<HD>) return launch_passes<T, HD, 1>(a, s);
  return launch_passes<T, HD, 128 / kPassRows<HD>>(a, s);
}

}  // namespace

template <typename T>
int launch_quant_append(const QAppendArgs& a, cudaStream_t s) {
  return a.c.hd == 64 ? launch_hd<T, 64>(a, s) : launch_hd<T, 128>(a, s);
}
template int launch_quant_append<float>(const QAppendArgs&, cudaStream_t);
template int launch_quant_append<__nv_bfloat16>(const QAppendArgs&, cudaStream_t);

}  // namespace vvs
