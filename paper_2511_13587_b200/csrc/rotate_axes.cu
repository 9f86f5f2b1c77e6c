// Rotary positions with several axes on the query and key heads of a block of rows.  Reads every element once and writes it
// once: bound by HBM for prompts, by the launch for a step's rows.  A thread has one unit of eight elements of a row, computes its
// four angles once and goes through a group of heads with them: sines and cosines of float32 angles (some 40 instructions each)
// cost more than the elements' traffic if every head computes its own.
//
// 5460 rows of 32 + 8 heads of 128: 23.8 us, 4.7 TB/s (73 % of a copy's rate); 18 rows of 40 heads of 64 4.2 us, as long as the call itself.
#include "quant_cache.cuh"

namespace vvs {

namespace {

constexpr int kThreads = 128;
constexpr int kFlight = 4;   // heads whose elements are on their way together (23.7 us; one 30.9; eight, with their registers, 33.2)

template <typename T>
__global__ void __launch_bounds__(kThreads, 7) rotate_axes_kernel(RotateArgs a, int heads_each) {
  grid_dep_launch();
  grid_dep_wait();
  const int units = a.hd / 8;
  const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (i >= (long long)a.n_seqs * a.n_rows * units) return;
  const int u = (int)(i % units);
  const int at = (int)(i / units), row = at % a.n_rows, seq = at / a.n_rows;
  const bool split = unit_split(a.rope, u);
  const int heads = a.n_heads + a.n_kv_heads, h0 = blockIdx.y * heads_each, h1 = min(heads, h0 + heads_each);
  const T* q = static_cast<const T*>(a.q.data) + seq * a.q.seq + row * a.q.row + unit_at(u, split);
  const T* k = static_cast<const T*>(a.k.data) + seq * a.k.seq + row * a.k.row + unit_at(u, split);
  T* qo = static_cast<T*>(a.q_out.data) + seq * a.q_out.seq + row * a.q_out.row + unit_at(u, split);
  T* ko = static_cast<T*>(a.k_out.data) + seq * a.k_out.seq + row * a.k_out.row + unit_at(u, split);
  auto request = [&](int h, Unit<T> (&x)[kFlight]) {
#pragma unroll
    for (int j = 0; j < kFlight; ++j)
      if (h + j < h1) x[j] = load_unit(h + j < a.n_heads ? q + (h + j) * a.q.head : k + (h + j - a.n_heads) * a.k.head, split, a.rope.n_pairs);
  };
  // the first heads travel beside the angles, the next ones beside the turning
  Unit<T> x[kFlight];
  request(h0, x);
  float c[4], s[4];
  int pos[4];
  PairAxis pa[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) pa[j] = pair_axis(a.rope, 4 * u + j, a.n_seqs, a.n_rows, a.status);
#pragma unroll
  for (int j = 0; j < 4; ++j) pos[j] = pa[j].pos ? pa[j].pos[(size_t)seq * a.n_rows + row] : 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) sincosf(__fmul_rn((float)pos[j], pa[j].freq), &s[j], &c[j]);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (!pa[j].pos) c[j] = kStays;
  const bool some = pairs_of(c) != kAllPairs;
  auto at_out = [&](int h) { return h < a.n_heads ? qo + h * a.q_out.head : ko + (h - a.n_heads) * a.k_out.head; };
  for (int h = h0; h < h1; h += kFlight) {
    Unit<T> next[kFlight];
    request(h + kFlight, next);
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      if (h + j >= h1) break;
      Unit<T> out = turned_unit(x[j], split, c, s);
      if (some) put_back(out, x[j], split, pairs_of(c));
      store_unit(at_out(h + j), split, a.rope.n_pairs, out);
      x[j] = next[j];
    }
  }
}

}  // namespace

template <typename T>
int launch_rotate_axes(const RotateArgs& a, cudaStream_t s) {
  const long long threads = (long long)a.n_seqs * a.n_rows * (a.hd / 8);
  const int heads = a.n_heads + a.n_kv_heads;
  // as many groups of heads as fill the device with threads (2048 an SM): 18 rows 4.2 us, with all heads in one thread 9.6
  const long long room = (long long)a.n_sms * 2048;
  int groups = (int)((room + threads - 1) / threads);
  groups = groups < 1 ? 1 : groups > heads ? heads : groups;
  const int each = (heads + groups - 1) / groups;
  const long long blocks = (threads + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffffLL) return VVS_ERR_SHAPE;
  const cudaError_t e = launch_kernel(rotate_axes_kernel<T>, dim3((unsigned)blocks, (heads + each - 1) / each), dim3(kThreads), 0, true, s, a, each);
  return e == cudaSuccess ? VVS_OK : VVS_ERR_CUDA;
}
template int launch_rotate_axes<float>(const RotateArgs&, cudaStream_t);
template int launch_rotate_axes<__nv_bfloat16>(const RotateArgs&, cudaStream_t);

}  // namespace vvs
