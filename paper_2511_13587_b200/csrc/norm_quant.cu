// A residual is added, the sum normalised by its root mean square, and the row rounded to e4m3 with a scale for each 128 columns.
//
//   s = x + residual,  y_k = s_k / sqrt(sum_j s_j^2 / n + eps) * weight_k,  scale_b = max |y_k| / 448,  code_k = e4m3(y_k / scale_b)
//
// Every element is read once and stays in registers between the sum of squares, the block's maximum and its code: bound by HBM for
// prompts, by the launch and two dependent steps (sum over the row, maximum over a block) for a step's rows.  A thread has units of eight
// elements; the sixteen lanes of half a warp have a block of 128 columns, so that a block's maximum is four shuffles.
//
// 10408 rows of 4096, residual and sum: 54.5 us, 5.5 TB/s (85 % of a copy's rate; 48.2 for the same rows each time, some of which L2 has); 18
// rows of 1280 4.4 us, as long as the call (1.8 in a graph).
#include "block_quant.cuh"

namespace vvs {

namespace {

// Of all threads of a row: a warp, or the CTA.
__device__ __forceinline__ float row_sum(float v, float* s_sum, int t, int threads) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (threads > 32) {                              // (one row a CTA then)
    if ((t & 31) == 0) s_sum[t >> 5] = v;
    __syncthreads();
    v = (t & 31) < (threads >> 5) ? s_sum[t & 31] : 0.f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    v = __shfl_sync(0xffffffffu, v, 0);
  }
  return v;
}

// U: units of a thread.  blockDim (threads of a row, rows of a CTA).
template <typename T, int U>
__global__ void __launch_bounds__(512) norm_quant_kernel(NormQuantArgs a) {
  __shared__ float s_sum[16];
  grid_dep_launch();
  const int t = threadIdx.x, threads = blockDim.x;
  const int units = a.n_cols >> 3, nb = qblocks(a.n_cols);
  const int row = min(blockIdx.x * blockDim.y + threadIdx.y, a.n_rows - 1);        // (a row of its own that is not there: the last one again)
  const bool there = blockIdx.x * blockDim.y + threadIdx.y < (unsigned)a.n_rows;
  grid_dep_wait();
  Unit<T> x[U], r[U], w[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int u = j * threads + t;
    x[j] = u < units ? load8<T>(a.x.data, row * a.x.row + 8 * u) : no_unit<T>();
  }
  if (a.residual.data)
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int u = j * threads + t;
      r[j] = u < units ? load8<T>(a.residual.data, row * a.residual.row + 8 * u) : no_unit<T>();
    }
  constexpr bool kEarly = U * sizeof(T) <= 8;      // the norm's weights travel beside the row, where there are registers for both
  auto weights = [&](int j) {
    const int u = j * threads + t;
    w[j] = u < units ? load8<T>(a.weight, 8 * u) : no_unit<T>();
  };
  if (kEarly)
#pragma unroll
    for (int j = 0; j < U; ++j) weights(j);
  float y[U][8], ss = 0.f;
#pragma unroll
  for (int j = 0; j < U; ++j) {
    widen_unit(x[j], y[j]);
    if (a.residual.data) {
      float z[8];
      widen_unit(r[j], z);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[j][e] += z[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(y[j][e], y[j][e], ss);
  }
  if (a.sum_out.data && there)
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int u = j * threads + t;
      if (u < units) store_unit(static_cast<T*>(a.sum_out.data) + row * a.sum_out.row + 8 * u, false, 0, narrow_unit(y[j], x[j]));
    }
  ss = row_sum(ss, s_sum, t, threads);
  float mean = ss / (float)a.n_cols + a.eps;
  if (mean < 0x1p-100f) {                          // (of the whole row) squares that float32 does not hold well: the row times 2^96, its squares times 2^192
    constexpr float k = 0x1p96f;
    ss = 0.f;
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[j][e] *= k;
        ss = fmaf(y[j][e], y[j][e], ss);
      }
    if (threads > 32) __syncthreads();             // (the first sum has been read)
    ss = row_sum(ss, s_sum, t, threads);
    mean = ss / (float)a.n_cols + a.eps * k * k;
  }
  const float rs = rsqrtf(mean);
  bool strange = false;
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int u = j * threads + t;
    float g[8];
    if (!kEarly) weights(j);
    widen_unit(w[j], g);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[j][e] = y[j][e] * rs * g[e];
    if (a.norm_out.data && there && u < units)
      store_unit(static_cast<T*>(a.norm_out.data) + row * a.norm_out.row + 8 * u, false, 0, narrow_unit(y[j], x[j]));
    float m = amax8(y[j]);
    const bool some = odd(m);
    if (some) m = amax8_finite(y[j]);
    const float scale = block_scale(half_warp_max(m));
    if (some) {
      strange = true;
      hold8(y[j], scale);
    }
    const uint2 c = codes8(y[j], scale, minus_inverse(scale));
    if (there && u < units) {
      *reinterpret_cast<uint2*>(a.codes + row * a.codes_row + 8 * u) = c;
      if ((u & 15) == 0) a.scale[(size_t)row * nb + (u >> 4)] = scale;
    }
  }
  // (squares that are no float32 numbers have made the row zeros)
  if ((strange || odd(ss)) && there) atomicOr(a.status, VVS_DEV_NONFINITE);
}

}  // namespace

template <typename T>
int launch_norm_quant(const NormQuantArgs& a, cudaStream_t s) {
  const int units = a.n_cols / 8;
  // Units of a thread: one as long as that leaves at most 2048 threads an SM, else up to four (two of float32), where whole warps do not leave
  // more lanes idle for it.  Microseconds with 1 / 2 / 4 units, of the same rows each time: 18 rows of 1280 1.76 / 1.88 / 2.39, 288 of 4096 3.05 / 3.93 / 4.63,
  // 10408 of 4096 62.4 / 50.8 / 48.2, 40000 of 256 12.3 / 17.9 / 32.7; float32, 5204 of 4096 42.8 / 42.2 / 45.5.  (Eight, for rows that are wider than 512
  // threads' four.)
  const long long room = (long long)a.n_sms * 2048;
  auto threads_of = [&](int per) { return ((units + per - 1) / per + 31) / 32 * 32; };
  int per = 1;
  while (per < (sizeof(T) == 2 ? 4 : 2) && (long long)a.n_rows * units > room * per && threads_of(2 * per) * 8 <= threads_of(per) * 5) per *= 2;
  while (per < 8 && threads_of(per) > 512) per *= 2;
  const int threads = threads_of(per);
  if (threads > 512) return VVS_ERR_SHAPE;
  const int rows = threads == 32 ? 4 : 1;
  auto* fn = per == 1 ? norm_quant_kernel<T, 1> : per == 2 ? norm_quant_kernel<T, 2> : per == 4 ? norm_quant_kernel<T, 4> : norm_quant_kernel<T, 8>;
  const cudaError_t e = launch_kernel(fn, dim3((a.n_rows + rows - 1) / rows), dim3(threads, rows), 0, true, s, a);
  return e == cudaSuccess ? VVS_OK : VVS_ERR_CUDA;
}
template int launch_norm_quant<float>(const NormQuantArgs&, cudaStream_t);
template int launch_norm_quant<__nv_bfloat16>(const NormQuantArgs&, cudaStream_t);

}  // namespace vvs
