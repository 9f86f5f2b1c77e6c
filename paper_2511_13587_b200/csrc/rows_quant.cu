// Rows, or SwiGLU's silu(gate) * rows, to e4m3 with a scale for each 128 columns; weights with one for each 128 x 128 elements.
//
//   y = x  or  gate / (1 + exp(-gate)) * x,  scale = max |y| / 448 over the block,  code = e4m3(y / scale)
//
// Bound by HBM (every element is read once and stays in registers until its code is written), small calls by the launch.  Rows: half a
// warp has a block of 128 columns, eight elements a lane.  Weights: a CTA has a block of 128 x 128, eight units of eight elements a thread.
#include "block_quant.cuh"

namespace vvs {

namespace {

constexpr int kThreads = 256;
constexpr int kFlight = 4;                         // blocks of a half warp whose elements are on their way together

template <typename T, bool GATE>
__global__ void __launch_bounds__(kThreads) rows_quant_kernel(RowsQuantArgs a, int each) {
  grid_dep_launch();
  grid_dep_wait();
  const int nb = qblocks(a.n_cols), lane16 = threadIdx.x & 15;
  const int total = a.n_rows * nb, first = (int)((blockIdx.x * kThreads + threadIdx.x) >> 4), step = (int)(gridDim.x * (kThreads / 16));
  bool odd = false;
  // (both halves of a warp take as many turns: `first` of the second is one more)
  for (int i = 0; i < each; i += kFlight) {
    Unit<T> x[kFlight], g[kFlight];
    int row[kFlight], col[kFlight];
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      const int b = first + (i + j) * step;                        // (below 2^31: kMaxBlocks)
      row[j] = b / nb;
      col[j] = (b - row[j] * nb) * kQBlock + 8 * lane16;
      const bool in = i + j < each && b < total && col[j] < a.n_cols;
      if (!in) row[j] = -1;
      x[j] = in ? load8<T>(a.x.data, row[j] * a.x.row + col[j]) : no_unit<T>();
      if (GATE) g[j] = in ? load8<T>(a.gate.data, row[j] * a.gate.row + col[j]) : no_unit<T>();
    }
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
      float y[8];
      widen_unit(x[j], y);
      if (GATE) {
        float z[8];
        widen_unit(g[j], z);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= __fdividef(z[e], 1.f + __expf(-z[e]));
      }
      float m = amax8(y);
      if (odd8(y)) {
        odd = true;
        m = amax8_finite(y);
        no_nan8(y);
      }
      const float scale = block_scale(half_warp_max(m));
      const uint2 c = codes8(y, __frcp_rn(scale));
      if (row[j] >= 0) {
        *reinterpret_cast<uint2*>(a.codes + row[j] * a.codes_row + col[j]) = c;
        if (lane16 == 0) a.scale[(size_t)row[j] * nb + (col[j] >> 7)] = scale;
      }
    }
  }
  if (odd) atomicOr(a.status, VVS_DEV_NONFINITE);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) weight_quant_kernel(RowsQuantArgs a) {
  __shared__ float s_max[kThreads / 32];
  constexpr int kRows = kThreads / 16, kUnits = kQBlock / kRows;   // rows that the CTA has at once, units of a thread
  grid_dep_wait();                                                 // (no early launch of what follows: it may read the codes ahead of its own wait)
  const int lane16 = threadIdx.x & 15, r0 = blockIdx.y * kQBlock + (threadIdx.x >> 4), col = blockIdx.x * kQBlock + 8 * lane16;
  const bool in = col < a.n_cols;
  Unit<T> x[kUnits];
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    const long long row = r0 + j * kRows;
    x[j] = in && row < a.n_rows ? load8<T>(a.x.data, row * a.x.row + col) : no_unit<T>();
  }
  float m = 0.f;
  bool odd = false;
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    float y[8];
    widen_unit(x[j], y);
    const bool strange = odd8(y);
    odd = odd || strange;
    m = fmaxf(m, strange ? amax8_finite(y) : amax8(y));
  }
  m = warp_max(m);
  if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) m = fmaxf(m, s_max[i]);
  const float scale = block_scale(m), inv = __frcp_rn(scale);
  if (threadIdx.x == 0) a.scale[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = scale;
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    const long long row = r0 + j * kRows;
    float y[8];
    widen_unit(x[j], y);
    if (odd) no_nan8(y);
    if (in && row < a.n_rows) *reinterpret_cast<uint2*>(a.codes + row * a.codes_row + col) = codes8(y, inv);
  }
  if (odd) atomicOr(a.status, VVS_DEV_NONFINITE);
}

}  // namespace

template <typename T>
int launch_rows_quant(const RowsQuantArgs& a, cudaStream_t s) {
  const long long total = (long long)a.n_rows * qblocks(a.n_cols), at_once = kThreads / 16;
  const long long most = (long long)a.n_sms * 8;                   // CTAs that are on the device together
  long long blocks = (total + at_once - 1) / at_once;
  if (blocks > most) {                                             // whole turns of kFlight blocks for each half warp
    const long long turns = (total + most * at_once * kFlight - 1) / (most * at_once * kFlight);
    blocks = (total + turns * kFlight * at_once - 1) / (turns * kFlight * at_once);
  }
  const long long each = (total + blocks * at_once - 1) / (blocks * at_once);
  auto* fn = a.gate.data ? rows_quant_kernel<T, true> : rows_quant_kernel<T, false>;
  const cudaError_t e = launch_kernel(fn, dim3((unsigned)blocks), dim3(kThreads), 0, true, s, a, (int)each);
  return e == cudaSuccess ? VVS_OK : VVS_ERR_CUDA;
}
template int launch_rows_quant<float>(const RowsQuantArgs&, cudaStream_t);
template int launch_rows_quant<__nv_bfloat16>(const RowsQuantArgs&, cudaStream_t);

template <typename T>
int launch_weight_quant(const RowsQuantArgs& a, cudaStream_t s) {
  const cudaError_t e =
      launch_kernel(weight_quant_kernel<T>, dim3(qblocks(a.n_cols), qblocks(a.n_rows)), dim3(kThreads), 0, true, s, a);
  return e == cudaSuccess ? VVS_OK : VVS_ERR_CUDA;
}
template int launch_weight_quant<float>(const RowsQuantArgs&, cudaStream_t);
template int launch_weight_quant<__nv_bfloat16>(const RowsQuantArgs&, cudaStream_t);

}  // namespace vvs
