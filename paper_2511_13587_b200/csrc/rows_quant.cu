// Rows, or SwiGLU's silu(gate) * rows, to e4m3 with a scale for each 128 columns; weights with one for each 128 x 128 elements.
//
//   y = x  or  gate / (1 + exp(-gate)) * x,  scale = max |y| / 448 over the block,  code = e4m3(y / scale)
//
// Bound by HBM (every element is read once and stays in registers until its code is written), small calls by the launch.  Rows: half a
// warp has a block of 128 columns, eight elements a lane; SwiGLU's also by the exponential's and the reciprocal's pipe (64 % of its rate at 57 us).
// Weights: a CTA has a block of 128 x 128, eight units of eight elements a thread.
//
// 5460 rows of 11008, gate and up: 60 us, 5.0 TB/s (78 % of a copy's rate; 53.8 for the same rows each time); 18 of 3456 3.6 us, as long as the call
// (1.4 in a graph).  22016 x 4096 weights 49.5 us, 5.5 TB/s (46.5 for the same each time; two CTAs of 512 threads an SM 50, one of 1024 88).
#include "block_quant.cuh"

namespace vvs {

namespace {

constexpr int kThreads = 256;
// Rows whose elements are on their way together, at four CTAs an SM: four (two, eight CTAs: 5 % slower), of float32 with gates two, for four do not fit
// the registers (2730 rows of 11008: 41.5 us, with four 64).
template <typename T, bool GATE>
constexpr int kFlight = sizeof(T) == 4 && GATE ? 2 : 4;

// gate / (1 + e^-gate) * x: within 2^-17, most of it by the exponent, whose product and constant round (1.3 * 2^-24 of 126 at most).  From e^-gate = 2^126
// on (gates below -87.3) the reciprocal is no normal number and the result 0, |y| below 2^-119 |x|.  (What large elements leave of that by a second
// form for such gates: 5460 rows of 11008 56.3 to 57.2 us for 53.8, whichever way they were looked for.)
__device__ __forceinline__ float gated(float gate, float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + ex2(gate * -1.442695041f)));
  return gate * r * x;
}

// A CTA has up to sixteen blocks of columns, a half warp each, and goes through `each` rows.
template <typename T, bool GATE>
__global__ void __launch_bounds__(kThreads, 4) rows_quant_kernel(RowsQuantArgs a, int each) {
  constexpr int kAt = kFlight<T, GATE>;
  grid_dep_launch();
  grid_dep_wait();
  const int nb = qblocks(a.n_cols), block = blockIdx.x * (blockDim.x >> 4) + (threadIdx.x >> 4), col = block * kQBlock + 8 * (threadIdx.x & 15);
  const bool in = col < a.n_cols;
  const int r0 = blockIdx.y * each, r1 = min(a.n_rows, r0 + each);
  const T* x = static_cast<const T*>(a.x.data) + (int64_t)r0 * a.x.row + col;
  const T* g = static_cast<const T*>(a.gate.data) + (int64_t)r0 * a.gate.row + col;
  uint8_t* codes = a.codes + (int64_t)r0 * a.codes_row + col;
  float* scale_at = a.scale + (size_t)r0 * nb + block;
  bool strange = false;
  for (int r = r0; r < r1; r += kAt) {
    Unit<T> ux[kAt], ug[kAt];
#pragma unroll
    for (int j = 0; j < kAt; ++j) {
      const bool there = in && r + j < r1;
      ux[j] = there ? load_unit(x, false, 0) : no_unit<T>();
      if (GATE) ug[j] = there ? load_unit(g, false, 0) : no_unit<T>();
      x += a.x.row;
      if (GATE) g += a.gate.row;
    }
#pragma unroll
    for (int j = 0; j < kAt; ++j) {
      if (r + j >= r1) break;                      // (of all lanes)
      float y[8];
      widen_unit(ux[j], y);
      if (GATE) {
        float z[8];
        widen_unit(ug[j], z);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = gated(z[e], y[e]);
      }
      float m = amax8(y);
      const bool some = odd(m);
      if (some) m = amax8_finite(y);
      const float scale = block_scale(half_warp_max(m));
      if (some) {
        strange = true;
        hold8(y, scale);
      }
      if (in) {
        *reinterpret_cast<uint2*>(codes) = codes8(y, scale, minus_inverse(scale));
        if ((threadIdx.x & 15) == 0) *scale_at = scale;
      }
      codes += a.codes_row;
      scale_at += nb;
    }
  }
  if (strange) atomicOr(a.status, VVS_DEV_NONFINITE);
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 3) weight_quant_kernel(RowsQuantArgs a) {
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
  bool strange = false;
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    float y[8];
    widen_unit(x[j], y);
    float n = amax8(y);
    if (odd(n)) {
      strange = true;
      n = amax8_finite(y);
    }
    m = fmaxf(m, n);
  }
  m = half_warp_max(m);
  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
  if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) m = fmaxf(m, s_max[i]);
  const float scale = block_scale(m), inv = minus_inverse(scale);
  if (threadIdx.x == 0) a.scale[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = scale;
#pragma unroll
  for (int j = 0; j < kUnits; ++j) {
    const long long row = r0 + j * kRows;
    float y[8];
    widen_unit(x[j], y);
    if (strange) {
      amax8_finite(y);
      hold8(y, scale);
    }
    if (in && row < a.n_rows) *reinterpret_cast<uint2*>(a.codes + row * a.codes_row + col) = codes8(y, scale, inv);
  }
  if (strange) atomicOr(a.status, VVS_DEV_NONFINITE);
}

}  // namespace

template <typename T>
int launch_rows_quant(const RowsQuantArgs& a, cudaStream_t s) {
  // Blocks of columns by CTAs of sixteen at most, an even number each (27 blocks: two of fourteen); rows by as many as are on the device together
  const int nb = qblocks(a.n_cols), groups = (nb + 15) / 16, mine = ((nb + groups - 1) / groups + 1) & ~1;
  const long long most = std::max(1LL, (long long)a.n_sms * 4 * (kThreads / (16 * mine)) / groups);
  long long each = (a.n_rows + most - 1) / most;
  if (each > 1) each = (each + 3) / 4 * 4;          // (of either number in flight)
  each = std::max(each, (a.n_rows + 65534LL) / 65535);
  auto* fn = a.gate.data ? rows_quant_kernel<T, true> : rows_quant_kernel<T, false>;
  const cudaError_t e =
      launch_kernel(fn, dim3(groups, (unsigned)((a.n_rows + each - 1) / each)), dim3(16 * mine), 0, true, s, a, (int)each);
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
