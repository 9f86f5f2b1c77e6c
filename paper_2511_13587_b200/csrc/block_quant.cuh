// Rows and weights in e4m3 with one float32 scale for each block of 128 columns (128 x 128 elements of a weight), and their product:
// parameters of the kernels, and what several of them do with a value.
#pragma once

#include <algorithm>

#include "quant_cache.cuh"

namespace vvs {

constexpr int kQBlock = 128;                       // columns (and rows of a weight) that share a scale
constexpr int kNormMaxCols = 32768;                // widest row of vvs_norm_quant: 512 threads of 64 elements each
constexpr int kMaxCols = 1 << 30;                  // (a column behind the last block is still an int)
constexpr int kMaxBlocks = 1 << 30;                // blocks of a call's rows
__host__ __device__ __forceinline__ int qblocks(int n) { return (n + kQBlock - 1) / kQBlock; }

struct RowsArg {
  void* data;                                      // null: not given
  int64_t row;                                     // elements from one row to the next
};

struct NormQuantArgs {
  RowsArg x, residual, sum_out, norm_out;
  const void* weight;
  uint8_t* codes;
  int64_t codes_row;
  float* scale;
  int n_rows, n_cols;
  float eps;
  int32_t* status;
  int n_sms;
};
template <typename T>
int launch_norm_quant(const NormQuantArgs& a, cudaStream_t s);

struct RowsQuantArgs {
  RowsArg x, gate;
  uint8_t* codes;
  int64_t codes_row;
  float* scale;
  int n_rows, n_cols;
  int32_t* status;
  int n_sms;
};
template <typename T>
int launch_rows_quant(const RowsQuantArgs& a, cudaStream_t s);
template <typename T>
int launch_weight_quant(const RowsQuantArgs& a, cudaStream_t s);

struct BlockMatmulArgs {
  const uint8_t *a, *w;
  int64_t a_row, w_row;                            // bytes, multiples of 16
  const float *a_scale, *w_scale;
  void* out;
  int64_t out_row;                                 // elements
  int m, n, k;
  bool f32;                                        // type of out
  int32_t* status;
  int n_sms;
};
int launch_block_matmul(const BlockMatmulArgs& a, cudaStream_t s);
int launch_block_matmul_pair(const BlockMatmulArgs& a, cudaStream_t s);          // many rows

// ---- eight elements of a row, as they are stored ----------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ Unit<T> load8(const void* base, int64_t at) {
  return load_unit(static_cast<const T*>(base) + at, false, 0);
}
template <typename T>
__device__ __forceinline__ Unit<T> no_unit() {
  return Unit<T>{};
}

// ---- a block's scale and codes ----------------------------------------------------------------------------------------
// A scale is the largest finite magnitude / 448, 2^-60 at least: not a power of two as in the cache, whose scales grow while their
// codes stay.  The largest element takes the largest code, so a block uses e4m3's whole range whatever its magnitude.  The quotient by a
// constant is its product with the reciprocal and one correction, rounded as a division is; the factor that codes are made with is within a
// unit of the last place of 1 / scale.  (All sixteen lanes of a block do this: a division each cost a third of what SwiGLU's rows took.)
__device__ __forceinline__ float block_scale(float amax) {
  constexpr float k = 1.f / 448.f;
  const float q = amax * k;
  return fmaxf(fmaf(fmaf(-448.f, q, amax), k, q), 0x1p-60f);
}
__device__ __forceinline__ float scale_inverse(float scale) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(scale));
  return fmaf(fmaf(-scale, r, 1.f), r, r);
}
// the largest magnitude of eight, NaN if one of them is
__device__ __forceinline__ float amax8(const float (&y)[8]) {
  auto three = [](float a, float b, float c) {
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
  };
  return three(three(y[0], y[1], y[2]), three(y[3], y[4], y[5]), three(y[6], y[7], y[7]));
}
__device__ __forceinline__ bool odd(float m) { return !(m <= 3.402823466e38f); }       // of an amax8: there is an infinity or a NaN
// Neither counts for the scale; an infinity becomes the largest code (the conversion saturates), a NaN 0.
__device__ __forceinline__ float amax8_finite(float (&y)[8]) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float a = fabsf(y[e]);
    m = fmaxf(m, a <= 3.402823466e38f ? a : 0.f);
    y[e] = y[e] != y[e] ? 0.f : y[e];
  }
  return m;
}
__device__ __forceinline__ uint2 codes8(const float (&y)[8], float inv) {
  return make_uint2(to_e4m3x4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv), to_e4m3x4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv));
}
// the largest of the sixteen lanes that have a block's 128 columns
__device__ __forceinline__ float half_warp_max(float m) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  return m;
}

}  // namespace vvs
