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
// constant is its product with the reciprocal and one correction by the residual (Markstein, 1990), rounded as a division is.
__device__ __forceinline__ float block_scale(float amax) {
  constexpr float k = 1.f / 448.f;
  const float q = amax * k;
  return fmaxf(fmaf(fmaf(-448.f, q, amax), k, q), 0x1p-60f);
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
// Neither counts for the scale; an infinity becomes the largest code (hold8), a NaN 0.
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
// infinities to where the largest code is (codes8 wants residuals that are numbers)
__device__ __forceinline__ void hold8(float (&y)[8], float scale) {
  const float most = fminf(448.f * scale, 3.402823466e38f);
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = fminf(fmaxf(y[e], -most), most);
}
// -1 / scale: an approximation within a unit of the last place and a Newton-Raphson step, which rounds right but where all bits of the scale's
// mantissa are ones (and there is one too low) and, of an approximation that is a unit too high, at 31 mantissas more.  (All sixteen lanes of a block do
// this; __frcp_rn took 22016 x 4096 weights from 44 to 50 us, float32 norms of 12000 columns from 30 to 37.)
__device__ __forceinline__ float minus_inverse(float scale) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(scale));
  r = fmaf(fmaf(-scale, r, 1.f), r, r);
  const uint32_t bits = __float_as_uint(r) | 0x80000000u;
  return __uint_as_float((__float_as_uint(scale) & 0x7fffffu) == 0x7fffffu ? bits + 1 : bits);
}
// Two quotients y / scale as a division rounds them, negative: the product with the reciprocal, corrected by its residual, which a
// multiply-add has exactly (Markstein, 1990).  Without the correction an element on the border of two codes, as bf16's elements often are,
// would take one or the other by the product's own rounding.  (At the 31 mantissas a quotient may be off by its last bit, at no border: all of
// them tried.)  Negative, for then zeros keep their signs through the correction.
__device__ __forceinline__ void quotients(float& a, float& b, float scale, float minus_inv) {
  asm("{\n\t.reg .b64 y, n, s, q, r;\n\t"
      "mov.b64 y, {%0, %1};\n\tmov.b64 n, {%3, %3};\n\tmov.b64 s, {%2, %2};\n\t"
      "mul.rn.f32x2 q, y, n;\n\tfma.rn.f32x2 r, s, q, y;\n\tfma.rn.f32x2 q, r, n, q;\n\t"
      "mov.b64 {%0, %1}, q;\n\t}"
      : "+f"(a), "+f"(b) : "f"(scale), "f"(minus_inv));
}
// The codes nearest to the elements over their block's scale, ties to the even one.
__device__ __forceinline__ uint2 codes8(const float (&y)[8], float scale, float minus_inv) {
  float q[8];
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    q[e] = y[e], q[e + 1] = y[e + 1];
    quotients(q[e], q[e + 1], scale, minus_inv);
  }
  return make_uint2(to_e4m3x4(q[0], q[1], q[2], q[3]) ^ 0x80808080u, to_e4m3x4(q[4], q[5], q[6], q[7]) ^ 0x80808080u);
}
// the largest of the sixteen lanes that have a block's 128 columns
__device__ __forceinline__ float half_warp_max(float m) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  return m;
}

}  // namespace vvs
