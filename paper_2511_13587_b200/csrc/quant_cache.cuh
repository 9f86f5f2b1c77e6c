// The 8-bit key / value cache (e4m3 codes, one float32 scale for each block of slots and head) and rotary positions with several
// axes: parameters of the kernels, and what several of them do with a value.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include <map>
#include <mutex>

#include "vvs_internal.cuh"

namespace vvs {

// rows of heads as the kernels read them (strides in elements)
struct HeadRows {
  void* data;
  int64_t seq, row, head;
};

struct RopeAxes {
  const float* inv_freq;
  const int32_t* axis;
  const int32_t* pos;    // [n_axes][n_seqs][n_rows]
  int n_axes, n_pairs, halves;
};

struct QCache {
  uint8_t *k, *v;
  float *k_scale, *v_scale, *mass;
  int32_t* age;
  int n_seqs, n_heads, hd, cap, block_log2;
};

struct RotateArgs {
  RopeAxes rope;
  HeadRows q, q_out, k, k_out;
  int n_seqs, n_rows, n_heads, n_kv_heads, hd;
  int32_t* status;
  int n_sms;
};
template <typename T>
int launch_rotate_axes(const RotateArgs& a, cudaStream_t s);

struct QAppendArgs {
  QCache c;
  HeadRows k, v, q, q_out;
  RopeAxes rope;               // inv_freq null: nothing is turned
  const int32_t *cache_len, *row_count, *row_index, *next_age;
  int n_rows, n_heads;         // n_heads 0: no q
  int32_t* status;
  int n_sms;
};
template <typename T>
int launch_quant_append(const QAppendArgs& a, cudaStream_t s);

struct QAttendArgs {
  QCache c;
  HeadRows q, out;
  const int32_t *cache_len, *row_count, *first_slot;
  const uint32_t* visible;
  float* lse;
  float scale, mass_decay;
  int n_rows, n_heads, mass_rows, max_len;
  int32_t* status;
  int n_sms;
};
template <typename T>
int launch_quant_attend(const QAttendArgs& a, cudaStream_t s);
int launch_quant_attend_rows(const QAttendArgs& a, cudaStream_t s);        // bf16, many rows, 128 summed ones at most

struct QEvictArgs {
  QCache c;
  const int32_t *cache_len, *next_age;
  int keep, n_sink, n_recent;
  float* mass_out;
  int32_t *age_out, *new_len, *kept;
  int32_t* status;
  int n_sms;
};
int launch_quant_evict(const QEvictArgs& a, cudaStream_t s);

// Clusters of 1 .. 16 CTAs of a kernel that the device holds at once, by their CTAs; null: an error.  A cluster's CTAs lie in one group
// of SMs: of CTAs that fill an SM, the device may hold 33 clusters of four, 15 of eight, 7 of sixteen.
constexpr int kMaxCluster = 16;
inline const int* resident_clusters(const void* kernel, int threads, int dynamic_smem) try {
  struct Counts { int there[kMaxCluster + 1]; };
  static std::mutex mu;
  static std::map<std::pair<int, const void*>, Counts> known;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return nullptr;
  std::lock_guard<std::mutex> lock(mu);
  const auto key = std::make_pair(dev, kernel);
  const auto it = known.find(key);
  if (it != known.end()) return it->second.there;
  Counts got{};
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return nullptr;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = dynamic_smem;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  for (int c = 1; c <= kMaxCluster; ++c) {
    attr[0].val.clusterDim.x = c;
    cfg.gridDim = dim3(c);
    if (cudaOccupancyMaxActiveClusters(&got.there[c], kernel, &cfg) != cudaSuccess) return nullptr;
  }
  return known.emplace(key, got).first->second.there;
} catch (...) {                                // no memory for the table, no lock
  return nullptr;
}

// ---- four values of a row, 8 bytes of bf16 or 16 of float32 -----------------------------------------------------------
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float* x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
}
__device__ __forceinline__ void store4(float* p, const float* x) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }

// ---- rotation ---------------------------------------------------------------------------------------------------------
// A head is worked on in units of eight elements.  Neighbouring pairs: unit u is elements 8u .. 8u + 7, pairs 4u .. 4u + 3.
// Halves: units below n_pairs / 4 are elements 4u .. 4u + 3 and n_pairs + 4u .. n_pairs + 4u + 3, pairs 4u .. 4u + 3; those behind
// are the elements that stay as they are, 8u .. 8u + 7 (n_pairs is a multiple of four there).
__device__ __forceinline__ bool unit_split(const RopeAxes& r, int u) { return r.halves && 4 * u < r.n_pairs; }

// A pair's positions [n_seqs][n_rows] (null: the pair stays as it is, being behind the last or of an unknown axis) and frequency.  Its angle is
// the float32 product of the two.
struct PairAxis {
  const int32_t* pos;
  float freq;
};
__device__ __forceinline__ PairAxis pair_axis(const RopeAxes& r, int pair, int n_seqs, int n_rows, int32_t* status) {
  if (pair >= r.n_pairs) return {nullptr, 0.f};
  const int ax = r.axis[pair];
  const float f = r.inv_freq[pair];
  if (ax < 0 || ax >= r.n_axes) {
    atomicOr(status, VVS_DEV_BAD_ARG);
    return {nullptr, 0.f};
  }
  return {r.pos + (size_t)ax * n_seqs * n_rows, f};
}

// products and sum rounded one by one: what a rotation gives does not depend on the kernel that it is part of
__device__ __forceinline__ void turn(float& x0, float& x1, float c, float s) {
  const float a = __fsub_rn(__fmul_rn(x0, c), __fmul_rn(x1, s));
  x1 = __fadd_rn(__fmul_rn(x1, c), __fmul_rn(x0, s));
  x0 = a;
}
// x: a unit's elements as unit_split orders them
__device__ __forceinline__ void turn_unit(float (&x)[8], bool split, const float* c, const float* s) {
  if (split) {
#pragma unroll
    for (int i = 0; i < 4; ++i) turn(x[i], x[4 + i], c[i], s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) turn(x[2 * i], x[2 * i + 1], c[i], s[i]);
  }
}
// In the place of a cosine: the pair stays as it is.  It is left alone, not turned by an angle of 0: next to an infinity,
// x * 1 + inf * 0 would be a NaN.  A unit of which only some pairs are turned (the last pair lies in it, or one of an unknown axis) has a
// path of its own: selections in the loops over whole units cost an append of prompts 83 us in the place of 71.5.
constexpr float kStays = 2.f;
// Which of a unit's four pairs are turned: bit i is pair 4u + i.
__device__ __forceinline__ uint32_t pairs_of(const float (&c)[4]) {
  uint32_t pairs = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) pairs |= c[j] != kStays ? 1u << j : 0u;
  return pairs;
}
constexpr uint32_t kAllPairs = 15u;
// those pairs alone
__device__ __forceinline__ void turn_some(float (&x)[8], bool split, const float* c, const float* s, uint32_t pairs) {
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = x[e];
  turn_unit(y, split, c, s);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (pairs >> (split ? e % 4 : e / 2) & 1u) x[e] = y[e];
}
// as they are stored
template <typename T>
struct Unit;
template <>
struct Unit<__nv_bfloat16> {
  uint2 a, b;
};
template <>
struct Unit<float> {
  float4 a, b;
};
// where a unit begins in its row; its second half lies n_pairs behind that, or next to the first
__device__ __forceinline__ int unit_at(int u, bool split) { return (split ? 4 : 8) * u; }
__device__ __forceinline__ Unit<__nv_bfloat16> load_unit(const __nv_bfloat16* p, bool split, int n_pairs) {
  if (split) return {*reinterpret_cast<const uint2*>(p), *reinterpret_cast<const uint2*>(p + n_pairs)};
  const uint4 t = *reinterpret_cast<const uint4*>(p);
  return {make_uint2(t.x, t.y), make_uint2(t.z, t.w)};
}
__device__ __forceinline__ Unit<float> load_unit(const float* p, bool split, int n_pairs) {
  return {*reinterpret_cast<const float4*>(p), *reinterpret_cast<const float4*>(p + (split ? n_pairs : 4))};
}
__device__ __forceinline__ void widen_unit(const Unit<__nv_bfloat16>& r, float (&x)[8]) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.b.x, r.b.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen_unit(const Unit<float>& r, float (&x)[8]) {
  x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w; x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
}
__device__ __forceinline__ Unit<__nv_bfloat16> narrow_unit(const float (&x)[8], const Unit<__nv_bfloat16>&) {
  return {make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])), make_uint2(pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]))};
}
__device__ __forceinline__ Unit<float> narrow_unit(const float (&x)[8], const Unit<float>&) {
  return {make_float4(x[0], x[1], x[2], x[3]), make_float4(x[4], x[5], x[6], x[7])};
}
// what is not turned as it came (rounding to bf16 would give another NaN for a NaN)
__device__ __forceinline__ void put_back(Unit<__nv_bfloat16>& out, const Unit<__nv_bfloat16>& raw, bool split, uint32_t pairs) {
  uint32_t* o[4] = {&out.a.x, &out.a.y, &out.b.x, &out.b.y};
  const uint32_t r[4] = {raw.a.x, raw.a.y, raw.b.x, raw.b.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int first = split ? 2 * i % 4 : i, second = split ? 2 * i % 4 + 1 : i;      // pairs of the word's two elements
    const uint32_t mask = (pairs >> first & 1u ? 0xffffu : 0u) | (pairs >> second & 1u ? 0xffff0000u : 0u);
    *o[i] = (*o[i] & mask) | (r[i] & ~mask);
  }
}
__device__ __forceinline__ void put_back(Unit<float>& out, const Unit<float>& raw, bool split, uint32_t pairs) {
  float* o[8] = {&out.a.x, &out.a.y, &out.a.z, &out.a.w, &out.b.x, &out.b.y, &out.b.z, &out.b.w};
  const float r[8] = {raw.a.x, raw.a.y, raw.a.z, raw.a.w, raw.b.x, raw.b.y, raw.b.z, raw.b.w};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (!(pairs >> (split ? e % 4 : e / 2) & 1u)) *o[e] = r[e];
}
template <typename T>
__device__ __forceinline__ Unit<T> turned_unit(const Unit<T>& raw, bool split, const float* c, const float* s) {
  float x[8];
  widen_unit(raw, x);
  turn_unit(x, split, c, s);
  return narrow_unit(x, raw);
}
template <typename T>
__device__ __forceinline__ Unit<T> turned_some(const Unit<T>& raw, bool split, const float* c, const float* s, uint32_t pairs) {
  Unit<T> out = turned_unit(raw, split, c, s);
  put_back(out, raw, split, pairs);
  return out;
}
__device__ __forceinline__ void store_unit(__nv_bfloat16* p, bool split, int n_pairs, const Unit<__nv_bfloat16>& x) {
  if (split) {
    *reinterpret_cast<uint2*>(p) = x.a;
    *reinterpret_cast<uint2*>(p + n_pairs) = x.b;
  } else {
    *reinterpret_cast<uint4*>(p) = make_uint4(x.a.x, x.a.y, x.b.x, x.b.y);
  }
}
__device__ __forceinline__ void store_unit(float* p, bool split, int n_pairs, const Unit<float>& x) {
  *reinterpret_cast<float4*>(p) = x.a;
  *reinterpret_cast<float4*>(p + (split ? n_pairs : 4)) = x.b;
}

// ---- e4m3 -------------------------------------------------------------------------------------------------------------
// the smallest power of two, 2^-60 at least, by which amax is at most 448 = 1.75 * 2^8
__device__ __forceinline__ float scale_of(float amax) {
  const uint32_t b = __float_as_uint(amax);
  int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);      // biased exponent of the scale
  e = e < 67 ? 67 : e;                                                      // (a subnormal amax has biased exponent 0)
  return __uint_as_float((uint32_t)e << 23);
}
// four values to four codes, to nearest, ties to even, values beyond 448 to 448
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}
// two codes (of the low half of w) to two halves
__device__ __forceinline__ uint32_t from_e4m3x2(uint32_t w) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)w));
  return r;
}
__device__ __forceinline__ float2 halves_to_float2(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }
// four codes times a factor, to codes again
__device__ __forceinline__ uint32_t rescale_e4m3x4(uint32_t w, float f) {
  const float2 lo = halves_to_float2(from_e4m3x2(w)), hi = halves_to_float2(from_e4m3x2(w >> 16));
  return to_e4m3x4(lo.x * f, lo.y * f, hi.x * f, hi.y * f);
}

// ---- weights ----------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Weights carry their value's scale, a row's sum does not: sum_j w_j / V_b.  Where values' scales lie up to 2^200 apart (a block of zeros has
// 2^-60, the largest is 2^120), weights of the smaller ones vanish at the row's reference although their keys may have most of the row's softmax.
// Nothing is lost from the outputs then, next to values so much larger, but it is from the sum.  So where a scale was met that is
// not an ordinary one, weights that vanish go into the sum from 2^100 times themselves; and sums come to another reference in two steps.
// Ordinary scales lie within 2^80: a key's weight at its row's reference is 2^(7 - 80) times its share of the softmax at least.
__device__ __forceinline__ bool odd_scale(float v) { return !(v >= 0x1p-62f && v <= 0x1p18f); }
constexpr float kGone = -126.f, kGoneUp = 100.f, kGoneDown = 0x1p-100f;
// 2^(a + 100) if 2^a vanishes, else nothing
__device__ __forceinline__ float gone_weight(float a) { return a < kGone ? ex2(a + kGoneUp) : 0.f; }
// x 2^d, y + x 2^d
__device__ __forceinline__ float times_ex2(float x, float d) { return x * ex2(fmaxf(d, -100.f)) * ex2(fminf(d + 100.f, 0.f)); }
__device__ __forceinline__ float add_times_ex2(float y, float x, float d) { return fmaf(x * ex2(fmaxf(d, -100.f)), ex2(fminf(d + 100.f, 0.f)), y); }

}  // namespace vvs
