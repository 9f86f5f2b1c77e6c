// What the two kernels of the 8-bit product share: e4m3 operands on tcgen05, their tensor maps, sums that take a block's scales.
#pragma once

#include "block_quant.cuh"
#include "tc_common.cuh"

namespace vvs {
namespace bmm {

using namespace tc;

constexpr int kTileBytes = 128 * kQBlock;          // 128 rows of one block of K

// [rows, cols] bytes, a box of `box_rows` rows of one block of K: a 128-byte swizzled tile
int make_tmap_e4m3(CUtensorMap* out, const void* base, int64_t rows, int64_t cols, int64_t row_bytes, uint32_t box_rows);

struct MatmulParams {
  const float *a_scale, *w_scale;
  void* out;
  int64_t out_row;
  int m, n, nkb;                                   // nkb: blocks of K
  int first;                                       // tile of weights that the clusters begin with whose CTAs share one
  int alone;                                       // clusters ahead of them whose CTAs have a tile each, from 0 to `first`
  int wide;                                        // four elements of out may be written together
  int32_t* status;
};

// Instruction descriptor, kind::f8f6f4: D = fp32 (bits 4-5 = 1), A = B = e4m3 (bits 7-9, 10-12 = 0), both K-major, N >> 3 in bits 17-22,
// M >> 4 in bits 24-28.
__device__ __forceinline__ uint32_t idesc_e4m3_f32(uint32_t m, uint32_t n) { return (1u << 4) | ((n >> 3) << 17) | ((m >> 4) << 24); }

// The four K steps (32 elements each) of a block: D = A B with both operands in 128-byte swizzled K-major tiles; the first overwrites D.
// Called by a converged warp, of which one lane issues.
template <int CG>
__device__ __forceinline__ void mma_e4m3_block(uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc) {
#define VVS_MMA_E4M3(cg)                                                                              \
  asm volatile(                                                                                       \
      "{\n\t.reg .pred e, p, q;\n\t.reg .b64 a, b;\n\t.reg .b32 x, y;\n\t"                            \
      "elect.sync _|e, 0xffffffff;\n\t"                                                               \
      "setp.ne.u32 p, %4, %4;\n\tsetp.eq.u32 q, %4, %4;\n\t"                                          \
      "mov.b64 a, {%1, %4};\n\tmov.b64 b, {%2, %4};\n\t"                                              \
      "@e tcgen05.mma.cta_group::" cg ".kind::f8f6f4 [%0], a, b, %3, p;\n\t"                          \
      "add.u32 x, %1, 2;\n\tadd.u32 y, %2, 2;\n\tmov.b64 a, {x, %4};\n\tmov.b64 b, {y, %4};\n\t"      \
      "@e tcgen05.mma.cta_group::" cg ".kind::f8f6f4 [%0], a, b, %3, q;\n\t"                          \
      "add.u32 x, %1, 4;\n\tadd.u32 y, %2, 4;\n\tmov.b64 a, {x, %4};\n\tmov.b64 b, {y, %4};\n\t"      \
      "@e tcgen05.mma.cta_group::" cg ".kind::f8f6f4 [%0], a, b, %3, q;\n\t"                          \
      "add.u32 x, %1, 6;\n\tadd.u32 y, %2, 6;\n\tmov.b64 a, {x, %4};\n\tmov.b64 b, {y, %4};\n\t"      \
      "@e tcgen05.mma.cta_group::" cg ".kind::f8f6f4 [%0], a, b, %3, q;\n\t}"                         \
      ::"r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(kDescHiSw128)                              \
      : "memory")
  if constexpr (CG == 1) VVS_MMA_E4M3("1");
  else VVS_MMA_E4M3("2");
#undef VVS_MMA_E4M3
}

__device__ __forceinline__ void tma_prefetch_2d(const CUtensorMap* m, int x, int y) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y) : "memory");
}

// Bounded wait of a warp, which goes on as one, in as few instructions as it takes where the phase is complete.
__device__ __forceinline__ bool warp_wait_lean(uint32_t bar, uint32_t parity, const volatile int* abort_flag) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .u32 n, a;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "@p bra VVS_DONE_%=;\n\t"
      "mov.u32 n, %4;\n"
      "VVS_AGAIN_%=:\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "@p bra VVS_DONE_%=;\n\t"
      "ld.volatile.shared.u32 a, [%3];\n\tsetp.ne.u32 p, a, 0;\n\t@p bra VVS_GONE_%=;\n\t"
      "sub.u32 n, n, 1;\n\tsetp.ne.u32 p, n, 0;\n\t@p bra VVS_AGAIN_%=;\n"
      "VVS_GONE_%=:\n\t"
      "setp.ne.u32 p, n, n;\n"
      "VVS_DONE_%=:\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity), "r"(smem_u32(const_cast<const int*>(abort_flag))), "n"(kSpinLimit) : "memory");
  return __all_sync(0xffffffffu, ok);
}

// N (8, 16 or 32) consecutive columns of the warp's 32 lanes are requested; tmem_wait before they are read
template <int N>
__device__ __forceinline__ void tmem_request(uint32_t taddr, float (&v)[N]) {
  static_assert(N == 8 || N == 16 || N == 32, "columns");
  if constexpr (N == 8) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "r"(taddr) : "memory");
  } else if constexpr (N == 16) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
                   "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]) : "r"(taddr) : "memory");
  } else {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]),
          "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]),
          "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(taddr) : "memory");
  }
}
// (the registers are named so that nothing reads them ahead of the wait)
template <int N>
__device__ __forceinline__ void tmem_wait(float (&v)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+f"(v[i]));
}

}  // namespace bmm
}  // namespace vvs
