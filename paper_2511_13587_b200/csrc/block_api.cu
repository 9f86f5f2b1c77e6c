// Entry points of rows and weights in 8 bits and of their product: checks of what the host can see, then one launch.
#include <cmath>

#include "block_quant.cuh"

namespace vvs {
namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// rows of elements of size `es`, of which `n_written` (0: they are read) are written; the stride of a single row is not looked at
int check_rows(const vvs_rows* r, int n_rows, int n_written, int es, RowsArg* out) {
  if (!r || !r->data) return VVS_ERR_INVALID_ARG;
  if (n_rows > 1 && n_written && r->row < n_written) return VVS_ERR_SHAPE;
  if (!aligned16(r->data) || (n_rows > 1 && r->row % (16 / es))) return VVS_ERR_ALIGN;
  *out = RowsArg{r->data, n_rows > 1 ? r->row : 0};
  return VVS_OK;
}

int check_qrows(const vvs_qrows* q, int n_rows, int n_cols) {
  if (!q || !q->codes || !q->scale) return VVS_ERR_INVALID_ARG;
  if (n_rows > 1 && (q->row < n_cols || q->row >= (int64_t)1 << 40)) return VVS_ERR_SHAPE;
  if (!aligned16(q->codes) || (reinterpret_cast<uintptr_t>(q->scale) & 3) || (n_rows > 1 && q->row % 16)) return VVS_ERR_ALIGN;
  return VVS_OK;
}

int check_qweight(const vvs_qweight* w) {
  if (!w || !w->codes || !w->scale) return VVS_ERR_INVALID_ARG;
  if (w->n_rows < 1 || w->n_cols < 16 || w->n_cols % 16 || w->n_cols > kMaxCols || w->n_rows > 65535 * kQBlock) return VVS_ERR_SHAPE;
  if (w->n_rows > 1 && (w->row < w->n_cols || w->row >= (int64_t)1 << 40)) return VVS_ERR_SHAPE;
  if (!aligned16(w->codes) || (reinterpret_cast<uintptr_t>(w->scale) & 3) || (w->n_rows > 1 && w->row % 16)) return VVS_ERR_ALIGN;
  return VVS_OK;
}

bool bad_size(int n_rows, int n_cols) {
  return n_rows < 1 || n_cols < 16 || n_cols % 16 || n_cols > kMaxCols || (int64_t)n_rows * qblocks(n_cols) > kMaxBlocks;
}
bool is_f32(const vvs_ctx* ctx) { return ctx->desc.dtype == VVS_DTYPE_FP32; }

}  // namespace
}  // namespace vvs

using namespace vvs;

#define VVS_TRY(expr)               \
  do {                              \
    const int rc__ = (expr);        \
    if (rc__ != VVS_OK) return rc__; \
  } while (0)

extern "C" {

int vvs_norm_quant(vvs_ctx* ctx, int32_t n_rows, int32_t n_cols, const vvs_rows* x, const vvs_rows* residual, const void* weight, float eps,
                   const vvs_rows* sum_out, const vvs_rows* norm_out, const vvs_qrows* out, void* stream) {
  if (!ctx || !weight || !std::isfinite(eps) || eps < 0.f) return VVS_ERR_INVALID_ARG;
  if (bad_size(n_rows, n_cols) || n_cols > kNormMaxCols) return VVS_ERR_SHAPE;
  NormQuantArgs a{};
  const int es = is_f32(ctx) ? 4 : 2;
  VVS_TRY(check_rows(x, n_rows, 0, es, &a.x));
  if (residual) VVS_TRY(check_rows(residual, n_rows, 0, es, &a.residual));
  if (sum_out) VVS_TRY(check_rows(sum_out, n_rows, n_cols, es, &a.sum_out));
  if (norm_out) VVS_TRY(check_rows(norm_out, n_rows, n_cols, es, &a.norm_out));
  VVS_TRY(check_qrows(out, n_rows, n_cols));
  if (!aligned16(weight)) return VVS_ERR_ALIGN;
  a.weight = weight; a.codes = static_cast<uint8_t*>(out->codes); a.codes_row = n_rows > 1 ? out->row : 0; a.scale = out->scale;
  a.n_rows = n_rows; a.n_cols = n_cols; a.eps = eps; a.status = ctx->ws.status; a.n_sms = ctx->n_sms;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return is_f32(ctx) ? launch_norm_quant<float>(a, s) : launch_norm_quant<__nv_bfloat16>(a, s);
}

int vvs_rows_quant(vvs_ctx* ctx, int32_t n_rows, int32_t n_cols, const vvs_rows* x, const vvs_rows* gate, const vvs_qrows* out, void* stream) {
  if (!ctx) return VVS_ERR_INVALID_ARG;
  if (bad_size(n_rows, n_cols)) return VVS_ERR_SHAPE;
  RowsQuantArgs a{};
  const int es = is_f32(ctx) ? 4 : 2;
  VVS_TRY(check_rows(x, n_rows, 0, es, &a.x));
  if (gate) VVS_TRY(check_rows(gate, n_rows, 0, es, &a.gate));
  VVS_TRY(check_qrows(out, n_rows, n_cols));
  a.codes = static_cast<uint8_t*>(out->codes); a.codes_row = n_rows > 1 ? out->row : 0; a.scale = out->scale;
  a.n_rows = n_rows; a.n_cols = n_cols; a.status = ctx->ws.status; a.n_sms = ctx->n_sms;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return is_f32(ctx) ? launch_rows_quant<float>(a, s) : launch_rows_quant<__nv_bfloat16>(a, s);
}

int vvs_weight_quant(vvs_ctx* ctx, const vvs_rows* w, const vvs_qweight* out, void* stream) {
  if (!ctx) return VVS_ERR_INVALID_ARG;
  VVS_TRY(check_qweight(out));
  RowsQuantArgs a{};
  VVS_TRY(check_rows(w, out->n_rows, 0, is_f32(ctx) ? 4 : 2, &a.x));
  a.codes = static_cast<uint8_t*>(out->codes); a.codes_row = out->n_rows > 1 ? out->row : 0; a.scale = out->scale;
  a.n_rows = out->n_rows; a.n_cols = out->n_cols; a.status = ctx->ws.status; a.n_sms = ctx->n_sms;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return is_f32(ctx) ? launch_weight_quant<float>(a, s) : launch_weight_quant<__nv_bfloat16>(a, s);
}

int vvs_block_matmul(vvs_ctx* ctx, int32_t n_rows, const vvs_qrows* a, const vvs_qweight* w, const vvs_rows* out, void* stream) {
  if (!ctx) return VVS_ERR_INVALID_ARG;
  VVS_TRY(check_qweight(w));
  if (bad_size(n_rows, w->n_cols)) return VVS_ERR_SHAPE;
  VVS_TRY(check_qrows(a, n_rows, w->n_cols));
  if (!out || !out->data) return VVS_ERR_INVALID_ARG;
  if (n_rows > 1 && out->row < w->n_rows) return VVS_ERR_SHAPE;
  if (!aligned16(out->data)) return VVS_ERR_ALIGN;
  BlockMatmulArgs g{};
  g.a = static_cast<const uint8_t*>(a->codes); g.w = static_cast<const uint8_t*>(w->codes);
  g.a_row = n_rows > 1 ? a->row : w->n_cols;         // (strides of tensor maps, which are looked at even where there is one row)
  g.w_row = w->n_rows > 1 ? w->row : w->n_cols;
  g.a_scale = a->scale; g.w_scale = w->scale;
  g.out = out->data; g.out_row = n_rows > 1 ? out->row : (w->n_rows + 15) / 16 * 16;
  g.m = n_rows; g.n = w->n_rows; g.k = w->n_cols; g.f32 = is_f32(ctx); g.status = ctx->ws.status; g.n_sms = ctx->n_sms;
  return launch_block_matmul(g, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
