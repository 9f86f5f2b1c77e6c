// Entry points of the 8-bit key / value cache and of the rotation with several axes: checks of what the host can see, then one launch.
#include <cmath>

#include "quant_cache.cuh"

namespace vvs {
namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// rows of heads of element size `es`; strides of dimensions of size one are not looked at
int check_heads(const vvs_heads* h, int n_seqs, int n_rows, int n_heads, int es, HeadRows* out) {
  if (!h || !h->data) return VVS_ERR_INVALID_ARG;
  const int64_t unit = 16 / es;
  if (!aligned16(h->data)) return VVS_ERR_ALIGN;
  if ((n_seqs > 1 && h->seq % unit) || (n_rows > 1 && h->row % unit) || (n_heads > 1 && h->head % unit)) return VVS_ERR_ALIGN;
  *out = HeadRows{h->data, n_seqs > 1 ? h->seq : 0, n_rows > 1 ? h->row : 0, n_heads > 1 ? h->head : 0};
  return VVS_OK;
}

int check_rope(const vvs_rope_axes* r, int head_dim, RopeAxes* out) {
  if (!r || !r->inv_freq || !r->axis || !r->pos) return VVS_ERR_INVALID_ARG;
  if (r->halves != 0 && r->halves != 1) return VVS_ERR_INVALID_ARG;
  if (r->n_axes < 1 || r->n_pairs < 1 || r->n_pairs > head_dim / 2 || (r->halves && r->n_pairs % 4)) return VVS_ERR_SHAPE;
  *out = RopeAxes{r->inv_freq, r->axis, r->pos, r->n_axes, r->n_pairs, r->halves};
  return VVS_OK;
}

int check_cache(const vvs_qcache* c, QCache* out) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return VVS_ERR_INVALID_ARG;
  if (c->n_seqs < 1 || c->n_seqs > 65535 || c->n_heads < 1 || (c->head_dim != 64 && c->head_dim != 128)) return VVS_ERR_SHAPE;
  int log2 = 4;
  while (log2 < 7 && (1 << log2) != c->block) ++log2;
  if ((1 << log2) != c->block || c->cap < c->block || c->cap % c->block || c->cap > (1 << 30)) return VVS_ERR_SHAPE;
  if (!aligned16(c->k) || !aligned16(c->v)) return VVS_ERR_ALIGN;
  *out = QCache{static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_scale, c->v_scale, c->mass, c->age,
                c->n_seqs, c->n_heads, c->head_dim, c->cap, log2};
  return VVS_OK;
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

int vvs_element_bytes(const vvs_ctx* ctx) { return !ctx ? VVS_ERR_INVALID_ARG : is_f32(ctx) ? 4 : 2; }

int vvs_rotate_axes(vvs_ctx* ctx, const vvs_rope_axes* rope, int32_t n_seqs, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads,
                    int32_t head_dim, const vvs_heads* q, const vvs_heads* q_out, const vvs_heads* k, const vvs_heads* k_out,
                    void* stream) {
  if (!ctx || (k == nullptr) != (k_out == nullptr)) return VVS_ERR_INVALID_ARG;
  if (n_seqs < 1 || n_rows < 1 || n_heads < 1 || n_kv_heads < 0 || head_dim < 8 || head_dim > 256 || head_dim % 8) return VVS_ERR_SHAPE;
  if (!k) n_kv_heads = 0;
  if (k && n_kv_heads < 1) return VVS_ERR_SHAPE;
  if (n_heads + (int64_t)n_kv_heads > 65535 || (int64_t)n_seqs * n_rows > 0x7fffffff) return VVS_ERR_SHAPE;
  RotateArgs a{};
  const int es = is_f32(ctx) ? 4 : 2;
  VVS_TRY(check_rope(rope, head_dim, &a.rope));
  VVS_TRY(check_heads(q, n_seqs, n_rows, n_heads, es, &a.q));
  VVS_TRY(check_heads(q_out, n_seqs, n_rows, n_heads, es, &a.q_out));
  if (k) {
    VVS_TRY(check_heads(k, n_seqs, n_rows, n_kv_heads, es, &a.k));
    VVS_TRY(check_heads(k_out, n_seqs, n_rows, n_kv_heads, es, &a.k_out));
  }
  a.n_seqs = n_seqs; a.n_rows = n_rows; a.n_heads = n_heads; a.n_kv_heads = n_kv_heads; a.hd = head_dim;
  a.status = ctx->ws.status; a.n_sms = ctx->n_sms;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return is_f32(ctx) ? launch_rotate_axes<float>(a, s) : launch_rotate_axes<__nv_bfloat16>(a, s);
}

int vvs_quant_cache_append(vvs_ctx* ctx, const vvs_qcache* qc, const vvs_heads* k, const vvs_heads* v, const int32_t* cache_len,
                           int32_t n_rows, const int32_t* row_count, const int32_t* row_index, const int32_t* next_age,
                           const vvs_rope_axes* rope, int32_t n_heads, const vvs_heads* q, const vvs_heads* q_out, void* stream) {
  if (!ctx || !cache_len || (q == nullptr) != (q_out == nullptr)) return VVS_ERR_INVALID_ARG;
  if (q && (!rope || row_index)) return VVS_ERR_INVALID_ARG;
  QAppendArgs a{};
  VVS_TRY(check_cache(qc, &a.c));
  if (n_rows < 1 || n_rows > (1 << 24) || (q && n_heads < 1)) return VVS_ERR_SHAPE;
  if (!q) n_heads = 0;
  if (2 * (int64_t)qc->n_heads + n_heads > 65535 || (q && (int64_t)qc->n_seqs * n_rows > 0x7fffffff)) return VVS_ERR_SHAPE;
  const int es = is_f32(ctx) ? 4 : 2;
  VVS_TRY(check_heads(k, qc->n_seqs, n_rows, qc->n_heads, es, &a.k));
  VVS_TRY(check_heads(v, qc->n_seqs, n_rows, qc->n_heads, es, &a.v));
  if (rope) VVS_TRY(check_rope(rope, qc->head_dim, &a.rope));
  if (q) {
    VVS_TRY(check_heads(q, qc->n_seqs, n_rows, n_heads, es, &a.q));
    VVS_TRY(check_heads(q_out, qc->n_seqs, n_rows, n_heads, es, &a.q_out));
  }
  a.cache_len = cache_len; a.row_count = row_count; a.row_index = row_index; a.next_age = next_age;
  a.n_rows = n_rows; a.n_heads = n_heads; a.status = ctx->ws.status; a.n_sms = ctx->n_sms;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return is_f32(ctx) ? launch_quant_append<float>(a, s) : launch_quant_append<__nv_bfloat16>(a, s);
}

int vvs_quant_cache_attend(vvs_ctx* ctx, const vvs_qcache* qc, const vvs_heads* q, const vvs_heads* out, const int32_t* cache_len,
                           int32_t n_rows, int32_t n_heads, const int32_t* row_count, const int32_t* first_slot,
                           const uint32_t* visible, float* lse, float scale, int32_t mass_rows, float mass_decay, int32_t max_len,
                           void* stream) {
  if (!ctx || !cache_len) return VVS_ERR_INVALID_ARG;
  QAttendArgs a{};
  VVS_TRY(check_cache(qc, &a.c));
  if (!std::isfinite(scale) || !std::isfinite(mass_decay) || mass_decay < 0.f || (mass_rows > 0 && !qc->mass)) return VVS_ERR_INVALID_ARG;
  if (n_rows < 1 || n_heads < 1 || n_heads % qc->n_heads || (visible && n_rows > 32) || mass_rows < 0 || max_len < 0) return VVS_ERR_SHAPE;
  // one row of the grid for each cached head and tile: of 16 rows where there are no more, else of 32 at least (a tile that is not full: with more
  // than 16 rows a head, at most 61680 heads are left by the second condition)
  if (qc->n_heads > 65535 || (int64_t)n_rows * n_heads > (int64_t)65535 * 16) return VVS_ERR_SHAPE;
  const int es = is_f32(ctx) ? 4 : 2;
  VVS_TRY(check_heads(q, qc->n_seqs, n_rows, n_heads, es, &a.q));
  VVS_TRY(check_heads(out, qc->n_seqs, n_rows, n_heads, es, &a.out));
  a.cache_len = cache_len; a.row_count = row_count; a.first_slot = first_slot; a.visible = visible; a.lse = lse;
  a.scale = scale > 0.f ? scale : 1.f / std::sqrt((float)qc->head_dim);
  a.n_rows = n_rows; a.n_heads = n_heads; a.mass_rows = mass_rows; a.mass_decay = mass_decay; a.max_len = max_len;
  a.status = ctx->ws.status; a.n_sms = ctx->n_sms;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return is_f32(ctx) ? launch_quant_attend<float>(a, s) : launch_quant_attend<__nv_bfloat16>(a, s);
}

int vvs_quant_cache_evict(vvs_ctx* ctx, const vvs_qcache* qc, const int32_t* cache_len, int32_t keep, int32_t n_sink, int32_t n_recent,
                          const int32_t* next_age, float* mass_out, int32_t* age_out, int32_t* new_len, int32_t* kept, void* stream) {
  if (!ctx || !cache_len || !mass_out || !new_len || !kept) return VVS_ERR_INVALID_ARG;
  QEvictArgs a{};
  VVS_TRY(check_cache(qc, &a.c));
  if (!qc->mass || mass_out == qc->mass || (age_out && age_out == qc->age) || new_len == cache_len) return VVS_ERR_INVALID_ARG;
  if (keep < 1 || keep > qc->cap || n_sink < 0 || n_recent < 0 || (int64_t)n_sink + n_recent > keep || qc->n_heads > 65535) return VVS_ERR_SHAPE;
  a.cache_len = cache_len; a.next_age = next_age; a.keep = keep; a.n_sink = n_sink; a.n_recent = n_recent;
  a.mass_out = mass_out; a.age_out = age_out; a.new_len = new_len; a.kept = kept;
  a.status = ctx->ws.status; a.n_sms = ctx->n_sms;
  return launch_quant_evict(a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
