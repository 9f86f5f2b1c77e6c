/* CPython entry points of the C ABI: argument marshalling of the calls a decoding loop makes per step.  A call through
 * ctypes costs 6-10 us of host time (two structures, ~15 attribute calls, the current-stream object); the small
 * calls of this library run 2-10 us on the GPU, so the host decided their time.  Here a call fills the C
 * structures straight from the keyword arguments. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "vvs.h"

static PyObject *g_error, *g_raw_stream, *g_get_device;   /* VvsError; torch's current raw stream and device */
static PyObject *s_data_ptr, *s_shape, *s_cuda_stream, *s_keep;

/* tensor (or integer address, or None) -> address; -1 with an exception set on failure */
static int to_ptr(PyObject* o, void** out) {
  if (o == Py_None) { *out = NULL; return 0; }
  if (PyLong_Check(o)) {
    *out = PyLong_AsVoidPtr(o);
    return PyErr_Occurred() ? -1 : 0;
  }
  PyObject* v = PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (!v) return -1;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return PyErr_Occurred() ? -1 : 0;
}
static int to_int(PyObject* o, int32_t* out) {
  PyObject* v = PyNumber_Long(o);
  if (!v) return -1;
  const long x = PyLong_AsLong(v);
  Py_DECREF(v);
  if (x == -1 && PyErr_Occurred()) return -1;
  *out = (int32_t)x;
  return 0;
}
static int to_float(PyObject* o, float* out) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) return -1;
  *out = (float)x;
  return 0;
}
/* the stream of a call: None = torch's current stream of the current device */
static int to_stream(PyObject* o, void** out) {
  PyObject* v;
  if (!o || o == Py_None) {
    PyObject* dev = PyObject_CallNoArgs(g_get_device);
    if (!dev) return -1;
    v = PyObject_CallOneArg(g_raw_stream, dev);
    Py_DECREF(dev);
  } else if (PyLong_Check(o)) {
    v = Py_NewRef(o);
  } else {
    v = PyObject_GetAttr(o, s_cuda_stream);
    if (!v && PyErr_ExceptionMatches(PyExc_AttributeError)) {
      PyErr_Clear();
      v = PyNumber_Long(o);
    }
  }
  if (!v) return -1;
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return PyErr_Occurred() ? -1 : 0;
}

/* One parameter of an entry point: where it goes and what it is. */
typedef struct {
  const char* name;
  char kind;          /* p tensor / address, i int32, f float, b truth value, c context, s stream, o object */
  char required;
  size_t off;         /* byte offset in the call's frame */
  PyObject* key;      /* interned name */
} Param;
#define MAX_PARAMS 40

static int put(const Param* q, PyObject* v, char* frame) {
  void* at = frame + q->off;
  switch (q->kind) {
    case 'p': return to_ptr(v, (void**)at);
    case 'i': return to_int(v, (int32_t*)at);
    case 'f': return to_float(v, (float*)at);
    case 'b': return to_int(v, (int32_t*)at);
    case 'c': *(void**)at = v == Py_None ? NULL : PyLong_AsVoidPtr(v); return PyErr_Occurred() ? -1 : 0;
    case 's': return to_stream(v, (void**)at);
    default: *(PyObject**)at = v; return 0;
  }
}

/* Fills `frame` from the call; positional arguments take the parameters in order (at most `n_pos` of them). */
static int parse(const char* fn, const Param* ps, int n, int n_pos, void* frame, PyObject* const* args, Py_ssize_t nargs,
                 PyObject* kwnames) {
  unsigned char seen[MAX_PARAMS] = {0};
  if (nargs > n_pos) {
    PyErr_Format(PyExc_TypeError, "%s() takes %d positional arguments but %zd were given", fn, n_pos, nargs);
    return -1;
  }
  for (Py_ssize_t i = 0; i < nargs; ++i) {
    if (put(&ps[i], args[i], frame) < 0) return -1;
    seen[i] = 1;
  }
  const Py_ssize_t nk = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
  int hint = (int)nargs;
  for (Py_ssize_t k = 0; k < nk; ++k) {
    PyObject* key = PyTuple_GET_ITEM(kwnames, k);
    int j = -1;
    for (int t = 0; t < n && j < 0; ++t) {           /* callers keep their order: start behind the previous match */
      const int c = hint + t < n ? hint + t : hint + t - n;
      if (ps[c].key == key) j = c;
    }
    for (int c = 0; j < 0 && c < n; ++c)
      if (PyUnicode_Compare(ps[c].key, key) == 0) j = c;
    if (j < 0) {
      PyErr_Format(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", fn, key);
      return -1;
    }
    if (seen[j]) {
      PyErr_Format(PyExc_TypeError, "%s() got multiple values for argument '%s'", fn, ps[j].name);
      return -1;
    }
    if (put(&ps[j], args[nargs + k], frame) < 0) return -1;
    seen[j] = 1;
    hint = j + 1 < n ? j + 1 : 0;
  }
  for (int i = 0; i < n; ++i) {
    if (seen[i]) continue;
    if (ps[i].required) {
      PyErr_Format(PyExc_TypeError, "%s() missing required argument: '%s'", fn, ps[i].name);
      return -1;
    }
    if (ps[i].kind == 's' && to_stream(NULL, (void**)((char*)frame + ps[i].off)) < 0) return -1;
  }
  return 0;
}

static PyObject* done(int status, const char* where) {
  if (status == VVS_OK) Py_RETURN_NONE;
  PyObject* e = PyObject_CallFunction(g_error, "is", status, where);
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  return NULL;
}
/* The library call runs without the interpreter lock (a first call captures a graph: milliseconds). */
#define CALL(name, expr)        \
  do {                          \
    int rc;                     \
    Py_BEGIN_ALLOW_THREADS      \
    rc = (expr);                \
    Py_END_ALLOW_THREADS        \
    return done(rc, name);      \
  } while (0)

/* ---- the decision-making calls: one frame for all of them ------------------------------------------------------ */
typedef struct {
  vvs_ctx* ctx;
  vvs_verify_args a;
  vvs_verify_out o;
  void* stream;
  void *hidden_in, *drafts, *target_probs, *nbr_row_ptr, *nbr_col, *status_bits;
  int32_t n_rows_per_seq, first_row, vocab, vocab_offset;
} Frame;
#define A(f) offsetof(Frame, a) + offsetof(vvs_verify_args, f)
#define O(f) offsetof(Frame, o) + offsetof(vvs_verify_out, f)
#define F(f) offsetof(Frame, f)

static void frame_init(Frame* f) {
  memset(f, 0, sizeof(*f));
  f->a.n_cfg = f->a.n_forced = f->a.nbr_k = 1;
  f->a.cfg_scale = f->a.temperature = 1.f;
  f->a.delta = Py_HUGE_VAL;
}

#define DECISION_PARAMS                                                                                              \
  {"draft_probs", 'p', 1, A(draft_probs)}, {"uniforms", 'p', 1, A(uniforms)}, {"accept_len", 'p', 1, O(accept_len)}, \
      {"next_token", 'p', 1, O(next_token)}, {"n_draft", 'p', 0, A(n_draft)}, {"mode", 'i', 0, A(mode)},             \
      {"nbr_k", 'i', 0, A(nbr_k)}, {"delta", 'f', 0, A(delta)}, {"accept_mask", 'p', 0, O(accept_mask)},             \
      {"margins", 'p', 0, O(margins)}, {"adjusted_residual", 'b', 0, A(adjusted_residual)}, {"stream", 's', 0, F(stream)}

static Param verify_params[] = {
    {"ctx", 'c', 1, F(ctx)}, {"n_images", 'i', 1, A(n_images)}, {"n_cfg", 'i', 1, A(n_cfg)}, {"n_forced", 'i', 1, A(n_forced)},
    {"n_draft_max", 'i', 1, A(n_draft_max)}, {"block", 'p', 1, A(block)}, {"kv_k", 'p', 1, A(kv_k)}, {"kv_v", 'p', 1, A(kv_v)},
    {"kv_rows", 'i', 1, A(kv_rows)}, {"cache_len", 'p', 1, A(cache_len)}, {"new_len", 'p', 1, O(new_len)},
    {"cache_len_host", 'p', 0, A(cache_len_host)}, {"cfg_scale", 'f', 0, A(cfg_scale)}, {"temperature", 'f', 0, A(temperature)},
    {"n_commit", 'p', 0, O(n_commit)}, {"target_probs", 'p', 0, O(target_probs)}, {"hidden", 'p', 0, O(hidden)},
    {"tree_parent", 'p', 0, A(tree_parent)}, {"accept_path", 'p', 0, O(accept_path)}, DECISION_PARAMS};
static Param epilogue_params[] = {
    {"ctx", 'c', 1, F(ctx)}, {"hidden_in", 'p', 1, F(hidden_in)}, {"n_rows_per_seq", 'i', 1, F(n_rows_per_seq)},
    {"first_row", 'i', 1, F(first_row)}, {"drafts", 'p', 1, F(drafts)}, {"n_images", 'i', 1, A(n_images)},
    {"n_cfg", 'i', 1, A(n_cfg)}, {"n_draft_max", 'i', 1, A(n_draft_max)}, {"cfg_scale", 'f', 0, A(cfg_scale)},
    {"temperature", 'f', 0, A(temperature)}, {"target_probs", 'p', 0, O(target_probs)}, DECISION_PARAMS};
static Param decide_params[] = {
    {"ctx", 'c', 1, F(ctx)}, {"target_probs", 'p', 1, F(target_probs)}, {"n_rows_per_seq", 'i', 1, F(n_rows_per_seq)},
    {"first_row", 'i', 1, F(first_row)}, {"drafts", 'p', 1, F(drafts)}, {"n_images", 'i', 1, A(n_images)},
    {"n_draft_max", 'i', 1, A(n_draft_max)}, {"tree_parent", 'p', 0, A(tree_parent)}, {"accept_path", 'p', 0, O(accept_path)},
    DECISION_PARAMS};
static Param noalloc_params[] = {
    {"target_probs", 'p', 1, F(target_probs)}, {"vocab", 'i', 1, F(vocab)}, {"vocab_offset", 'i', 1, F(vocab_offset)},
    {"n_rows_per_seq", 'i', 1, F(n_rows_per_seq)}, {"first_row", 'i', 1, F(first_row)}, {"drafts", 'p', 1, F(drafts)},
    {"n_images", 'i', 1, A(n_images)}, {"n_draft_max", 'i', 1, A(n_draft_max)}, {"nbr_row_ptr", 'p', 0, F(nbr_row_ptr)},
    {"nbr_col", 'p', 0, F(nbr_col)}, {"status_bits", 'p', 0, F(status_bits)}, {"tree_parent", 'p', 0, A(tree_parent)},
    {"accept_path", 'p', 0, O(accept_path)}, DECISION_PARAMS};
#define N(ps) (int)(sizeof(ps) / sizeof(ps[0]))
#define FAST PyObject *self, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames
#define PARSE(name, ps, n_pos) parse(name, ps, N(ps), n_pos, &f, args, nargs, kwnames)

static PyObject* py_verify(FAST) {
  (void)self;
  Frame f;
  frame_init(&f);
  if (PARSE("vvs_verify", verify_params, 1) < 0) return NULL;
  CALL("vvs_verify", vvs_verify(f.ctx, &f.a, &f.o, f.stream));
}
static PyObject* py_epilogue(FAST) {
  (void)self;
  Frame f;
  frame_init(&f);
  if (PARSE("vvs_epilogue", epilogue_params, 1) < 0) return NULL;
  CALL("vvs_epilogue", vvs_epilogue(f.ctx, f.hidden_in, f.n_rows_per_seq, f.first_row, f.drafts, &f.a, &f.o, f.stream));
}
static PyObject* py_decide(FAST) {
  (void)self;
  Frame f;
  frame_init(&f);
  if (PARSE("vvs_decide", decide_params, 1) < 0) return NULL;
  CALL("vvs_decide", vvs_decide(f.ctx, f.target_probs, f.n_rows_per_seq, f.first_row, f.drafts, &f.a, &f.o, f.stream));
}
static PyObject* py_decide_noalloc(FAST) {
  (void)self;
  Frame f;
  frame_init(&f);
  if (PARSE("vvs_decide_noalloc", noalloc_params, 0) < 0) return NULL;
  CALL("vvs_decide_noalloc", vvs_decide_noalloc(f.target_probs, f.vocab, f.vocab_offset, f.n_rows_per_seq, f.first_row, f.drafts,
                                                f.nbr_row_ptr, f.nbr_col, &f.a, &f.o, f.status_bits, f.stream));
}

/* ---- feature cache and the verification-free step -------------------------------------------------------------- */
typedef struct {
  vvs_ctx* ctx;
  PyObject *fc, *paths, *codebook;
  void *hidden, *base_pos, *n_store, *skip_mask, *gamma, *out, *out_pos, *stream;
  void *path_len, *last_verified, *decision, *similarity, *uniforms, *out_path, *out_gamma, *out_tokens;
  int32_t n_rows_per_seq, n_images, gamma_max, staleness, stride;
  float alpha, threshold;
} Frame2;
#define G(f) offsetof(Frame2, f)
static Param reset_params[] = {{"ctx", 'c', 1, G(ctx)}, {"fc", 'o', 1, G(fc)}, {"stream", 's', 0, G(stream)}};
static Param store_params[] = {
    {"ctx", 'c', 1, G(ctx)}, {"fc", 'o', 1, G(fc)}, {"hidden", 'p', 1, G(hidden)}, {"n_rows_per_seq", 'i', 1, G(n_rows_per_seq)},
    {"base_pos", 'p', 1, G(base_pos)}, {"n_store", 'p', 1, G(n_store)}, {"stream", 's', 0, G(stream)}};
static Param fetch_params[] = {
    {"ctx", 'c', 1, G(ctx)}, {"fc", 'o', 1, G(fc)}, {"skip_mask", 'p', 1, G(skip_mask)}, {"n_images", 'i', 1, G(n_images)},
    {"gamma", 'p', 1, G(gamma)}, {"gamma_max", 'i', 1, G(gamma_max)}, {"staleness", 'i', 1, G(staleness)}, {"out", 'p', 1, G(out)},
    {"out_pos", 'p', 1, G(out_pos)}, {"stream", 's', 0, G(stream)}};
static Param skip_params[] = {
    {"ctx", 'c', 1, G(ctx)}, {"paths", 'o', 1, G(paths)}, {"path_len", 'p', 1, G(path_len)}, {"codebook", 'o', 1, G(codebook)},
    {"last_verified", 'p', 1, G(last_verified)}, {"stride", 'i', 1, G(stride)}, {"alpha", 'f', 1, G(alpha)},
    {"threshold", 'f', 1, G(threshold)}, {"decision", 'p', 1, G(decision)}, {"similarity", 'p', 1, G(similarity)},
    {"stream", 's', 0, G(stream)}};
static Param select_params[] = {
    {"ctx", 'c', 1, G(ctx)}, {"paths", 'o', 1, G(paths)}, {"path_len", 'p', 1, G(path_len)}, {"uniforms", 'p', 1, G(uniforms)},
    {"out_path", 'p', 1, G(out_path)}, {"out_gamma", 'p', 1, G(out_gamma)}, {"out_tokens", 'p', 1, G(out_tokens)},
    {"stream", 's', 0, G(stream)}};

static int shape_of(PyObject* t, int want, int32_t* dims) {
  PyObject* sh = PyObject_GetAttr(t, s_shape);
  if (!sh) return -1;
  int rc = -1;
  if (!PyTuple_Check(sh) || PyTuple_GET_SIZE(sh) != want) {
    PyErr_Format(PyExc_ValueError, "expected a tensor of %d dimensions", want);
  } else {
    rc = 0;
    for (int i = 0; i < want && rc == 0; ++i) rc = to_int(PyTuple_GET_ITEM(sh, i), &dims[i]);
  }
  Py_DECREF(sh);
  return rc;
}
/* the structure behind a ctypes object of the given size */
static int struct_of(PyObject* o, void* out, size_t size, const char* what) {
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) < 0) return -1;
  const int ok = b.len == (Py_ssize_t)size;
  if (ok) memcpy(out, b.buf, size);
  PyBuffer_Release(&b);
  if (!ok) PyErr_Format(PyExc_TypeError, "expected a %s", what);
  return ok ? 0 : -1;
}
static int fcache_of(PyObject* o, vvs_fcache* out) { return struct_of(o, out, sizeof(*out), "vvs_fcache"); }

static PyObject* py_reset(FAST) {
  (void)self;
  Frame2 f = {0};
  vvs_fcache fc;
  if (PARSE("vvs_feature_cache_reset", reset_params, N(reset_params)) < 0 || fcache_of(f.fc, &fc) < 0) return NULL;
  CALL("vvs_feature_cache_reset", vvs_feature_cache_reset(f.ctx, &fc, f.stream));
}
static PyObject* py_store(FAST) {
  (void)self;
  Frame2 f = {0};
  vvs_fcache fc;
  if (PARSE("vvs_feature_cache_store", store_params, N(store_params)) < 0 || fcache_of(f.fc, &fc) < 0) return NULL;
  CALL("vvs_feature_cache_store", vvs_feature_cache_store(f.ctx, &fc, f.hidden, f.n_rows_per_seq, f.base_pos, f.n_store, f.stream));
}
static PyObject* py_fetch(FAST) {
  (void)self;
  Frame2 f = {0};
  vvs_fcache fc;
  if (PARSE("vvs_feature_cache_fetch", fetch_params, N(fetch_params)) < 0 || fcache_of(f.fc, &fc) < 0) return NULL;
  CALL("vvs_feature_cache_fetch", vvs_feature_cache_fetch(f.ctx, &fc, f.skip_mask, f.n_images, f.gamma, f.gamma_max, f.staleness,
                                                          f.out, f.out_pos, f.stream));
}
static PyObject* py_skip(FAST) {
  (void)self;
  Frame2 f = {0};
  int32_t d[3], e[2];
  void *paths, *codebook;
  if (PARSE("vvs_skip_decide", skip_params, N(skip_params)) < 0 || shape_of(f.paths, 3, d) < 0 || shape_of(f.codebook, 2, e) < 0 ||
      to_ptr(f.paths, &paths) < 0 || to_ptr(f.codebook, &codebook) < 0)
    return NULL;
  CALL("vvs_skip_decide", vvs_skip_decide(f.ctx, paths, f.path_len, d[0], d[1], d[2], codebook, e[0], e[1], f.last_verified,
                                          f.stride, f.alpha, f.threshold, f.decision, f.similarity, f.stream));
}
static PyObject* py_select(FAST) {
  (void)self;
  Frame2 f = {0};
  int32_t d[3];
  void* paths;
  if (PARSE("vvs_select_unverified", select_params, N(select_params)) < 0 || shape_of(f.paths, 3, d) < 0 ||
      to_ptr(f.paths, &paths) < 0)
    return NULL;
  CALL("vvs_select_unverified", vvs_select_unverified(f.ctx, paths, f.path_len, d[0], d[1], d[2], f.uniforms, f.out_path,
                                                      f.out_gamma, f.out_tokens, f.stream));
}

/* ---- 8-bit cache and rotation with several axes ------------------------------------------------------------------ */
/* What a tensor is, by the C interface that torch.Tensor offers for it (__dlpack_c_exchange_api__ of DLPack 1.3; the layouts are that
 * standard's).  One call of some 40 ns; each of data_ptr(), shape, stride() and is_contiguous() costs more, and these entry points look at
 * up to nine tensors of a call that takes 6 us. */
enum { kInt = 0, kUint = 1, kFloat = 2, kBfloat = 4, kDeviceCuda = 2 };
typedef struct {
  void* data;
  int32_t device, device_id, ndim;
  uint8_t code, bits;
  uint16_t lanes;
  int64_t *shape, *strides;
  uint64_t byte_offset;
} TensorView;
typedef struct {
  uint32_t major, minor;
  void *older, *allocate, *managed_from, *managed_to;
  int (*view)(void* tensor, TensorView* out);
  void* work_stream;
} ExchangeApi;
static const ExchangeApi* g_exchange;
static PyObject *g_tensor, *g_rope;              /* torch.Tensor; the class of make_rope_axes' results */

static int look(PyObject* o, const char* name, TensorView* v) {
  if (!PyObject_TypeCheck(o, (PyTypeObject*)g_tensor)) {
    PyErr_Format(PyExc_TypeError, "%s: expected a tensor", name);
    return -1;
  }
  if (g_exchange->view(o, v) < 0) return -1;
  v->data = (char*)v->data + v->byte_offset;
  return 0;
}
/* vvs_rope_axes, and of which block its positions are */
typedef struct {
  vvs_rope_axes r;
  int32_t n_seqs, n_rows;                        /* -1: a structure that the caller has made */
} RopeAxes;

typedef struct {
  vvs_ctx* ctx;
  PyObject *qc, *rope, *q, *k, *v, *q_out, *k_out, *out;
  PyObject *cache_len, *row_count, *row_index, *next_age, *first_slot, *visible, *lse, *mass_out, *age_out, *new_len, *kept;
  PyObject *inv_freq, *axis, *pos;
  void* stream;
  const char* elsewhere;                         /* a tensor that is not on a CUDA device */
  int32_t mass_rows, max_len, keep, n_sink, n_recent, halves;
  float scale, mass_decay;
} Frame3;

/* A contiguous array of 32-bit numbers (kind kInt: with or without a sign, kFloat), or an address that the caller answers for, or nothing: of
 * as many elements as the dimensions say, or flat and longer (n_dims 0: of any, where the library refuses what the dimensions come from). */
static int array_of(Frame3* f, PyObject* o, const char* name, int kind, int n_dims, const int64_t* dims, void** out) {
  if (!o || o == Py_None || PyLong_Check(o)) return o ? to_ptr(o, out) : 0;
  TensorView v;
  if (look(o, name, &v) < 0) return -1;
  const char* type = kind == kFloat ? "float32" : "int32";
  if (v.bits != 32 || v.lanes != 1 || (kind == kFloat ? v.code != kFloat : v.code != kInt && v.code != kUint)) {
    PyErr_Format(PyExc_ValueError, "%s: expected %s elements", name, type);
    return -1;
  }
  int64_t count = 1, side = 1;
  int dense = 1;
  for (int i = 0; i < n_dims; ++i) count *= dims[i];
  for (int i = v.ndim - 1; i >= 0; --i) {
    dense = dense && (v.shape[i] <= 1 || !v.strides || v.strides[i] == side);
    side *= v.shape[i];
  }
  if (n_dims && side != count && !(v.ndim == 1 && side > count)) {
    char text[128] = "";
    for (int i = 0, at = 0; i < n_dims && at < 100; ++i) at += snprintf(text + at, sizeof(text) - at, "%s%lld", i ? ", " : "", (long long)dims[i]);
    PyErr_Format(PyExc_ValueError, "%s: expected %s [%s]", name, type, text);
    return -1;
  }
  if (!dense) {
    PyErr_Format(PyExc_ValueError, "%s: expected a contiguous tensor", name);
    return -1;
  }
  *out = v.data;
  if (v.device != kDeviceCuda) f->elsewhere = name;
  return 0;
}
/* asked once all the tensors of a call are known to be what they should be */
static int all_on_device(const Frame3* f) {
  if (!f->elsewhere) return 0;
  PyErr_Format(PyExc_ValueError, "%s: expected a CUDA tensor", f->elsewhere);
  return -1;
}

#define H(f) offsetof(Frame3, f)
static Param rotate_params[] = {
    {"ctx", 'c', 1, H(ctx)}, {"rope", 'o', 1, H(rope)}, {"q", 'o', 1, H(q)}, {"q_out", 'o', 1, H(q_out)}, {"k", 'o', 0, H(k)},
    {"k_out", 'o', 0, H(k_out)}, {"stream", 's', 0, H(stream)}};
static Param append_params[] = {
    {"ctx", 'c', 1, H(ctx)}, {"qc", 'o', 1, H(qc)}, {"k", 'o', 1, H(k)}, {"v", 'o', 1, H(v)}, {"cache_len", 'o', 1, H(cache_len)},
    {"rope", 'o', 0, H(rope)}, {"q", 'o', 0, H(q)}, {"q_out", 'o', 0, H(q_out)}, {"row_count", 'o', 0, H(row_count)},
    {"row_index", 'o', 0, H(row_index)}, {"next_age", 'o', 0, H(next_age)}, {"stream", 's', 0, H(stream)}};
static Param attend_params[] = {
    {"ctx", 'c', 1, H(ctx)}, {"qc", 'o', 1, H(qc)}, {"q", 'o', 1, H(q)}, {"out", 'o', 1, H(out)}, {"cache_len", 'o', 1, H(cache_len)},
    {"row_count", 'o', 0, H(row_count)}, {"first_slot", 'o', 0, H(first_slot)}, {"visible", 'o', 0, H(visible)},
    {"lse", 'o', 0, H(lse)}, {"scale", 'f', 0, H(scale)}, {"mass_rows", 'i', 0, H(mass_rows)}, {"mass_decay", 'f', 0, H(mass_decay)},
    {"max_len", 'i', 0, H(max_len)}, {"stream", 's', 0, H(stream)}};
static Param evict_params[] = {
    {"ctx", 'c', 1, H(ctx)}, {"qc", 'o', 1, H(qc)}, {"cache_len", 'o', 1, H(cache_len)}, {"keep", 'i', 1, H(keep)},
    {"n_sink", 'i', 1, H(n_sink)}, {"n_recent", 'i', 1, H(n_recent)}, {"next_age", 'o', 1, H(next_age)}, {"mass_out", 'o', 1, H(mass_out)},
    {"age_out", 'o', 1, H(age_out)}, {"new_len", 'o', 1, H(new_len)}, {"kept", 'o', 1, H(kept)}, {"stream", 's', 0, H(stream)}};
static Param rope_params[] = {{"inv_freq", 'o', 1, H(inv_freq)}, {"axis", 'o', 1, H(axis)}, {"pos", 'o', 1, H(pos)}, {"halves", 'b', 0, H(halves)}};

/* a tensor [n_seqs, n_rows, n_heads, head_dim] whose last dimension lies side by side, of the context's type; dims: its sizes, checked where
 * they are not 0 */
static int heads_of(Frame3* f, PyObject* t, const char* name, vvs_heads* out, int32_t dims[4]) {
  TensorView v;
  if (look(t, name, &v) < 0) return -1;
  if (v.ndim != 4) {
    PyErr_Format(PyExc_ValueError, "%s: expected a tensor of 4 dimensions", name);
    return -1;
  }
  for (int i = 0; i < 4; ++i) {
    if ((dims[i] && dims[i] != v.shape[i]) || v.shape[i] > INT32_MAX) {
      PyErr_Format(PyExc_ValueError, "%s: dimension %d is %lld, expected %d", name, i, (long long)v.shape[i], dims[i]);
      return -1;
    }
    dims[i] = (int32_t)v.shape[i];
  }
  const int wide = f->ctx && vvs_element_bytes(f->ctx) == 4;
  if (f->ctx && (v.code != (wide ? kFloat : kBfloat) || v.bits != (wide ? 32 : 16) || v.lanes != 1)) {
    PyErr_Format(PyExc_ValueError, "%s: expected %s elements, the context's", name, wide ? "float32" : "bfloat16");
    return -1;
  }
  if (v.strides && v.strides[3] != 1 && v.shape[3] > 1) {
    PyErr_Format(PyExc_ValueError, "%s: the elements of a head do not lie side by side", name);
    return -1;
  }
  out->data = v.data;
  out->head = v.strides ? v.strides[2] : v.shape[3];
  out->row = v.strides ? v.strides[1] : out->head * v.shape[2];
  out->seq = v.strides ? v.strides[0] : out->row * v.shape[1];
  if (v.device != kDeviceCuda) f->elsewhere = name;
  return 0;
}
static int given(PyObject* o) { return o && o != Py_None; }

/* the structure behind make_rope_axes' result, or one that the caller has made; its positions have to be those of the call's rows */
static int rope_of(PyObject* o, int32_t n_seqs, int32_t n_rows, RopeAxes* out) {
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) < 0) return -1;
  const Py_ssize_t len = b.len;
  out->n_seqs = out->n_rows = -1;
  if (len == (Py_ssize_t)sizeof(RopeAxes) || len == (Py_ssize_t)sizeof(vvs_rope_axes)) memcpy(out, b.buf, len);
  PyBuffer_Release(&b);
  if (len != (Py_ssize_t)sizeof(RopeAxes) && len != (Py_ssize_t)sizeof(vvs_rope_axes)) {
    PyErr_SetString(PyExc_TypeError, "expected a vvs_rope_axes");
    return -1;
  }
  if (out->n_rows != -1 && (out->n_seqs != n_seqs || out->n_rows != n_rows)) {
    PyErr_Format(PyExc_ValueError, "rope: positions of %d sequences and %d rows, the call has %d and %d", out->n_seqs, out->n_rows, n_seqs, n_rows);
    return -1;
  }
  return 0;
}
static PyObject* py_rope(FAST) {
  (void)self;
  Frame3 f = {0};
  if (PARSE("make_rope_axes", rope_params, N(rope_params)) < 0) return NULL;
  TensorView freq, pos;
  if (look(f.inv_freq, "inv_freq", &freq) < 0 || look(f.pos, "pos", &pos) < 0) return NULL;
  if (freq.ndim != 1 || pos.ndim != 3 || freq.shape[0] > INT32_MAX || pos.shape[0] > INT32_MAX || pos.shape[1] > INT32_MAX ||
      pos.shape[2] > INT32_MAX) {
    PyErr_SetString(PyExc_ValueError, "expected inv_freq [n_pairs], axis [n_pairs] and pos [n_axes, n_seqs, n_rows]");
    return NULL;
  }
  const int64_t pairs[1] = {freq.shape[0]}, where[3] = {pos.shape[0], pos.shape[1], pos.shape[2]};
  void *p_freq = NULL, *p_axis = NULL, *p_pos = NULL;
  if (array_of(&f, f.inv_freq, "inv_freq", kFloat, 1, pairs, &p_freq) < 0 || array_of(&f, f.axis, "axis", kInt, 1, pairs, &p_axis) < 0 ||
      array_of(&f, f.pos, "pos", kInt, 3, where, &p_pos) < 0 || all_on_device(&f) < 0)
    return NULL;
  const RopeAxes r = {{p_freq, p_axis, p_pos, (int32_t)where[0], (int32_t)pairs[0], f.halves != 0}, (int32_t)where[1], (int32_t)where[2]};
  PyObject* made = PyObject_CallNoArgs(g_rope);
  if (!made) return NULL;
  Py_buffer b;
  PyObject* keep = NULL;
  int rc = PyObject_GetBuffer(made, &b, PyBUF_WRITABLE);
  if (rc == 0) {
    if (b.len == (Py_ssize_t)sizeof(r)) memcpy(b.buf, &r, sizeof(r));
    else rc = -1, PyErr_SetString(PyExc_SystemError, "the class of make_rope_axes' results has another layout");
    PyBuffer_Release(&b);
  }
  if (rc == 0) {
    keep = PyTuple_Pack(3, f.inv_freq, f.axis, f.pos);
    rc = keep ? PyObject_SetAttr(made, s_keep, keep) : -1;
    Py_XDECREF(keep);
  }
  if (rc < 0) Py_CLEAR(made);
  return made;
}

static PyObject* py_rotate(FAST) {
  (void)self;
  Frame3 f = {0};
  RopeAxes rope;
  vvs_heads q, q_out, k, k_out;
  int32_t d[4] = {0}, e[4] = {0};
  if (PARSE("vvs_rotate_axes", rotate_params, N(rotate_params)) < 0 || heads_of(&f, f.q, "q", &q, d) < 0 ||
      heads_of(&f, f.q_out, "q_out", &q_out, d) < 0 || rope_of(f.rope, d[0], d[1], &rope) < 0)
    return NULL;
  const int two = given(f.k), two_out = given(f.k_out);
  e[0] = d[0], e[1] = d[1], e[3] = d[3];
  if (two && heads_of(&f, f.k, "k", &k, e) < 0) return NULL;
  if ((two_out && heads_of(&f, f.k_out, "k_out", &k_out, e) < 0) || all_on_device(&f) < 0) return NULL;
  CALL("vvs_rotate_axes", vvs_rotate_axes(f.ctx, &rope.r, d[0], d[1], d[2], e[2], d[3], &q, &q_out, two ? &k : NULL,
                                          two_out ? &k_out : NULL, f.stream));
}
static PyObject* py_append(FAST) {
  (void)self;
  Frame3 f = {0};
  vvs_qcache qc;
  RopeAxes rope;
  vvs_heads q, q_out, k, v;
  if (PARSE("vvs_quant_cache_append", append_params, N(append_params)) < 0 || struct_of(f.qc, &qc, sizeof(qc), "vvs_qcache") < 0)
    return NULL;
  int32_t d[4] = {qc.n_seqs, 0, qc.n_heads, qc.head_dim}, e[4] = {0};
  if (heads_of(&f, f.k, "k", &k, d) < 0 || heads_of(&f, f.v, "v", &v, d) < 0) return NULL;
  const int turn = given(f.rope), also_q = given(f.q), also_out = given(f.q_out);
  if (turn && rope_of(f.rope, d[0], d[1], &rope) < 0) return NULL;
  e[0] = d[0], e[1] = d[1], e[3] = d[3];
  if (also_q && heads_of(&f, f.q, "q", &q, e) < 0) return NULL;
  if (also_out && heads_of(&f, f.q_out, "q_out", &q_out, e) < 0) return NULL;
  const int64_t seqs[2] = {d[0], d[1]};
  void *cache_len = NULL, *row_count = NULL, *row_index = NULL, *next_age = NULL;
  if (array_of(&f, f.cache_len, "cache_len", kInt, 1, seqs, &cache_len) < 0 ||
      array_of(&f, f.row_count, "row_count", kInt, 1, seqs, &row_count) < 0 ||
      array_of(&f, f.row_index, "row_index", kInt, also_q ? 0 : 2, seqs, &row_index) < 0 ||
      array_of(&f, f.next_age, "next_age", kInt, 1, seqs, &next_age) < 0 || all_on_device(&f) < 0)
    return NULL;
  CALL("vvs_quant_cache_append",
       vvs_quant_cache_append(f.ctx, &qc, &k, &v, cache_len, d[1], row_count, row_index, next_age, turn ? &rope.r : NULL, e[2],
                              also_q ? &q : NULL, also_out ? &q_out : NULL, f.stream));
}
static PyObject* py_attend(FAST) {
  (void)self;
  Frame3 f = {0};
  vvs_qcache qc;
  vvs_heads q, out;
  f.mass_decay = 1.f;
  if (PARSE("vvs_quant_cache_attend", attend_params, N(attend_params)) < 0 || struct_of(f.qc, &qc, sizeof(qc), "vvs_qcache") < 0)
    return NULL;
  int32_t d[4] = {qc.n_seqs, 0, 0, qc.head_dim};
  if (heads_of(&f, f.q, "q", &q, d) < 0 || heads_of(&f, f.out, "out", &out, d) < 0) return NULL;
  const int64_t seqs[3] = {d[0], d[1], d[2]};
  void *cache_len = NULL, *row_count = NULL, *first_slot = NULL, *visible = NULL, *lse = NULL;
  if (array_of(&f, f.cache_len, "cache_len", kInt, 1, seqs, &cache_len) < 0 ||
      array_of(&f, f.row_count, "row_count", kInt, 1, seqs, &row_count) < 0 ||
      array_of(&f, f.first_slot, "first_slot", kInt, 1, seqs, &first_slot) < 0 ||
      array_of(&f, f.visible, "visible", kInt, d[1] > 32 ? 0 : 2, seqs, &visible) < 0 ||
      array_of(&f, f.lse, "lse", kFloat, 3, seqs, &lse) < 0 || all_on_device(&f) < 0)
    return NULL;
  CALL("vvs_quant_cache_attend", vvs_quant_cache_attend(f.ctx, &qc, &q, &out, cache_len, d[1], d[2], row_count, first_slot, visible, lse, f.scale,
                                                        f.mass_rows, f.mass_decay, f.max_len, f.stream));
}
static PyObject* py_evict(FAST) {
  (void)self;
  Frame3 f = {0};
  vvs_qcache qc;
  if (PARSE("vvs_quant_cache_evict", evict_params, N(evict_params)) < 0 || struct_of(f.qc, &qc, sizeof(qc), "vvs_qcache") < 0)
    return NULL;
  const int64_t slots[3] = {qc.n_seqs, qc.n_heads, qc.cap}, stay[3] = {qc.n_seqs, qc.n_heads, f.keep};
  void *cache_len = NULL, *next_age = NULL, *mass_out = NULL, *age_out = NULL, *new_len = NULL, *kept = NULL;
  if (array_of(&f, f.cache_len, "cache_len", kInt, 1, slots, &cache_len) < 0 || array_of(&f, f.next_age, "next_age", kInt, 1, slots, &next_age) < 0 ||
      array_of(&f, f.mass_out, "mass_out", kFloat, 3, slots, &mass_out) < 0 || array_of(&f, f.age_out, "age_out", kInt, 3, slots, &age_out) < 0 ||
      array_of(&f, f.new_len, "new_len", kInt, 1, slots, &new_len) < 0 ||
      array_of(&f, f.kept, "kept", kInt, f.keep < 1 || f.keep > qc.cap ? 0 : 3, stay, &kept) < 0 || all_on_device(&f) < 0)
    return NULL;
  CALL("vvs_quant_cache_evict", vvs_quant_cache_evict(f.ctx, &qc, cache_len, f.keep, f.n_sink, f.n_recent, next_age, mass_out, age_out, new_len, kept,
                                                      f.stream));
}

/* setup(VvsError, current_raw_stream, current_device, Tensor, class of make_rope_axes' results) */
static PyObject* py_setup(PyObject* self, PyObject* args) {
  (void)self;
  PyObject *e, *r, *d, *t, *rope;
  if (!PyArg_ParseTuple(args, "OOOO!O", &e, &r, &d, &PyType_Type, &t, &rope)) return NULL;
  PyObject* api = PyObject_GetAttrString(t, "__dlpack_c_exchange_api__");
  if (!api) return NULL;
  g_exchange = PyCapsule_GetPointer(api, "dlpack_exchange_api");        /* (torch's own, for as long as it is loaded) */
  Py_DECREF(api);
  if (!g_exchange) return NULL;
  if (g_exchange->major != 1 || g_exchange->minor < 3) {
    PyErr_Format(PyExc_ImportError, "torch offers tensors by DLPack %u.%u, expected 1.3 or a later 1.x", g_exchange->major, g_exchange->minor);
    return NULL;
  }
  Py_XSETREF(g_error, Py_NewRef(e));
  Py_XSETREF(g_raw_stream, Py_NewRef(r));
  Py_XSETREF(g_get_device, Py_NewRef(d));
  Py_XSETREF(g_tensor, Py_NewRef(t));
  Py_XSETREF(g_rope, Py_NewRef(rope));
  Py_RETURN_NONE;
}

#define FN(name, f, doc) {name, (PyCFunction)(void (*)(void))f, METH_FASTCALL | METH_KEYWORDS, doc}
static PyMethodDef methods[] = {
    {"setup", py_setup, METH_VARARGS, NULL},
    FN("vvs_verify", py_verify, "vvs_verify(ctx, **fields of vvs_verify_args and vvs_verify_out, stream=None): one verification step."),
    FN("vvs_epilogue", py_epilogue, "LM head and decisions on given features."),
    FN("vvs_decide", py_decide, "Decisions on given target probabilities."),
    FN("vvs_decide_noalloc", py_decide_noalloc,
       "vvs_decide for callers that must not allocate device memory: no context (limits: 64 images, 16 drafts, 64 "
       "neighbours, vocab 65536; chains only: tree_parent / accept_path are refused)."),
    FN("vvs_feature_cache_reset", py_reset, "vvs_feature_cache_reset(ctx, fc, stream=None)"),
    FN("vvs_feature_cache_store", py_store, "vvs_feature_cache_store(ctx, fc, hidden, n_rows_per_seq, base_pos, n_store, stream=None)"),
    FN("vvs_feature_cache_fetch", py_fetch,
       "vvs_feature_cache_fetch(ctx, fc, skip_mask, n_images, gamma, gamma_max, staleness, out, out_pos, stream=None)"),
    FN("vvs_skip_decide", py_skip,
       "Alg. 1 / Eq. 2 of the paper: vvs_skip_decide(ctx, paths, path_len, codebook, last_verified, stride, alpha, threshold, "
       "decision, similarity, stream=None); paths int32 [B, N, L], path_len int32 [B, N] or None, codebook float32 [V, dim], "
       "last_verified uint8 [B] or None -> decision uint8 [B], similarity float32 [B]."),
    FN("vvs_select_unverified", py_select,
       "Sec. 4.2 / Eq. 3: uniform draw of one candidate path per image, cut to gamma tokens: vvs_select_unverified(ctx, paths, "
       "path_len, uniforms, out_path, out_gamma, out_tokens, stream=None)."),
    FN("make_rope_axes", py_rope,
       "make_rope_axes(inv_freq, axis, pos, halves=False): inv_freq float32 [n_pairs], axis int32 [n_pairs], pos int32 [n_axes, n_seqs, n_rows] "
       "(CUDA tensors, contiguous), for calls of n_seqs sequences and n_rows rows."),
    FN("vvs_rotate_axes", py_rotate,
       "vvs_rotate_axes(ctx, rope, q, q_out, k=None, k_out=None, stream=None): q, k [n_seqs, n_rows, heads, head_dim], any strides of "
       "whole 16 bytes but the last; rope from make_rope_axes."),
    FN("vvs_quant_cache_append", py_append,
       "vvs_quant_cache_append(ctx, qc, k, v, cache_len, rope=None, q=None, q_out=None, row_count=None, row_index=None, next_age=None, "
       "stream=None): k, v [n_seqs, n_rows, cached heads, head_dim] behind cache_len int32 [n_seqs]; qc from make_qcache."),
    FN("vvs_quant_cache_attend", py_attend,
       "vvs_quant_cache_attend(ctx, qc, q, out, cache_len, row_count=None, first_slot=None, visible=None, lse=None, scale=0.0, mass_rows=0, "
       "mass_decay=1.0, max_len=0, stream=None): q, out [n_seqs, n_rows, heads, head_dim]; scale 0 = 1 / sqrt(head_dim)."),
    FN("vvs_quant_cache_evict", py_evict,
       "vvs_quant_cache_evict(ctx, qc, cache_len, keep, n_sink, n_recent, next_age, mass_out, age_out, new_len, kept, stream=None)"),
    {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", NULL, -1, methods, NULL, NULL, NULL, NULL};

static int intern(Param* ps, int n) {
  for (int i = 0; i < n; ++i)
    if (!(ps[i].key = PyUnicode_InternFromString(ps[i].name))) return -1;
  return 0;
}
PyMODINIT_FUNC PyInit__native(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_shape = PyUnicode_InternFromString("shape");
  s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  s_keep = PyUnicode_InternFromString("_keep");
#define I(ps) intern(ps, N(ps)) < 0
  if (!s_data_ptr || !s_shape || !s_cuda_stream || !s_keep || I(verify_params) || I(epilogue_params) || I(decide_params) || I(noalloc_params) ||
      I(reset_params) || I(store_params) || I(fetch_params) || I(skip_params) || I(select_params) || I(rotate_params) ||
      I(append_params) || I(attend_params) || I(evict_params) || I(rope_params))
    return NULL;
  return PyModule_Create(&module);
}
