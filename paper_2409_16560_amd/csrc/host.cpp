// The host side of the calls that a decoding step makes several times and whose kernels are short (draft layers, the forest
// layout, and what runs once per transformer layer or row of logits): checks, output tensors and the call into libdsbd.so without the interpreter in between.  From Python a draft layer
// took 17.5 us of host time, 6 of them its two launches, which is longer than its kernels.
//
// A module of its own: libdsbd.so knows nothing of torch.  binding.py holds the public functions, with their defaults, the
// fault words and the error codes' exceptions; these take every argument by position.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ATen.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include "dsbd.h"

namespace {

// A tensor argument; `optional`: None stands for none.
const at::Tensor* tensor(PyObject* o, bool optional = false) {
  if (optional && o == Py_None) return nullptr;
  TORCH_CHECK_TYPE(THPVariable_Check(o), "expected a tensor");
  return &THPVariable_Unpack(o);
}
long long integer(PyObject* o) {
  PyObject* const n = PyNumber_Long(o);
  if (!n) throw python_error();
  const long long v = PyLong_AsLongLong(n);
  Py_DECREF(n);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}
int32_t int32(PyObject* o) {
  const long long v = integer(o);
  TORCH_CHECK_VALUE(v >= INT32_MIN && v <= INT32_MAX, "integer argument out of range");
  return (int32_t)v;
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return v;
}
void* stream(PyObject* o) {
  void* const p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw python_error();
  return p;
}
// What the binding asserts of its arguments.
#define EXPECT(x)                                              \
  do {                                                         \
    if (!(x)) {                                                \
      PyErr_SetString(PyExc_AssertionError, #x);               \
      throw python_error();                                    \
    }                                                          \
  } while (0)

PyObject* wrap(const at::Tensor& t) {
  PyObject* const o = THPVariable_Wrap(t);
  if (!o) throw python_error();
  return o;
}

// draft_layer(beam_off, logits, logp, u, W_S, max_prompt_beams, top_k, top_p, workspace, fault, stream): the outputs (parent,
// token, logp), or an error code of the library; a workspace query that fails is the code -2 as an empty tuple.
PyObject* draft_layer(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(n == 11, "draft_layer takes 11 arguments");
  const at::Tensor &beam_off = *tensor(args[0]), &z = *tensor(args[1]), &cum = *tensor(args[2]), &u = *tensor(args[3]);
  const int32_t W_S = int32(args[4]), top_k = int32(args[6]);
  const float top_p = (float)number(args[7]);
  const at::Tensor* const given = tensor(args[8], true);
  const at::Tensor& fault = *tensor(args[9]);
  void* const s = stream(args[10]);
  TORCH_CHECK_VALUE(z.dim() == 2, "logits_draft is [n_beams, V]");
  const int64_t P = beam_off.numel() - 1;
  EXPECT(beam_off.scalar_type() == at::kInt && z.scalar_type() == at::kFloat && z.is_contiguous());
  EXPECT(cum.scalar_type() == at::kDouble && u.scalar_type() == at::kFloat && u.is_contiguous());
  EXPECT(u.numel() == P * W_S && cum.numel() == z.size(0));
  dsbd_draft_in in;
  in.n_prompts = (int32_t)P; in.n_beams = (int32_t)z.size(0); in.max_prompt_beams = int32(args[5]); in.V = (int32_t)z.size(1);
  in.beam_off = (const int32_t*)beam_off.data_ptr(); in.logits_draft = (const float*)z.data_ptr();
  in.beam_logp_draft = (const double*)cum.data_ptr(); in.u = (const float*)u.data_ptr();
  const auto on = z.options();
  const at::Tensor parent = at::empty({P, W_S}, on.dtype(at::kInt)), token = at::empty({P, W_S}, on.dtype(at::kInt));
  const at::Tensor logp = at::empty({P, W_S}, on.dtype(at::kDouble));
  dsbd_draft_out out;
  out.parent = (int32_t*)parent.data_ptr(); out.token = (int32_t*)token.data_ptr(); out.logp_draft = (double*)logp.data_ptr();
  at::Tensor workspace;
  if (given) workspace = *given;
  else {
    const size_t bytes = dsbd_draft_layer_workspace_bytes(&in, W_S, top_k, top_p);
    if (bytes == 0) return PyTuple_New(0);
    workspace = at::empty({(int64_t)(bytes > 256 ? bytes : 256)}, on.dtype(at::kByte));
  }
  void* const ws = workspace.data_ptr();
  const size_t ws_bytes = (size_t)workspace.numel();
  int32_t* const fw = (int32_t*)fault.data_ptr();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = dsbd_draft_layer(&in, W_S, top_k, top_p, &out, ws, ws_bytes, fw, s);
  Py_END_ALLOW_THREADS
  if (rc != DSBD_OK) return PyLong_FromLong(rc);
  PyObject* const r = PyTuple_New(3);
  if (!r) throw python_error();
  PyTuple_SET_ITEM(r, 0, wrap(parent));
  PyTuple_SET_ITEM(r, 1, wrap(token));
  PyTuple_SET_ITEM(r, 2, wrap(logp));
  return r;
  END_HANDLE_TH_ERRORS
}

// build_forest(root_off, layer_parent, layer_token, root_token, n_roots, fault, stream): (gamma, tree_prompt, tree_off,
// parent, token, draft_rank, node_of_root, node_of, max_tree_nodes), or an error code.
PyObject* build_forest(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(n == 7, "build_forest takes 7 arguments");
  const at::Tensor& root_off = *tensor(args[0]);
  const at::Tensor *layer_parent = tensor(args[1], true), *layer_token = tensor(args[2], true), *root_token = tensor(args[3], true);
  const int64_t n_roots = integer(args[4]);
  const at::Tensor& fault = *tensor(args[5]);
  void* const s = stream(args[6]);
  const int64_t P = root_off.numel() - 1;
  const int64_t gamma = layer_parent && layer_parent->numel() > 0 ? layer_parent->size(0) : 0;
  if (gamma && P == 0) {
    PyErr_SetString(PyExc_ZeroDivisionError, "layers without prompts");
    throw python_error();
  }
  const int64_t W_S = gamma ? layer_parent->size(1) / P : 0;
  const int64_t D = gamma * P * W_S, N = n_roots + D;
  const at::Tensor* const all[4] = {&root_off, layer_parent, layer_token, root_token};
  for (const at::Tensor* t : all) EXPECT(t == nullptr || (t->scalar_type() == at::kInt && t->is_contiguous()));
  // one allocation, cut into the arrays (an array of no entries has no pointer of its own)
  const int64_t sizes[8] = {n_roots, n_roots + 1, N, N, N, n_roots, D, 1};
  int64_t total = 0;
  for (int64_t k : sizes) total += k;
  const at::Tensor buf = at::empty({total}, root_off.options().dtype(at::kInt));
  int32_t* at_ = (int32_t*)buf.data_ptr();
  at::Tensor part[8];
  int32_t* place[8];
  int64_t off = 0;
  for (int k = 0; k < 8; ++k) {
    place[k] = at_ + off;
    part[k] = k == 6 && gamma ? buf.as_strided({gamma, P * W_S}, {P * W_S, 1}, off) : buf.as_strided({sizes[k]}, {1}, off);
    off += sizes[k];
  }
  dsbd_forest_out out;
  out.tree_prompt = place[0]; out.tree_off = place[1]; out.parent = place[2]; out.token = place[3]; out.draft_rank = place[4];
  out.node_of_root = place[5]; out.node_of = place[6]; out.max_tree_nodes = place[7];
  const int32_t* const ro = (const int32_t*)root_off.data_ptr();
  const int32_t* const rt = root_token ? (const int32_t*)root_token->data_ptr() : nullptr;
  const int32_t* const lp = gamma ? (const int32_t*)layer_parent->data_ptr() : nullptr;
  const int32_t* const lt = gamma && layer_token ? (const int32_t*)layer_token->data_ptr() : nullptr;
  int32_t* const fw = (int32_t*)fault.data_ptr();
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = dsbd_build_forest((int32_t)P, (int32_t)n_roots, (int32_t)gamma, (int32_t)W_S, ro, rt, lp, lt, &out, fw, s);
  Py_END_ALLOW_THREADS
  if (rc != DSBD_OK) return PyLong_FromLong(rc);
  PyObject* const r = PyTuple_New(9);
  if (!r) throw python_error();
  PyTuple_SET_ITEM(r, 0, PyLong_FromLongLong(gamma));
  for (int k = 0; k < 8; ++k) PyTuple_SET_ITEM(r, k + 1, wrap(part[k]));
  return r;
  END_HANDLE_TH_ERRORS
}

// ---- rows of a projection, paged caches, rules on logits

// An attribute of a handle.  (The names are interned once.)
struct Name {
  PyObject* const s;
  explicit Name(const char* n) : s(PyUnicode_InternFromString(n)) {}
};
struct Attr {
  PyObject* const o;
  Attr(PyObject* from, const Name& n) : o(PyObject_GetAttr(from, n.s)) { if (!o) throw python_error(); }
  ~Attr() { Py_DECREF(o); }
  Attr(const Attr&) = delete;
};
// The attributes that a call takes of its handles, until it returns: a handle may work one out on demand, or be given another by a
// thread that runs meanwhile.
struct Held {
  PyObject* o[24];
  int n = 0;
  Held() = default;
  Held(const Held&) = delete;
  ~Held() { while (n) Py_DECREF(o[--n]); }
};
// A tensor attribute, or none.
const at::Tensor* tensor_of(Held& held, PyObject* o, const Name& n, bool optional = false) {
  EXPECT(held.n < (int)(sizeof(held.o) / sizeof(held.o[0])));
  PyObject* const t = PyObject_GetAttr(o, n.s);
  if (!t) throw python_error();
  held.o[held.n++] = t;
  return tensor(t, optional);
}
int64_t integer_of(PyObject* o, const Name& n) { return integer(Attr(o, n).o); }
int32_t int32_of(PyObject* o, const Name& n) { return int32(Attr(o, n).o); }
bool truth_of(PyObject* o, const Name& n) {
  const int r = PyObject_IsTrue(Attr(o, n).o);
  if (r < 0) throw python_error();
  return r != 0;
}

int32_t element_type(const at::Tensor& t) {
  return t.scalar_type() == at::kBFloat16 ? DSBD_BF16 : t.scalar_type() == at::kHalf ? DSBD_F16 : t.scalar_type() == at::kFloat ? DSBD_F32 : -1;
}
void* data(const at::Tensor* t) { return t && t->numel() ? t->data_ptr() : nullptr; }
// The handles' arrays of one type, on the call's device.
const at::Tensor* array(const at::Tensor* t, at::ScalarType type, const at::Tensor& like) {
  if (t) {
    EXPECT(t->scalar_type() == type && t->is_contiguous());
    EXPECT(t->device() == like.device());
  }
  return t;
}

// Rows [n,H,D].  (The stride of a dimension of one entry says nothing.)
dsbd_rows rows(const at::Tensor& t, const at::Tensor& like, bool output) {
  EXPECT(t.dim() == 3 && t.scalar_type() == like.scalar_type());
  EXPECT(t.size(2) <= 1 || t.stride(2) == 1);
  EXPECT(t.device() == like.device());
  const int64_t n = t.size(0), H = t.size(1), D = t.size(2), ts = n > 1 ? t.stride(0) : 0, hs = H > 1 ? t.stride(1) : 0;
  if (output)   // no two rows share memory
    EXPECT((H <= 1 || hs >= D) && (n <= 1 || ts >= (H - 1) * hs + D || (ts >= D && (H <= 1 || hs >= (n - 1) * ts + D))));
  return dsbd_rows{t.numel() ? t.data_ptr() : nullptr, ts, hs};
}
bool same_shape(const at::Tensor& a, int64_t n, int64_t H, int64_t D) {
  return a.dim() == 3 && a.size(0) == n && a.size(1) == H && a.size(2) == D;
}

dsbd_qk_prep prep_of(Held& held, PyObject* o, const at::Tensor& like, int64_t Hq, int64_t Hk, int64_t D) {
  static const Name q_weight("q_weight"), k_weight("k_weight"), inv_freq("inv_freq"), eps("eps"), rot_scale("rot_scale"), norm("norm"),
      interleaved("interleaved");
  dsbd_qk_prep p;
  const at::Tensor* const w[2] = {array(tensor_of(held, o, q_weight, true), like.scalar_type(), like),
                                  array(tensor_of(held, o, k_weight, true), like.scalar_type(), like)};
  const at::Tensor* const f = array(tensor_of(held, o, inv_freq, true), at::kDouble, like);
  const int64_t heads[2] = {Hq, Hk};
  int64_t dims = 0;
  for (int i = 0; i < 2; ++i)
    if (w[i] && heads[i] > 0) {      // one vector for all heads, or one per head, for q and k alike
      EXPECT((w[i]->dim() == 1 && w[i]->size(0) == D) || (w[i]->dim() == 2 && w[i]->size(0) == heads[i] && w[i]->size(1) == D));
      EXPECT(dims == 0 || dims == w[i]->dim());
      dims = w[i]->dim();
    }
  p.q_weight = data(w[0]); p.k_weight = data(w[1]); p.inv_freq = (const double*)data(f);
  p.eps = (float)number(Attr(o, eps).o); p.rot_scale = (float)number(Attr(o, rot_scale).o);
  EXPECT(f == nullptr || 2 * f->numel() <= D);
  p.rot_dim = f ? (int32_t)(2 * f->numel()) : 0;
  p.norm = truth_of(o, norm); p.per_head = dims == 2; p.interleaved = truth_of(o, interleaved);
  return p;
}

// The cache of a handle; `Hkv` and `D` as its pages have them.
dsbd_paged_kv cache_of(Held& held, PyObject* o, const at::Tensor& like, int64_t& Hkv, int64_t& D) {
  static const Name k_pages("k_pages"), v_pages("v_pages"), page_table("page_table"), ctx_len("ctx_len"), q_off("q_off"),
      max_new("max_new"), max_len("max_len"), head_major("head_major");
  const at::Tensor &k = *tensor_of(held, o, k_pages), &v = *tensor_of(held, o, v_pages), &table = *tensor_of(held, o, page_table);
  const at::Tensor &ctx = *tensor_of(held, o, ctx_len), &off = *tensor_of(held, o, q_off);
  EXPECT(k.dim() == 4 && v.sizes() == k.sizes() && k.scalar_type() == like.scalar_type() && v.scalar_type() == like.scalar_type());
  EXPECT(k.numel() == 0 || (k.strides() == v.strides() && k.stride(3) == 1));
  EXPECT(table.dim() == 2 && off.numel() == ctx.numel() + 1 && table.size(0) == ctx.numel());
  array(&table, at::kInt, like); array(&ctx, at::kInt, like); array(&off, at::kInt, like);
  EXPECT(k.device() == like.device() && v.device() == like.device());
  const bool hm = truth_of(o, head_major);
  const int64_t slots = hm ? k.size(2) : k.size(1);
  Hkv = hm ? k.size(1) : k.size(2);
  D = k.size(3);
  const auto stride = [&](int64_t d) { return k.numel() && k.size(d) > 1 ? k.stride(d) : 0; };
  // a page's slots, and the pages, are written side by side: none may share memory with another
  EXPECT(k.numel() == 0 || k.is_non_overlapping_and_dense() || (k.stride(0) > 0 && k.stride(1) > 0 && k.stride(2) > 0));
  EXPECT(k.size(0) <= INT32_MAX && slots <= INT32_MAX && table.size(1) <= INT32_MAX && ctx.numel() < INT32_MAX);
  dsbd_paged_kv c;
  c.k_pages = data(&k); c.v_pages = data(&v);
  c.page_table = (const int32_t*)data(&table); c.ctx_len = (const int32_t*)data(&ctx); c.q_off = (const int32_t*)data(&off);
  c.page_stride = stride(0); c.token_stride = stride(hm ? 2 : 1); c.head_stride = stride(hm ? 1 : 2);
  c.n_pages = (int32_t)k.size(0); c.page_size = (int32_t)slots; c.table_stride = (int32_t)table.size(1); c.n_seqs = (int32_t)ctx.numel();
  c.max_new = int32_of(o, max_new); c.max_len = int32_of(o, max_len);
  return c;
}

// Rows of `like`'s kind, packed.
at::Tensor packed(const at::Tensor& like) { return at::empty(like.sizes(), like.options()); }
int32_t* fault_word(const at::Tensor& f, const at::Tensor& like) {
  EXPECT(f.scalar_type() == at::kInt && f.numel() >= 1);
  EXPECT(f.device() == like.device());
  return (int32_t*)f.data_ptr();
}
// The launches need a GPU's memory; everything else has been checked by then.
void on_gpu(const at::Tensor& t) { TORCH_CHECK_VALUE(t.is_cuda(), "the tensors must be on a GPU"); }

// qk_norm_rope(q, k, v, positions, prep, q_out, k_out, v_out, stream): (q_out, k_out, v_out), or an error code.
PyObject* qk_norm_rope(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(n == 9, "qk_norm_rope takes 9 arguments");
  Held held;
  const at::Tensor* const in[3] = {tensor(args[0], true), tensor(args[1], true), tensor(args[2], true)};
  const at::Tensor* const like_ = in[0] ? in[0] : in[1] ? in[1] : in[2];
  TORCH_CHECK_VALUE(like_ != nullptr, "no rows given");
  const at::Tensor& like = *like_;
  TORCH_CHECK_VALUE(like.dim() == 3, "rows are [n, heads, D]");
  const int64_t N = like.size(0), D = like.size(2);
  const at::Tensor* const pos = array(tensor(args[3], true), at::kInt, like);
  EXPECT(pos == nullptr || pos->numel() == N);
  EXPECT(N <= INT32_MAX && D <= INT32_MAX);
  EXPECT(in[1] == nullptr || in[2] == nullptr || in[1]->sizes() == in[2]->sizes());
  at::Tensor made[3];
  dsbd_rows from[3], to[3];
  int64_t H[3] = {0, 0, 0};
  for (int i = 0; i < 3; ++i) {
    const at::Tensor* const given = tensor(args[5 + i], true);
    EXPECT(in[i] != nullptr || given == nullptr);
    if (!in[i]) continue;
    H[i] = in[i]->dim() == 3 ? in[i]->size(1) : 0;
    EXPECT(same_shape(*in[i], N, H[i], D) && H[i] <= INT32_MAX);
    from[i] = rows(*in[i], like, false);
    made[i] = given ? *given : packed(*in[i]);
    EXPECT(same_shape(made[i], N, H[i], D));
    to[i] = rows(made[i], like, true);
  }
  dsbd_qk_prep prep;
  if (args[4] != Py_None) prep = prep_of(held, args[4], like, H[0], H[1], D);
  void* const s = stream(args[8]);
  on_gpu(like);
  int32_t rc = DSBD_OK;
  const dsbd_rows *x[3], *y[3];      // (what has no heads is not there for the library)
  for (int i = 0; i < 3; ++i) { x[i] = H[i] > 0 ? &from[i] : nullptr; y[i] = H[i] > 0 ? &to[i] : nullptr; }
  if (N > 0 && D > 0 && (x[0] || x[1] || x[2])) {
    Py_BEGIN_ALLOW_THREADS
    rc = dsbd_qk_norm_rope((int32_t)N, (int32_t)H[0], (int32_t)(in[1] ? H[1] : H[2]), (int32_t)D, element_type(like), x[0], x[1], x[2],
                           (const int32_t*)data(pos), args[4] != Py_None ? &prep : nullptr, y[0], y[1], y[2], s);
    Py_END_ALLOW_THREADS
  }
  if (rc != DSBD_OK) return PyLong_FromLong(rc);
  PyObject* const r = PyTuple_New(3);
  if (!r) throw python_error();
  for (int i = 0; i < 3; ++i) {
    if (!in[i]) Py_INCREF(Py_None);
    PyTuple_SET_ITEM(r, i, in[i] ? wrap(made[i]) : Py_None);
  }
  return r;
  END_HANDLE_TH_ERRORS
}

// paged_append(cache, k, v, q, positions, prep, q_out, fault, stream): q_out (None without q), or an error code.
PyObject* paged_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(n == 9, "paged_append takes 9 arguments");
  Held held;
  const at::Tensor &k = *tensor(args[1]), &v = *tensor(args[2]);
  const at::Tensor *const q = tensor(args[3], true), *const given = tensor(args[6], true);
  TORCH_CHECK_VALUE(k.dim() == 3, "k is [n, heads, D]");
  int64_t Hkv, D;
  const dsbd_paged_kv cache = cache_of(held, args[0], k, Hkv, D);
  const int64_t N = k.size(0), Hq = q && q->dim() == 3 ? q->size(1) : 0;
  EXPECT(same_shape(k, N, Hkv, D) && same_shape(v, N, Hkv, D) && N <= INT32_MAX && Hkv <= INT32_MAX && D <= INT32_MAX);
  EXPECT(q == nullptr || (same_shape(*q, N, Hq, D) && Hq <= INT32_MAX));
  EXPECT(q != nullptr || given == nullptr);
  const at::Tensor* const pos = array(tensor(args[4], true), at::kInt, k);
  EXPECT(pos == nullptr || pos->numel() == N);
  const dsbd_rows kr = rows(k, k, false), vr = rows(v, k, false);
  dsbd_rows qr, to;
  at::Tensor made;
  if (q) {
    qr = rows(*q, k, false);
    made = given ? *given : packed(*q);
    EXPECT(same_shape(made, N, Hq, D));
    to = rows(made, k, true);
  }
  dsbd_qk_prep prep;
  if (args[5] != Py_None) prep = prep_of(held, args[5], k, Hq, Hkv, D);
  int32_t* const fw = fault_word(*tensor(args[7]), k);
  void* const s = stream(args[8]);
  on_gpu(k);
  int32_t rc = DSBD_OK;
  if (N > 0) {
    Py_BEGIN_ALLOW_THREADS
    rc = dsbd_paged_append(&cache, (int32_t)N, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, element_type(k), q ? &qr : nullptr, &kr, &vr,
                           (const int32_t*)data(pos), args[5] != Py_None ? &prep : nullptr, q ? &to : nullptr, fw, s);
    Py_END_ALLOW_THREADS
  }
  if (rc != DSBD_OK) return PyLong_FromLong(rc);
  if (!q) Py_RETURN_NONE;
  return wrap(made);
  END_HANDLE_TH_ERRORS
}

// paged_attention(cache, q, scale, anc_mask, out, lse, want_lse, workspace, fault, stream): (out, lse), or an error code; a
// workspace query that fails is the code -2 as an empty tuple.
PyObject* paged_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(n == 10, "paged_attention takes 10 arguments");
  Held held;
  const at::Tensor& q = *tensor(args[1]);
  TORCH_CHECK_VALUE(q.dim() == 3, "q is [n, heads, D]");
  int64_t Hkv, D;
  const dsbd_paged_kv cache = cache_of(held, args[0], q, Hkv, D);
  const int64_t N = q.size(0), Hq = q.size(1);
  EXPECT(q.size(2) == D && N <= INT32_MAX && Hq <= INT32_MAX && Hkv <= INT32_MAX && D <= INT32_MAX);
  const float scale = (float)number(args[2]);
  const at::Tensor *const anc = tensor(args[3], true), *const out_ = tensor(args[4], true), *const lse_ = tensor(args[5], true);
  const at::Tensor* const given = tensor(args[7], true);
  if (anc) {
    EXPECT(anc->scalar_type() == at::kLong || anc->scalar_type() == at::kUInt64);
    EXPECT(anc->is_contiguous() && anc->numel() == N && anc->device() == q.device());
  }
  const dsbd_rows qr = rows(q, q, false);
  const at::Tensor out = out_ ? *out_ : packed(q);
  EXPECT(same_shape(out, N, Hq, D));
  const dsbd_rows to = rows(out, q, true);
  const bool want = lse_ || PyObject_IsTrue(args[6]) == 1;
  if (lse_) EXPECT(array(lse_, at::kFloat, q)->numel() == N * Hq);
  int32_t* const fw = fault_word(*tensor(args[8]), q);
  void* const s = stream(args[9]);
  const size_t need = dsbd_paged_attention_workspace_bytes(&cache, (int32_t)N, (int32_t)Hq, (int32_t)Hkv, (int32_t)D);
  if (need == 0 && q.numel() > 0) return PyTuple_New(0);
  if (given) {
    EXPECT(given->is_contiguous());
    EXPECT(given->device() == q.device());
  }
  on_gpu(q);
  const at::Tensor lse = lse_ ? *lse_ : want ? at::empty({N, Hq}, q.options().dtype(at::kFloat)) : at::Tensor();
  const at::Tensor workspace = given ? *given : at::empty({(int64_t)(need > 256 ? need : 256)}, q.options().dtype(at::kByte));
  int32_t rc = DSBD_OK;
  if (q.numel() > 0) {
    void* const ws = workspace.data_ptr();
    const size_t ws_bytes = workspace.nbytes();
    float* const lp = want ? (float*)lse.data_ptr() : nullptr;
    Py_BEGIN_ALLOW_THREADS
    rc = dsbd_paged_attention(&cache, (int32_t)N, (int32_t)Hq, (int32_t)Hkv, (int32_t)D, element_type(q), &qr, scale,
                              (const uint64_t*)data(anc), &to, lp, ws, ws_bytes, fw, s);
    Py_END_ALLOW_THREADS
  }
  if (rc != DSBD_OK) return PyLong_FromLong(rc);
  PyObject* const r = PyTuple_New(2);
  if (!r) throw python_error();
  PyTuple_SET_ITEM(r, 0, wrap(out));
  if (!want) Py_INCREF(Py_None);
  PyTuple_SET_ITEM(r, 1, want ? wrap(lse) : Py_None);
  return r;
  END_HANDLE_TH_ERRORS
}

// paged_attention_workspace_bytes(cache, like, n_rows, Hq): bytes, 0 for what is not supported.
PyObject* paged_attention_workspace_bytes(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(n == 3, "paged_attention_workspace_bytes takes 3 arguments");
  Held held;
  static const Name k_pages("k_pages");
  int64_t Hkv, D;
  const dsbd_paged_kv cache = cache_of(held, args[0], *tensor_of(held, args[0], k_pages), Hkv, D);
  EXPECT(Hkv <= INT32_MAX && D <= INT32_MAX);
  return PyLong_FromSize_t(dsbd_paged_attention_workspace_bytes(&cache, int32(args[1]), int32(args[2]), (int32_t)Hkv, (int32_t)D));
  END_HANDLE_TH_ERRORS
}

// process_logits(forest, logits, rules, row_node, out, fault, stream): out, or an error code.
PyObject* process_logits(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(n == 7, "process_logits takes 7 arguments");
  Held held;
  static const Name tree_prompt("tree_prompt"), tree_off("tree_off"), parent("parent"), token("token"), n_prompts("n_prompts"),
      n_trees("n_trees"), n_nodes("n_nodes"), max_tree_nodes("max_tree_nodes"), max_depth("max_depth"), max_prompt_trees("max_prompt_trees");
  static const Name hist("hist"), hist_off("hist_off"), prompt_len("prompt_len"), repetition("repetition"), frequency("frequency"),
      presence("presence"), temperature("temperature"), bias_off("bias_off"), bias_token("bias_token"), bias_value("bias_value"), mask("mask"),
      mask_row("mask_row");
  PyObject *const fo = args[0], *const ro = args[2];
  const at::Tensor& z = *tensor(args[1]);
  TORCH_CHECK_VALUE(z.dim() == 2, "logits are [n_rows, V]");
  const int64_t R = z.size(0), V = z.size(1);
  EXPECT(R <= INT32_MAX && V <= INT32_MAX && element_type(z) >= 0 && (V <= 1 || z.stride(1) == 1));
  dsbd_forest f;
  const at::Tensor *const tp = array(tensor_of(held, fo, tree_prompt), at::kInt, z), *const to = array(tensor_of(held, fo, tree_off), at::kInt, z);
  const at::Tensor *const pa = array(tensor_of(held, fo, parent), at::kInt, z), *const tk = array(tensor_of(held, fo, token, true), at::kInt, z);
  f.n_prompts = int32_of(fo, n_prompts); f.n_trees = int32_of(fo, n_trees); f.n_nodes = int32_of(fo, n_nodes);
  EXPECT(f.n_trees >= 0 && f.n_nodes >= 0 && f.n_prompts >= 0);
  EXPECT(tp->numel() == f.n_trees && to->numel() == (int64_t)f.n_trees + 1 && pa->numel() == f.n_nodes);
  TORCH_CHECK_VALUE(tk != nullptr && tk->numel() == f.n_nodes, "the forest has no tokens");
  f.tree_prompt = (const int32_t*)data(tp); f.tree_off = (const int32_t*)data(to); f.parent = (const int32_t*)data(pa);
  f.token = (const int32_t*)data(tk); f.draft_rank = nullptr;
  f.max_tree_nodes = int32_of(fo, max_tree_nodes); f.max_depth = int32_of(fo, max_depth); f.max_prompt_trees = int32_of(fo, max_prompt_trees);
  dsbd_logit_rules r;
  const auto ints = [&](const Name& name, int64_t count) {
    const at::Tensor* const t = array(tensor_of(held, ro, name, true), at::kInt, z);
    EXPECT(t == nullptr || count < 0 || t->numel() == count);
    return t;
  };
  const auto floats = [&](const Name& name, int64_t count) {
    const at::Tensor* const t = array(tensor_of(held, ro, name, true), at::kFloat, z);
    EXPECT(t == nullptr || count < 0 || t->numel() == count);
    return t;
  };
  const at::Tensor *const h = ints(hist, -1), *const ho = ints(hist_off, (int64_t)f.n_trees + 1);
  EXPECT(h == nullptr || ho != nullptr);
  const at::Tensor *const bo = ints(bias_off, (int64_t)f.n_prompts + 1), *const bt = ints(bias_token, -1);
  const at::Tensor* const bv = floats(bias_value, bt ? bt->numel() : 0);
  EXPECT((bo != nullptr) == (bt != nullptr) && (bt != nullptr) == (bv != nullptr));
  const at::Tensor *const mk = ints(mask, -1), *const mr = ints(mask_row, R);
  EXPECT(mk == nullptr || (mk->dim() == 2 && mk->size(1) >= (V + 31) / 32 && mk->size(0) <= INT32_MAX));
  EXPECT(mk == nullptr || mr != nullptr || mk->size(0) == R);
  r.hist = (const int32_t*)data(h); r.hist_off = ho ? (const int32_t*)ho->data_ptr() : nullptr;
  r.prompt_len = (const int32_t*)data(ints(prompt_len, f.n_trees));
  r.repetition = (const float*)data(floats(repetition, f.n_prompts)); r.frequency = (const float*)data(floats(frequency, f.n_prompts));
  r.presence = (const float*)data(floats(presence, f.n_prompts)); r.temperature = (const float*)data(floats(temperature, f.n_prompts));
  r.bias_off = bo ? (const int32_t*)bo->data_ptr() : nullptr; r.bias_token = (const int32_t*)data(bt); r.bias_value = (const float*)data(bv);
  r.mask = (const uint32_t*)data(mk); r.mask_row = (const int32_t*)data(mr); r.mask_stride = mk ? mk->size(1) : 0;
  r.n_masks = mk ? (int32_t)mk->size(0) : 0;
  EXPECT((!h || h->numel() <= INT32_MAX) && (!bt || bt->numel() <= INT32_MAX));
  r.n_hist = h ? (int32_t)h->numel() : 0; r.n_bias = bt ? (int32_t)bt->numel() : 0;
  const at::Tensor* const rn = array(tensor(args[3], true), at::kInt, z);
  EXPECT(rn ? rn->numel() == R : f.n_nodes == R);
  const at::Tensor* const given = tensor(args[4], true);
  if (given) {
    EXPECT(given->dim() == 2 && given->size(0) == R && given->size(1) == V && given->scalar_type() == at::kFloat);
    EXPECT((V <= 1 || given->stride(1) == 1) && (R <= 1 || given->stride(0) >= V));
    EXPECT(given->device() == z.device());
  }
  int32_t* const fw = fault_word(*tensor(args[5]), z);
  void* const s = stream(args[6]);
  on_gpu(z);
  const at::Tensor out = given ? *given : at::empty({R, V}, z.options().dtype(at::kFloat));
  int32_t rc = DSBD_OK;
  if (z.numel() > 0) {
    const void* const zp = z.data_ptr();
    float* const op = (float*)out.data_ptr();
    const int64_t zs = R > 1 ? z.stride(0) : V, os = R > 1 ? out.stride(0) : V;
    Py_BEGIN_ALLOW_THREADS
    rc = dsbd_process_logits(&f, (const int32_t*)data(rn), (int32_t)R, (int32_t)V, element_type(z), zp, zs, &r, op, os, fw, s);
    Py_END_ALLOW_THREADS
  }
  if (rc != DSBD_OK) return PyLong_FromLong(rc);
  return wrap(out);
  END_HANDLE_TH_ERRORS
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    FAST(qk_norm_rope), FAST(paged_append), FAST(paged_attention), FAST(paged_attention_workspace_bytes), FAST(process_logits),
    {"draft_layer", (PyCFunction)(void (*)(void))draft_layer, METH_FASTCALL, nullptr},
    {"build_forest", (PyCFunction)(void (*)(void))build_forest, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_dsbd_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dsbd_host(void) { return PyModule_Create(&module); }
