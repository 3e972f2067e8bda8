// Native half of the Python binding: the calls that a loop over chunks makes, from tensors to the C ABI.  A call of the
// library costs 10 to 25 us of host time in kernel launches; marshalled through ctypes it took another 6 us and more
// (every pointer an object, every shape and stride tuple built and compared in Python), which short calls felt.
// Every function returns the library's status, or -1 if a tensor does not fit the descriptor -- the Python wrapper
// then says which, or takes the call itself --, or -2 if the page lists have to be copied first.  So it does where torch throws (strides of a 0-dim or sparse tensor, the
// address of a tensor without storage): no exception leaves this file.  The interpreter lock is released during the
// call of the library.
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/oomb.h"

namespace {

PyObject* g_raw_stream = nullptr;   // torch._C._cuda_getCurrentRawStream(device index)

template <typename S> struct DescOf {
  Py_buffer view{};
  S* d = nullptr;
  explicit DescOf(PyObject* o) {
    if (PyObject_GetBuffer(o, &view, PyBUF_WRITABLE) == 0) {
      if (view.len == (Py_ssize_t)sizeof(S)) d = (S*)view.buf;
    } else {
      PyErr_Clear();
    }
  }
  ~DescOf() { if (view.obj) PyBuffer_Release(&view); }
};
using Desc = DescOf<oomb_attn_desc>;

// one argument: a tensor, None (nullptr), or neither (bad)
const at::Tensor* tensor(PyObject* o, bool& bad) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) { bad = true; return nullptr; }
  return &THPVariable_Unpack(o);
}
void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
size_t bytes(const at::Tensor* t) { return t ? t->numel() * t->element_size() : 0; }
at::ScalarType type_of(int32_t dt) { return dt == OOMB_BF16 ? at::kBFloat16 : at::kFloat; }

bool like(const at::Tensor* t, const at::Tensor& ref, at::ScalarType dt) {
  return !t || (t->scalar_type() == dt && t->sizes() == ref.sizes() && t->strides() == ref.strides());
}
// q and the pools against the descriptor, as the Python wrapper checks them
bool family(const oomb_attn_desc& d, const at::Tensor* q, const at::Tensor* k, const at::Tensor* lse) {
  if (!q || !k || q->dim() != 3 || k->dim() != 4) return false;
  if (lse && (lse->scalar_type() != at::kFloat || lse->dim() != 2 || lse->size(0) != d.n_q_heads || lse->size(1) != d.chunk_len || !lse->is_contiguous()))
    return false;
  return q->stride(0) == d.q_tok_stride && q->stride(1) == d.q_head_stride && q->scalar_type() == type_of(d.dtype) &&
         k->stride(0) == d.pool_page_stride && k->stride(1) == d.pool_head_stride && k->stride(2) == d.pool_tok_stride;
}
bool stream_of(const at::Tensor* t, void** st) {
  if (!t || !t->is_cuda()) return false;
  PyObject* idx = PyLong_FromLong(t->get_device());
  PyObject* r = idx ? PyObject_CallOneArg(g_raw_stream, idx) : nullptr;
  Py_XDECREF(idx);
  if (!r) { PyErr_Clear(); return false; }
  *st = PyLong_AsVoidPtr(r);
  Py_DECREF(r);
  return true;
}
PyObject* status(int s) { return PyLong_FromLong(s); }
struct Unlocked {   // (taken back on an exception too)
  PyThreadState* s = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(s); }
};
#define OOMB_CALL(expr) \
  oomb_status s_; \
  { Unlocked u_; s_ = (expr); } \
  return status((int)s_)

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)> PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  try {
    return F(self, a, nargs);
  } catch (const std::exception&) {
    PyErr_Clear();
    return status(-1);
  }
}

// 0, -1 (does not fit), or -2: lists that are a view whose last row ends with the memory before its stride does.  The kernels
// read whole rows of min(stride, n) entries before they know how many are valid.
int list_args(const oomb_attn_desc& d, const at::Tensor* sel, const at::Tensor* cnt, bool qp, int32_t* stride) {
  if (!qp) {
    *stride = sel ? (int32_t)sel->stride(0) : 0;
    if (!sel || sel->dim() != 2 || sel->size(0) != d.n_kv_heads || sel->size(1) >= sel->stride(0) || d.page_size <= 0) return 0;
    const int64_t n = d.ctx_len / d.page_size, row = sel->stride(0) < n ? sel->stride(0) : n;
    return (size_t)(sel->storage_offset() + (d.n_kv_heads - 1) * sel->stride(0) + row) * sel->element_size() > sel->storage().nbytes() ? -2 : 0;
  }
  const int64_t m = d.page_size > 0 ? d.chunk_len / d.page_size : 0;
  if (!sel || !cnt || sel->dim() != 3 || sel->size(0) != d.n_kv_heads || sel->size(1) != m || !sel->is_contiguous() || cnt->dim() != 2 ||
      cnt->size(0) != d.n_kv_heads || cnt->size(1) != m || !cnt->is_contiguous())
    return -1;
  *stride = (int32_t)sel->size(2);
  return 0;
}

#define OOMB_ARGS(n) if (nargs != (n)) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; } \
  bool bad = false; Desc desc(a[0]); void* st = nullptr; if (!desc.d) return status(-1); const oomb_attn_desc& d = *desc.d; (void)d; (void)bad; (void)st

// make_desc(desc, q, k_pool, ctx_len, sm_scale, grad_is_bf16)
PyObject* make_desc(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ARGS(6);
  const at::Tensor *q = tensor(a[1], bad), *k = tensor(a[2], bad);
  if (bad || !q || !k || q->dim() != 3 || k->dim() != 4 || q->stride(2) != 1 || k->stride(3) != 1 || q->size(2) != k->size(3)) return status(-1);
  if (q->scalar_type() != at::kFloat && q->scalar_type() != at::kBFloat16) return status(-1);
  const long long ctx = PyLong_AsLongLong(a[3]);
  const double scale = PyFloat_AsDouble(a[4]);
  if (PyErr_Occurred()) { PyErr_Clear(); return status(-1); }
  oomb_attn_desc& w = *desc.d;
  w.n_q_heads = (int32_t)q->size(1); w.n_kv_heads = (int32_t)k->size(1); w.head_dim = (int32_t)q->size(2); w.page_size = (int32_t)k->size(2);
  w.chunk_len = (int32_t)q->size(0); w.dtype = q->scalar_type() == at::kBFloat16 ? OOMB_BF16 : OOMB_F32;
  w.grad_dtype = a[5] == Py_True ? OOMB_BF16 : OOMB_F32; w.sm_scale = (float)scale; w.ctx_len = ctx;
  w.pool_page_stride = k->stride(0); w.pool_head_stride = k->stride(1); w.pool_tok_stride = k->stride(2);
  w.q_tok_stride = q->stride(0); w.q_head_stride = q->stride(1); w.num_phys_pages = k->size(0);
  return status(0);
}

// score_topk(desc, q, k_pool, page_table, top_k, sel_pages, sel_count, scores_out, workspace)
PyObject* score_topk(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ARGS(9);
  const at::Tensor *q = tensor(a[1], bad), *k = tensor(a[2], bad), *pt = tensor(a[3], bad), *sel = tensor(a[5], bad), *cnt = tensor(a[6], bad),
                   *sc = tensor(a[7], bad), *ws = tensor(a[8], bad);
  const long top_k = PyLong_AsLong(a[4]);
  if (PyErr_Occurred()) { PyErr_Clear(); return status(-1); }
  if (bad || !stream_of(q, &st)) return status(-1);
  OOMB_CALL(oomb_page_score_topk(&d, ptr(q), ptr(k), (const int32_t*)ptr(pt), (int32_t)top_k, (int32_t*)ptr(sel), (int32_t*)ptr(cnt), (float*)ptr(sc), ptr(ws),
                                 bytes(ws), st));
}

// score_topk_cached / vote_topk(desc, q, kbar_cache, top_k, sel_pages, sel_count, out, workspace)
template <oomb_status (*F)(const oomb_attn_desc*, const void*, const float*, int32_t, int32_t*, int32_t*, float*, void*, size_t, void*)>
PyObject* from_means(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ARGS(8);
  const at::Tensor *q = tensor(a[1], bad), *kb = tensor(a[2], bad), *sel = tensor(a[4], bad), *cnt = tensor(a[5], bad), *out = tensor(a[6], bad),
                   *ws = tensor(a[7], bad);
  const long top_k = PyLong_AsLong(a[3]);
  if (PyErr_Occurred()) { PyErr_Clear(); return status(-1); }
  if (bad || !stream_of(q, &st)) return status(-1);
  OOMB_CALL(F(&d, ptr(q), (const float*)ptr(kb), (int32_t)top_k, (int32_t*)ptr(sel), (int32_t*)ptr(cnt), (float*)ptr(out), ptr(ws), bytes(ws), st));
}

// attn_fwd / attn_fwd_qp(desc, q, k_pool, v_pool, page_table, sel_pages, sel_count, o, lse, workspace)
template <bool QP> PyObject* attn_fwd(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ARGS(10);
  const at::Tensor *q = tensor(a[1], bad), *k = tensor(a[2], bad), *v = tensor(a[3], bad), *pt = tensor(a[4], bad), *sel = tensor(a[5], bad),
                   *cnt = tensor(a[6], bad), *o = tensor(a[7], bad), *lse = tensor(a[8], bad), *ws = tensor(a[9], bad);
  int32_t stride = 0;
  if (bad || !family(d, q, k, lse) || !like(o, *q, q->scalar_type()) || !like(v, *k, k->scalar_type())) return status(-1);
  if (const int s = list_args(d, sel, cnt, QP, &stride); s != 0) return status(s);
  if (!stream_of(q, &st)) return status(-1);
  OOMB_CALL((QP ? oomb_paged_attn_fwd_qp : oomb_paged_attn_fwd)(&d, ptr(q), ptr(k), ptr(v), (const int32_t*)ptr(pt), (const int32_t*)ptr(sel),
                                                                (const int32_t*)ptr(cnt), stride, ptr(o), (float*)ptr(lse), ptr(ws), bytes(ws), st));
}

// attn_bwd / attn_bwd_qp(desc, q, k_pool, v_pool, page_table, sel_pages, sel_count, o, lse, d_o, d_q, dk_pool, dv_pool, workspace)
template <bool QP> PyObject* attn_bwd(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ARGS(14);
  const at::Tensor *q = tensor(a[1], bad), *k = tensor(a[2], bad), *v = tensor(a[3], bad), *pt = tensor(a[4], bad), *sel = tensor(a[5], bad),
                   *cnt = tensor(a[6], bad), *o = tensor(a[7], bad), *lse = tensor(a[8], bad), *d_o = tensor(a[9], bad), *d_q = tensor(a[10], bad),
                   *dk = tensor(a[11], bad), *dv = tensor(a[12], bad), *ws = tensor(a[13], bad);
  int32_t stride = 0;
  if (bad || !family(d, q, k, lse)) return status(-1);
  const at::ScalarType t = q->scalar_type(), gt = type_of(d.grad_dtype);
  if (!like(o, *q, t) || !like(d_o, *q, t) || !like(d_q, *q, t) || !like(v, *k, k->scalar_type()) || !like(dk, *k, gt) || !like(dv, *k, gt)) return status(-1);
  if (const int s = list_args(d, sel, cnt, QP, &stride); s != 0) return status(s);
  if (!stream_of(q, &st)) return status(-1);
  OOMB_CALL((QP ? oomb_paged_attn_bwd_qp : oomb_paged_attn_bwd)(&d, ptr(q), ptr(k), ptr(v), (const int32_t*)ptr(pt), (const int32_t*)ptr(sel),
                                                                (const int32_t*)ptr(cnt), stride, ptr(o), (const float*)ptr(lse), ptr(d_o), ptr(d_q), ptr(dk),
                                                                ptr(dv), ptr(ws), bytes(ws), st));
}

// kv_append(desc, k_chunk, v_chunk, page_table, k_pool, v_pool, kbar_cache)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ARGS(7);
  const at::Tensor *kc = tensor(a[1], bad), *vc = tensor(a[2], bad), *pt = tensor(a[3], bad), *k = tensor(a[4], bad), *v = tensor(a[5], bad),
                   *kb = tensor(a[6], bad);
  if (bad || !kc || !vc || !k || !kc->is_contiguous() || !vc->is_contiguous() || kc->sizes() != vc->sizes() || kc->scalar_type() != k->scalar_type() ||
      vc->scalar_type() != k->scalar_type() || !like(v, *k, k->scalar_type()) || !stream_of(k, &st))
    return status(-1);
  OOMB_CALL(oomb_kv_append(&d, ptr(kc), ptr(vc), (const int32_t*)ptr(pt), ptr(k), ptr(v), (float*)ptr(kb), st));
}

// local_page_list(desc, window_pages, sel_pages, sel_count)
PyObject* local_page_list(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ARGS(4);
  const long window = PyLong_AsLong(a[1]);
  if (PyErr_Occurred()) { PyErr_Clear(); return status(-1); }
  const at::Tensor *sel = tensor(a[2], bad), *cnt = tensor(a[3], bad);
  if (bad || !stream_of(sel, &st)) return status(-1);
  OOMB_CALL(oomb_local_page_list(&d, (int32_t)window, (int32_t*)ptr(sel), (int32_t*)ptr(cnt), st));
}

// ---- packed rows ----------------------------------------------------------------------------------------------
// The tensors of such a call lie on one device, which need not be the current one.

int64_t pages_of(const oomb_rows_desc& d) { return d.page_size > 0 ? (d.max_len + d.page_size - 1) / d.page_size : 0; }
bool row_tensor(const oomb_rows_desc& d, const at::Tensor* t, int32_t heads, oomb_rows* out) {
  if (!t || t->dim() != 3 || t->scalar_type() != type_of(d.dtype) || t->size(0) != d.n_rows || t->size(1) != heads || t->size(2) != d.head_dim || t->stride(2) != 1)
    return false;
  *out = {t->data_ptr(), t->stride(0), t->stride(1)};
  return true;
}
bool ints(const at::Tensor* t, int64_t n) { return !t || (t->scalar_type() == at::kInt && t->dim() == 1 && t->size(0) == n && t->is_contiguous()); }
bool seqs_of(const oomb_rows_desc& d, const at::Tensor* tables, const at::Tensor* lens, const at::Tensor* starts, oomb_seqs* out) {
  if (!tables || tables->scalar_type() != at::kInt || !ints(lens, d.n_seqs) || !ints(starts, (int64_t)d.n_seqs + 1)) return false;
  if (tables->dim() == 1 ? d.n_seqs != 1 : tables->dim() != 2 || tables->size(0) != d.n_seqs || (d.n_seqs > 1 && tables->stride(0) != d.table_stride)) return false;
  if (tables->size(-1) < pages_of(d) || (tables->size(-1) > 1 && tables->stride(-1) != 1)) return false;
  *out = {(const int32_t*)tables->data_ptr(), (const int32_t*)ptr(lens), (const int32_t*)ptr(starts)};
  return true;
}
bool pool(const oomb_rows_desc& d, const at::Tensor* t, at::ScalarType dt, bool kvq) {
  if (!t || t->scalar_type() != dt || t->dim() != (kvq ? 3 : 4) || t->size(0) != d.num_phys_pages || t->size(1) != d.n_kv_heads) return false;
  if (t->stride(0) != d.pool_page_stride || t->stride(1) != d.pool_head_stride) return false;
  if (kvq) return t->size(2) == (int64_t)d.page_size * (d.head_dim / 2 + d.head_dim / 32) && t->stride(2) == 1;
  return t->size(2) == d.page_size && t->size(3) == d.head_dim && t->stride(2) == d.pool_tok_stride && t->stride(3) == 1;
}
bool rope_of(const oomb_rows_desc& d, const at::Tensor* cos, const at::Tensor* sin, bool interleaved, oomb_rope* out) {
  *out = {nullptr, nullptr, 0, 0, interleaved};
  if (!cos && !sin) return true;
  if (!cos || !sin || cos->scalar_type() != at::kFloat || sin->scalar_type() != at::kFloat || cos->dim() != 2 || cos->sizes() != sin->sizes() ||
      !cos->is_contiguous() || !sin->is_contiguous() || cos->size(1) > d.head_dim)
    return false;
  *out = {(const float*)cos->data_ptr(), (const float*)sin->data_ptr(), cos->size(0), (int32_t)(2 * cos->size(1)), interleaved};
  return true;
}
bool means(const oomb_rows_desc& d, const at::Tensor* t) {
  return !t || (t->scalar_type() == at::kFloat && t->dim() >= 3 && t->is_contiguous() && t->size(-2) == d.n_kv_heads && t->size(-1) == d.head_dim &&
                t->numel() >= ((d.n_seqs - 1) * d.table_stride + pages_of(d)) * d.n_kv_heads * d.head_dim &&
                (t->dim() == 3 ? d.n_seqs == 1 : t->dim() == 4 && t->size(0) == d.n_seqs && (d.n_seqs == 1 || t->size(1) == d.table_stride)));
}
// All on one device, where its current stream goes to *st; the guard keeps that device current during the call.
bool place(std::initializer_list<const at::Tensor*> ts, void** st, c10::OptionalDeviceGuard* guard) {
  const at::Tensor* one = nullptr;
  for (const at::Tensor* t : ts) {
    if (!t) continue;
    if (one && t->device() != one->device()) return false;
    one = t;
  }
  if (!stream_of(one, st)) return false;
  guard->reset_device(one->device());
  return true;
}

#define OOMB_ROWS_ARGS(n) if (nargs != (n)) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; } \
  bool bad = false; DescOf<oomb_rows_desc> desc(a[0]); void* st = nullptr; if (!desc.d) return status(-1); const oomb_rows_desc& d = *desc.d; \
  c10::OptionalDeviceGuard guard

// make_rows_desc(desc, q, pool, page_tables, max_len, sm_scale, max_rows); max_rows 0: the rows of all
PyObject* make_rows_desc(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ROWS_ARGS(7);
  (void)d; (void)st;
  const at::Tensor *q = tensor(a[1], bad), *k = tensor(a[2], bad), *t = tensor(a[3], bad);
  if (bad || !q || !k || !t || q->dim() != 3 || (t->dim() != 1 && t->dim() != 2)) return status(-1);
  if (q->scalar_type() != at::kFloat && q->scalar_type() != at::kBFloat16) return status(-1);
  const bool kvq = k->scalar_type() == at::kByte;
  if (k->dim() != (kvq ? 3 : 4)) return status(-1);
  const long long len = PyLong_AsLongLong(a[4]);
  const double scale = PyFloat_AsDouble(a[5]);
  const long most = PyLong_AsLong(a[6]);
  if (PyErr_Occurred()) { PyErr_Clear(); return status(-1); }
  const int64_t D = q->size(2), seqs = t->dim() == 1 ? 1 : t->size(0), token = D / 2 + D / 32;
  if (kvq && (token <= 0 || k->size(2) % token)) return status(-1);
  if (q->size(0) > INT32_MAX || seqs > INT32_MAX || most < 0 || most > INT32_MAX) return status(-1);
  oomb_rows_desc& w = *desc.d;
  w = {};
  w.n_q_heads = (int32_t)q->size(1); w.n_kv_heads = (int32_t)k->size(1); w.head_dim = (int32_t)D;
  w.page_size = (int32_t)(kvq ? k->size(2) / token : k->size(2));
  w.dtype = q->scalar_type() == at::kBFloat16 ? OOMB_BF16 : OOMB_F32;
  w.n_seqs = (int32_t)seqs; w.n_rows = (int32_t)q->size(0); w.max_rows = most ? (int32_t)most : w.n_rows;
  w.sm_scale = (float)scale; w.max_len = len;
  w.table_stride = t->dim() == 2 && seqs > 1 ? t->stride(0) : t->size(-1);
  w.num_phys_pages = k->size(0);
  w.pool_page_stride = k->stride(0); w.pool_head_stride = k->stride(1); w.pool_tok_stride = kvq ? 0 : k->stride(2);
  return status(0);
}

// append_rope(desc, cos, sin, interleaved, q, q_out, k, v, page_tables, seq_lens, row_starts, k_pool, v_pool, kbar_cache)
template <bool KVQ> PyObject* append_rope(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ROWS_ARGS(14);
  const at::Tensor *cos = tensor(a[1], bad), *sin = tensor(a[2], bad), *q = tensor(a[4], bad), *qo = tensor(a[5], bad), *k = tensor(a[6], bad), *v = tensor(a[7], bad),
                   *pt = tensor(a[8], bad), *lens = tensor(a[9], bad), *starts = tensor(a[10], bad), *kp = tensor(a[11], bad), *vp = tensor(a[12], bad),
                   *kb = tensor(a[13], bad);
  oomb_rope rope; oomb_seqs seqs; oomb_rows rq{}, rqo{}, rk, rv;
  const at::ScalarType pt_ = KVQ ? at::kByte : type_of(d.dtype);
  if (bad || !rope_of(d, cos, sin, a[3] == Py_True, &rope) || !seqs_of(d, pt, lens, starts, &seqs) || (q == nullptr) != (qo == nullptr) ||
      (q && (!row_tensor(d, q, d.n_q_heads, &rq) || !row_tensor(d, qo, d.n_q_heads, &rqo))) || !row_tensor(d, k, d.n_kv_heads, &rk) ||
      !row_tensor(d, v, d.n_kv_heads, &rv) || !pool(d, kp, pt_, KVQ) || !pool(d, vp, pt_, KVQ) || !means(d, kb) ||
      !place({cos, sin, q, qo, k, v, pt, lens, starts, kp, vp, kb}, &st, &guard))
    return status(-1);
  OOMB_CALL((KVQ ? oomb_kvq_append_rope : oomb_kv_append_rope)(&d, &seqs, &rope, q ? &rq : nullptr, q ? &rqo : nullptr, &rk, &rv, ptr(kp), ptr(vp), (float*)ptr(kb), st));
}

// append_rope_bwd(desc, cos, sin, interleaved, d_q, d_q_out, d_k, d_v, page_tables, seq_lens, row_starts, dk_pool, dv_pool)
PyObject* append_rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ROWS_ARGS(13);
  const at::Tensor *cos = tensor(a[1], bad), *sin = tensor(a[2], bad), *q = tensor(a[4], bad), *qo = tensor(a[5], bad), *k = tensor(a[6], bad), *v = tensor(a[7], bad),
                   *pt = tensor(a[8], bad), *lens = tensor(a[9], bad), *starts = tensor(a[10], bad), *kp = tensor(a[11], bad), *vp = tensor(a[12], bad);
  oomb_rope rope; oomb_seqs seqs; oomb_rows rq{}, rqo{}, rk, rv;
  if (bad || !kp) return status(-1);
  const at::ScalarType gt = kp->scalar_type();
  if ((gt != at::kFloat && gt != at::kBFloat16) || !rope_of(d, cos, sin, a[3] == Py_True, &rope) || !seqs_of(d, pt, lens, starts, &seqs) ||
      (q == nullptr) != (qo == nullptr) || (q && (!row_tensor(d, q, d.n_q_heads, &rq) || !row_tensor(d, qo, d.n_q_heads, &rqo))) ||
      !row_tensor(d, k, d.n_kv_heads, &rk) || !row_tensor(d, v, d.n_kv_heads, &rv) || !pool(d, kp, gt, false) || !pool(d, vp, gt, false) ||
      !place({cos, sin, q, qo, k, v, pt, lens, starts, kp, vp}, &st, &guard))
    return status(-1);
  OOMB_CALL(oomb_kv_append_rope_bwd(&d, &seqs, &rope, q ? &rq : nullptr, q ? &rqo : nullptr, ptr(kp), ptr(vp), gt == at::kBFloat16 ? OOMB_BF16 : OOMB_F32, &rk, &rv, st));
}

// kvq_read(desc, page_tables, seq_lens, row_starts, k_pool, v_pool, k_out, v_out)
PyObject* kvq_read(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ROWS_ARGS(8);
  const at::Tensor *pt = tensor(a[1], bad), *lens = tensor(a[2], bad), *starts = tensor(a[3], bad), *kp = tensor(a[4], bad), *vp = tensor(a[5], bad), *k = tensor(a[6], bad),
                   *v = tensor(a[7], bad);
  oomb_seqs seqs; oomb_rows rk, rv;
  if (bad || !seqs_of(d, pt, lens, starts, &seqs) || !pool(d, kp, at::kByte, true) || !pool(d, vp, at::kByte, true) || !row_tensor(d, k, d.n_kv_heads, &rk) ||
      !row_tensor(d, v, d.n_kv_heads, &rv) || !place({pt, lens, starts, kp, vp, k, v}, &st, &guard))
    return status(-1);
  OOMB_CALL(oomb_kvq_read(&d, &seqs, ptr(kp), ptr(vp), &rk, &rv, st));
}

// attn_fwd_kvq(desc, q, k_pool, v_pool, page_tables, seq_lens, row_starts, sel_pages, sel_count, o, lse, workspace)
PyObject* attn_fwd_kvq(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  OOMB_ROWS_ARGS(12);
  const at::Tensor *q = tensor(a[1], bad), *kp = tensor(a[2], bad), *vp = tensor(a[3], bad), *pt = tensor(a[4], bad), *lens = tensor(a[5], bad), *starts = tensor(a[6], bad),
                   *sel = tensor(a[7], bad), *cnt = tensor(a[8], bad), *o = tensor(a[9], bad), *lse = tensor(a[10], bad), *ws = tensor(a[11], bad);
  oomb_seqs seqs; oomb_rows rq, ro;
  if (bad || !row_tensor(d, q, d.n_q_heads, &rq) || !row_tensor(d, o, d.n_q_heads, &ro) || !pool(d, kp, at::kByte, true) || !pool(d, vp, at::kByte, true) ||
      !seqs_of(d, pt, lens, starts, &seqs) || !lse || lse->scalar_type() != at::kFloat || lse->dim() != 2 || lse->size(0) != d.n_q_heads || lse->size(1) != d.n_rows ||
      !lse->is_contiguous() || (ws && !ws->is_contiguous()))
    return status(-1);
  const int64_t lists = (int64_t)d.n_seqs * d.n_kv_heads;
  int32_t stride = 0;
  if (sel) {
    if (!cnt || sel->scalar_type() != at::kInt || cnt->scalar_type() != at::kInt || !sel->is_contiguous() || !cnt->is_contiguous() || cnt->numel() != lists ||
        sel->dim() < 2 || sel->size(-1) > INT32_MAX || sel->numel() != lists * sel->size(-1))
      return status(-1);
    stride = (int32_t)sel->size(-1);
  }
  if (!place({q, kp, vp, pt, lens, starts, sel, sel ? cnt : nullptr, o, lse, ws}, &st, &guard)) return status(-1);
  // (lists without room are lists all the same: a tensor without elements has no address, so they go by that of the counts, which is not read through)
  const int32_t* lists_at = (const int32_t*)ptr(sel && stride == 0 ? cnt : sel);
  OOMB_CALL(oomb_paged_attn_fwd_kvq(&d, &seqs, &rq, ptr(kp), ptr(vp), lists_at, (const int32_t*)ptr(cnt), stride, &ro, (float*)ptr(lse), ptr(ws), bytes(ws), st));
}

#define OOMB_METHOD(name, fn) {name, (PyCFunction)(void (*)(void))(guarded<fn>), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    OOMB_METHOD("make_desc", make_desc),
    OOMB_METHOD("score_topk", score_topk),
    OOMB_METHOD("score_topk_cached", from_means<oomb_page_score_topk_cached>),
    OOMB_METHOD("vote_topk", from_means<oomb_page_vote_topk>),
    OOMB_METHOD("attn_fwd", attn_fwd<false>),
    OOMB_METHOD("attn_fwd_qp", attn_fwd<true>),
    OOMB_METHOD("attn_bwd", attn_bwd<false>),
    OOMB_METHOD("attn_bwd_qp", attn_bwd<true>),
    OOMB_METHOD("kv_append", kv_append),
    OOMB_METHOD("local_page_list", local_page_list),
    OOMB_METHOD("make_rows_desc", make_rows_desc),
    OOMB_METHOD("kv_append_rope", append_rope<false>),
    OOMB_METHOD("kvq_append_rope", append_rope<true>),
    OOMB_METHOD("kv_append_rope_bwd", append_rope_bwd),
    OOMB_METHOD("kvq_read", kvq_read),
    OOMB_METHOD("attn_fwd_kvq", attn_fwd_kvq),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
  PyObject* c = PyImport_ImportModule("torch._C");
  if (!c) return nullptr;
  g_raw_stream = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
  Py_DECREF(c);
  return g_raw_stream ? PyModule_Create(&module) : nullptr;
}
