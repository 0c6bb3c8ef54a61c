// Python binding of the serving operators (module _serve): the host side of lsa_cache_append, lsa_norm_append, lsa_cache_read,
// lsa_prefill_attn, lsa_chunk_attn and lsa_decode_attn for torch tensors.
//
// A decode step's kernels take 3 to 20 us, as long as a host in Python that looks at a dozen tensors, so the
// checks that a good call passes, its allocations and the call itself are compiled. What is not as it should be is not explained
// here: the functions return None, also where the library refuses, and lsa.py says why. An error of the HIP runtime is
// raised here (by `check`, a function that lsa.py gives this module), since the call may have run in part. us of a call that the
// host bounds, with the checks in Python and here: append of one token 12.0, 7.4, of which the launch takes 3.2;
// 1001 rows of a cache read back 15.3, 6.2.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "lsa.h"

namespace {

PyObject* raw_stream = nullptr;  // torch._C._cuda_getCurrentRawStream

constexpr const char* kAppendNames[] = {"n_heads", "n_kv_heads", "d_k", "d_v", "rot_start", "rot_dim", "interleaved", "fp8"};
constexpr const char* kAttnNames[] = {"n_heads", "n_kv_heads", "d_qk", "d_v", "latent", "fp8", "k_sink", "k_swa"};
constexpr const char* kReadNames[] = {"n_kv_heads", "d_k", "d_v", "fp8"};
constexpr const char* kPrefillNames[] = {"n_heads", "n_kv_heads", "d_qk", "d_v", "causal", "k_sink", "k_swa"};
PyObject *append_names[8], *attn_names[8], *read_names[4], *prefill_names[7], *sm_scale_name;

// (bools are ints; anything else that is no int of 32 bits is refused)
bool to_int(PyObject* o, int32_t& x) {
  int over = 0;
  const long v = PyLong_AsLongAndOverflow(o, &over);
  if ((v == -1 && PyErr_Occurred()) || over != 0 || v != (int32_t)v) {
    PyErr_Clear();
    return false;
  }
  x = (int32_t)v;
  return true;
}
bool int_attr(PyObject* o, PyObject* name, int32_t& x) {
  PyObject* a = PyObject_GetAttr(o, name);
  if (a == nullptr) {
    PyErr_Clear();
    return false;
  }
  const bool ok = to_int(a, x);
  Py_DECREF(a);
  return ok;
}

// The softmax scale of an attention's parameters; false where it is no number.
bool scale_attr(PyObject* o, float& x) {
  PyObject* scale = PyObject_GetAttr(o, sm_scale_name);
  const double v = scale == nullptr ? -1.0 : PyFloat_AsDouble(scale);
  Py_XDECREF(scale);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  x = (float)v;
  return true;
}

// The tensors of a call, all on one GPU.
struct Tensors {
  c10::DeviceIndex device = -1;
  bool ok = true;

  // nullptr where `o` is None; otherwise a tensor on the call's GPU, or ok = false
  const at::Tensor* get(PyObject* o) {
    if (!ok || o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) return fail();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) return fail();
    if (device < 0) device = t.get_device();
    return t.get_device() == device ? &t : fail();
  }
  const at::Tensor* fail() {
    ok = false;
    return nullptr;
  }
  void need(bool b) { ok = ok && b; }

  // contiguous, of one type and shape; nullptr where `o` is None, which is refused unless `optional`
  const at::Tensor* whole(PyObject* o, at::ScalarType type, at::IntArrayRef shape, bool optional = false) {
    const at::Tensor* t = get(o);
    if (t == nullptr) {
      need(optional);
      return nullptr;
    }
    need(t->scalar_type() == type && t->sizes() == shape && t->is_contiguous());
    return t;
  }
  // [n, heads, width] bf16 whose tokens lie `stride` apart, the heads of one after the other
  const at::Tensor* tokens(PyObject* o, int64_t n, int64_t heads, int64_t width, int64_t& stride) {
    const at::Tensor* t = get(o);
    if (t == nullptr) return fail();
    need(t->scalar_type() == at::kBFloat16 && t->dim() == 3 && t->size(0) == n && t->size(1) == heads && t->size(2) == width);
    if (!ok) return nullptr;
    need((t->stride(2) == 1 || width <= 1) && (t->stride(1) == width || heads <= 1));
    stride = n > 1 ? t->stride(0) : heads * width;
    return t;
  }
  // a cache [n_phys, heads, page, width], or without the head dimension when there is one head; n_phys < 0: any
  const at::Tensor* cache(PyObject* o, bool fp8, int64_t heads, int64_t width, int64_t& n_phys, int64_t& page) {
    const at::Tensor* t = get(o);
    if (t == nullptr) return fail();
    const auto type = t->scalar_type();
    need(fp8 ? type == at::kByte || type == at::kFloat8_e4m3fn : type == at::kBFloat16);
    const int64_t dim = t->dim();
    need((dim == 4 && t->size(1) == heads) || (dim == 3 && heads == 1));
    if (!ok) return nullptr;
    need(t->size(dim - 1) == width && t->is_contiguous() && (n_phys < 0 || (t->size(0) == n_phys && t->size(dim - 2) == page)));
    n_phys = t->size(0);
    page = t->size(dim - 2);
    return t;
  }
  // scales [n_phys, heads, page] or [n_phys, page], exactly for fp8 caches
  const at::Tensor* scales(PyObject* o, bool given, int64_t n_phys, int64_t heads, int64_t page) {
    const at::Tensor* t = get(o);
    need(given == (t != nullptr));
    if (!ok || t == nullptr) return nullptr;
    need(t->scalar_type() == at::kFloat && t->is_contiguous() &&
         (t->sizes() == at::IntArrayRef({n_phys, heads, page}) || (heads == 1 && t->sizes() == at::IntArrayRef({n_phys, page}))));
    return t;
  }
  // offsets [n_seq + 1] of sequences
  const at::Tensor* offsets(PyObject* o, int64_t& n_seq) {
    const at::Tensor* t = get(o);
    if (t == nullptr) return fail();
    need(t->scalar_type() == at::kInt && t->dim() == 1 && t->is_contiguous());
    if (!ok) return nullptr;
    n_seq = t->size(0) - 1;
    need(n_seq >= 0 && n_seq <= INT32_MAX);
    return t;
  }
  // A page table [n_seq, max_pages]
  const at::Tensor* table(PyObject* o, int32_t& max_pages) {
    const at::Tensor* t = get(o);
    max_pages = 1;
    if (t == nullptr) return nullptr;
    need(t->scalar_type() == at::kInt && t->dim() == 2 && t->is_contiguous());
    if (!ok) return nullptr;
    need(t->size(1) <= INT32_MAX);
    max_pages = (int32_t)t->size(1);
    return t;
  }
};

struct Unlocked {  // other threads may run while one allocates and launches
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

template <class T = void>
T* at_of(const at::Tensor* t) {
  return t == nullptr ? nullptr : static_cast<T*>(t->data_ptr());
}

// The current stream of the call's GPU; false with a Python error set.
bool stream_of(c10::DeviceIndex device, void*& stream) {
  PyObject* index = PyLong_FromLong(device);
  if (index == nullptr) return false;
  PyObject* s = PyObject_CallOneArg(raw_stream, index);
  Py_DECREF(index);
  if (s == nullptr) return false;
  stream = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  return !PyErr_Occurred();
}

PyObject* tuple_of(std::initializer_list<const at::Tensor*> ts) {
  PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
  Py_ssize_t i = 0;
  for (const at::Tensor* t : ts) {
    PyObject* o = r == nullptr ? nullptr : t == nullptr ? Py_NewRef(Py_None) : THPVariable_Wrap(*t);
    if (o == nullptr) {
      Py_XDECREF(r);
      return nullptr;
    }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

// What becomes of a call that the library did not do. Refusals come before its first launch and are left to lsa.py; after an
// error of the runtime nothing is tried again: an append that rotates queries in place would rotate them twice.
PyObject* not_done(PyObject* module, lsa_status st, const char* call) {
  if (st != LSA_ERR_HIP) Py_RETURN_NONE;
  PyObject* r = PyObject_CallMethod(module, "check", "is", (int)st, call);
  if (r != nullptr) {
    Py_DECREF(r);
    PyErr_Format(PyExc_RuntimeError, "%s: status %d", call, (int)st);
  }
  return nullptr;
}

// cache_append(prm, k, k_cache, page_table, ctx_len, pos, seq, rows_per_seq, n_seq, rope, k_rot, v, v_cache, k_scale, v_scale,
//              q, q_rot, q_out, rows), and with NORM as norm_append(.., q_weight, k_weight, eps, k_out)
template <bool NORM>
PyObject* append(PyObject* module, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != (NORM ? 23 : 19)) Py_RETURN_NONE;
  int32_t p[8], rows_per_seq, max_pages;
  for (int i = 0; i < 8; ++i)
    if (!int_attr(a[0], append_names[i], p[i])) Py_RETURN_NONE;
  if (!to_int(a[7], rows_per_seq)) Py_RETURN_NONE;
  const int64_t nq = p[0], nk = p[1], d_k = p[2], d_v = p[3], rot = p[5];
  const bool fp8 = p[7] != 0;
  lsa_append_params prm{p[0], p[1], p[2], p[3], p[4], p[5], p[6], fp8 ? LSA_KEY_FP8_E4M3FN : LSA_KEY_BF16};
  lsa_append_tensors x{};
  Tensors ts;
  const at::Tensor* k = ts.get(a[1]);
  if (k == nullptr || k->dim() != 3) Py_RETURN_NONE;
  const int64_t n = k->size(0);
  int64_t n_phys = -1, page = 0;
  ts.tokens(a[1], n, nk, a[10] == Py_None ? d_k : d_k - rot, x.k_stride);
  x.k_rot = a[10] == Py_None ? nullptr : at_of(ts.tokens(a[10], n, nk, rot, x.k_rot_stride));
  x.k_cache = at_of(ts.cache(a[2], fp8, nk, d_k, n_phys, page));
  ts.need((d_v != 0) == (a[11] != Py_None) && (d_v != 0) == (a[12] != Py_None) && (nq != 0) == (a[15] != Py_None));
  if (!ts.ok) Py_RETURN_NONE;
  if (d_v != 0) {
    x.v = at_of(ts.tokens(a[11], n, nk, d_v, x.v_stride));
    x.v_cache = at_of(ts.cache(a[12], fp8, nk, d_v, n_phys, page));
  }
  x.k_scale = at_of<float>(ts.scales(a[13], fp8, n_phys, nk, page));
  x.v_scale = at_of<float>(ts.scales(a[14], fp8 && d_v != 0, n_phys, nk, page));
  const at::Tensor* q_out = nullptr;
  if (nq != 0) {
    x.q = at_of(ts.tokens(a[15], n, nq, a[16] == Py_None ? d_k : d_k - rot, x.q_stride));
    x.q_rot = a[16] == Py_None ? nullptr : at_of(ts.tokens(a[16], n, nq, rot, x.q_rot_stride));
    q_out = ts.whole(a[17], at::kBFloat16, {n, nq, d_k}, true);
  } else {
    ts.need(a[16] == Py_None && a[17] == Py_None);
  }
  const at::Tensor* rope = ts.get(a[9]);
  ts.need((rot != 0) == (rope != nullptr));
  if (!ts.ok) Py_RETURN_NONE;
  if (rope != nullptr) {
    ts.need(rope->scalar_type() == at::kFloat && rope->dim() == 2 && rope->is_contiguous());
    if (!ts.ok) Py_RETURN_NONE;
    ts.need(rope->size(1) == rot);
    x.rope = at_of<float>(rope);
    x.rope_rows = rope->size(0);
  }
  lsa_append_norm norm{};
  const at::Tensor* k_out = nullptr;
  if constexpr (NORM) {
    norm.q_weight = at_of(ts.whole(a[19], at::kBFloat16, {a[16] == Py_None ? d_k : d_k - rot}, true));
    norm.k_weight = at_of(ts.whole(a[20], at::kBFloat16, {a[10] == Py_None ? d_k : d_k - rot}, true));
    const double eps = PyFloat_AsDouble(a[21]);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    norm.eps = (float)eps;
    k_out = a[22] == Py_True || a[22] == Py_False ? nullptr : ts.whole(a[22], at::kBFloat16, {n, nk, d_k}, true);
  }
  // the tokens' places
  const at::Tensor *table = ts.table(a[3], max_pages), *ctx_len = ts.get(a[4]);
  ts.need((a[4] == Py_None) != (a[5] == Py_None) && (ctx_len == nullptr || ctx_len->dim() == 1));
  if (!ts.ok) Py_RETURN_NONE;
  int64_t seqs = table != nullptr ? table->size(0) : ctx_len != nullptr ? ctx_len->size(0) : n_phys;
  if (a[8] != Py_None) {
    int32_t n_seq;
    if (!to_int(a[8], n_seq) || (n_seq != seqs && (table != nullptr || ctx_len != nullptr || n_seq < 0 || n_seq > seqs))) Py_RETURN_NONE;
    seqs = n_seq;
  }
  if (ctx_len != nullptr) {
    ts.whole(a[4], at::kInt, {seqs});
    ts.need(a[6] == Py_None && n == seqs * rows_per_seq);
  } else {
    x.pos = at_of<int32_t>(ts.whole(a[5], at::kInt, {n}));
    x.seq = at_of<int32_t>(ts.whole(a[6], at::kInt, {n}, true));
  }
  const at::Tensor* rows = a[18] == Py_True || a[18] == Py_False ? nullptr : ts.whole(a[18], at::kLong, {n}, true);
  ts.need(seqs <= INT32_MAX && page <= INT32_MAX);
  if (!ts.ok) Py_RETURN_NONE;
  x.k = at_of(k);
  x.page_table = at_of<int32_t>(table);
  x.ctx_len = at_of<int32_t>(ctx_len);
  const c10::DeviceGuard guard(c10::Device(c10::kCUDA, ts.device));  // (stream 0 is that of whichever GPU is current)
  void* stream;
  if (!stream_of(ts.device, stream)) return nullptr;
  lsa_status st;
  at::Tensor new_q, new_rows, new_k;
  {
    Unlocked unlocked;
    if (nq != 0 && q_out == nullptr) {
      new_q = at::empty({n, nq, d_k}, k->options());
      q_out = &new_q;
    }
    if (a[18] == Py_True) {
      new_rows = at::empty({n}, k->options().dtype(at::kLong));
      rows = &new_rows;
    }
    x.q_out = at_of(q_out);
    x.rows = at_of<int64_t>(rows);
    if constexpr (NORM) {
      if (a[22] == Py_True) {
        new_k = at::empty({n, nk, d_k}, k->options());
        k_out = &new_k;
      }
      norm.k_out = at_of(k_out);
      st = lsa_norm_append(&prm, &norm, &x, n, (int32_t)seqs, rows_per_seq, max_pages, (int32_t)page, n_phys, stream);
    } else {
      st = lsa_cache_append(&prm, &x, n, (int32_t)seqs, rows_per_seq, max_pages, (int32_t)page, n_phys, stream);
    }
  }
  if (st != LSA_OK) return not_done(module, st, NORM ? "lsa_norm_append" : "lsa_cache_append");
  return NORM ? tuple_of({q_out, k_out, rows}) : tuple_of({q_out, rows});
  END_HANDLE_TH_ERRORS
}

// decode_attn(prm, q, k_cache, v_cache, ctx_len, page_table, rows_per_seq, k_scale, v_scale, out, lse, workspace)
PyObject* decode_attn(PyObject* module, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 12) Py_RETURN_NONE;
  int32_t p[8], rows_per_seq, max_pages;
  for (int i = 0; i < 8; ++i)
    if (!int_attr(a[0], attn_names[i], p[i])) Py_RETURN_NONE;
  float sm_scale;
  if (!scale_attr(a[0], sm_scale) || !to_int(a[6], rows_per_seq)) Py_RETURN_NONE;
  const int64_t H = p[0], nk = p[1], d_qk = p[2], d_v = p[3];
  const bool latent = p[4] != 0, fp8 = p[5] != 0;
  lsa_decode_attn_params prm{p[0], p[1], p[2], p[3], p[4], fp8 ? LSA_KEY_FP8_E4M3FN : LSA_KEY_BF16, p[6], p[7], sm_scale};
  Tensors ts;
  const at::Tensor* q = ts.get(a[1]);
  if (q == nullptr || q->dim() != 3) Py_RETURN_NONE;
  const int64_t n = q->size(0);
  ts.whole(a[1], at::kBFloat16, {n, H, d_qk});
  int64_t n_phys = -1, page = 0;
  const at::Tensor* k = ts.cache(a[2], fp8, nk, d_qk, n_phys, page);
  ts.need(latent == (a[3] == Py_None));
  if (!ts.ok) Py_RETURN_NONE;
  const at::Tensor* v = latent ? nullptr : ts.cache(a[3], fp8, nk, d_v, n_phys, page);
  const at::Tensor* k_scale = ts.scales(a[7], fp8, n_phys, nk, page);
  const at::Tensor* v_scale = ts.scales(a[8], fp8 && !latent, n_phys, nk, page);
  const at::Tensor* ctx_len = ts.get(a[4]);
  if (ctx_len == nullptr || ctx_len->dim() != 1) Py_RETURN_NONE;
  const int64_t n_seq = ctx_len->size(0);
  ts.whole(a[4], at::kInt, {n_seq});
  const at::Tensor* table = ts.table(a[5], max_pages);
  ts.need(n == n_seq * rows_per_seq && (table == nullptr || table->size(0) == n_seq) && n_seq <= INT32_MAX && page <= INT32_MAX);
  const at::Tensor* out = ts.whole(a[9], at::kBFloat16, {n, H, d_v}, true);
  const at::Tensor* lse = a[10] == Py_True || a[10] == Py_False ? nullptr : ts.whole(a[10], at::kFloat, {n, H}, true);
  const at::Tensor* workspace = ts.get(a[11]);
  ts.need(workspace == nullptr || workspace->is_contiguous());
  if (!ts.ok) Py_RETURN_NONE;
  const c10::DeviceGuard guard(c10::Device(c10::kCUDA, ts.device));  // (stream 0 is that of whichever GPU is current)
  void* stream;
  if (!stream_of(ts.device, stream)) return nullptr;
  lsa_status st;
  at::Tensor new_out, new_lse, new_workspace;
  {
    Unlocked unlocked;
    const size_t need = lsa_decode_attn_workspace_size(&prm, (int32_t)n_seq, rows_per_seq, max_pages, (int32_t)page);
    if (out == nullptr) {
      new_out = at::empty({n, H, d_v}, q->options());
      out = &new_out;
    }
    if (a[10] == Py_True) {
      new_lse = at::empty({n, H}, q->options().dtype(at::kFloat));
      lse = &new_lse;
    }
    if (need == 0) {
      workspace = nullptr;
    } else if (workspace == nullptr) {
      new_workspace = at::empty({(int64_t)need}, q->options().dtype(at::kByte));
      workspace = &new_workspace;
    }
    st = lsa_decode_attn(&prm, (int32_t)n_seq, rows_per_seq, at_of(q), at_of(k), at_of<float>(k_scale), at_of(v), at_of<float>(v_scale),
                         at_of<int32_t>(ctx_len), at_of<int32_t>(table), max_pages, (int32_t)page, n_phys, at_of(out), at_of<float>(lse),
                         at_of(workspace), workspace == nullptr ? 0 : workspace->nbytes(), stream);
  }
  if (st != LSA_OK) return not_done(module, st, "lsa_decode_attn");
  return tuple_of({out, lse});
  END_HANDLE_TH_ERRORS
}

// cache_read(prm, k_cache, cu, n_tok, page_table, start, v_cache, k_scale, v_scale, k_out, v_out)
PyObject* cache_read(PyObject* module, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 11) Py_RETURN_NONE;
  int32_t p[4], n, max_pages;
  for (int i = 0; i < 4; ++i)
    if (!int_attr(a[0], read_names[i], p[i])) Py_RETURN_NONE;
  if (!to_int(a[3], n) || n < 0) Py_RETURN_NONE;
  const int64_t nk = p[0], d_k = p[1], d_v = p[2];
  const bool fp8 = p[3] != 0, values = d_v != 0;
  lsa_cache_read_params prm{p[0], p[1], p[2], fp8 ? LSA_KEY_FP8_E4M3FN : LSA_KEY_BF16};
  Tensors ts;
  int64_t n_phys = -1, page = 0, n_seq = 0;
  const at::Tensor* k = ts.cache(a[1], fp8, nk, d_k, n_phys, page);
  ts.need(values == (a[6] != Py_None) && (values || a[10] == Py_None));
  if (!ts.ok) Py_RETURN_NONE;
  const at::Tensor* v = values ? ts.cache(a[6], fp8, nk, d_v, n_phys, page) : nullptr;
  const at::Tensor* k_scale = ts.scales(a[7], fp8, n_phys, nk, page);
  const at::Tensor* v_scale = ts.scales(a[8], fp8 && values, n_phys, nk, page);
  const at::Tensor* cu = ts.offsets(a[2], n_seq);
  if (!ts.ok) Py_RETURN_NONE;
  const at::Tensor* start = ts.whole(a[5], at::kInt, {n_seq}, true);
  const at::Tensor* table = ts.table(a[4], max_pages);
  ts.need((table == nullptr || table->size(0) == n_seq) && page <= INT32_MAX);
  const at::Tensor* k_out = ts.whole(a[9], at::kBFloat16, {n, nk, d_k}, true);
  const at::Tensor* v_out = values ? ts.whole(a[10], at::kBFloat16, {n, nk, d_v}, true) : nullptr;
  if (!ts.ok) Py_RETURN_NONE;
  const c10::DeviceGuard guard(c10::Device(c10::kCUDA, ts.device));
  void* stream;
  if (!stream_of(ts.device, stream)) return nullptr;
  lsa_status st;
  at::Tensor new_k, new_v;
  {
    Unlocked unlocked;
    const auto options = k->options().dtype(at::kBFloat16);
    if (k_out == nullptr) {
      new_k = at::empty({n, nk, d_k}, options);
      k_out = &new_k;
    }
    if (values && v_out == nullptr) {
      new_v = at::empty({n, nk, d_v}, options);
      v_out = &new_v;
    }
    st = lsa_cache_read(&prm, n, (int32_t)n_seq, at_of(k), at_of<float>(k_scale), at_of(v), at_of<float>(v_scale), at_of<int32_t>(cu),
                        at_of<int32_t>(start), at_of<int32_t>(table), max_pages, (int32_t)page, n_phys, at_of(k_out), at_of(v_out), stream);
  }
  if (st != LSA_OK) return not_done(module, st, "lsa_cache_read");
  return tuple_of({k_out, v_out});
  END_HANDLE_TH_ERRORS
}

// What the attentions of prompts and chunks return and work in: `out`, `lse` (None, True, False or a tensor) and `workspace` as they are given.
struct Outputs {
  const at::Tensor *out, *lse, *workspace;
  at::Tensor made[3];
  Outputs(Tensors& ts, PyObject* o, PyObject* l, PyObject* w, int64_t n, int64_t H, int64_t d_v) {
    out = ts.whole(o, at::kBFloat16, {n, H, d_v}, true);
    lse = l == Py_True || l == Py_False ? nullptr : ts.whole(l, at::kFloat, {n, H}, true);
    workspace = ts.get(w);
    ts.need(workspace == nullptr || workspace->is_contiguous());
  }
  void make(const at::Tensor* q, bool want_lse, size_t need, int64_t n, int64_t H, int64_t d_v) {
    if (out == nullptr) out = &(made[0] = at::empty({n, H, d_v}, q->options()));
    if (want_lse) lse = &(made[1] = at::empty({n, H}, q->options().dtype(at::kFloat)));
    if (need == 0) workspace = nullptr;
    else if (workspace == nullptr) workspace = &(made[2] = at::empty({(int64_t)need}, q->options().dtype(at::kByte)));
  }
};

// prefill_attn(prm, q, k, v, cu_q, cu_kv, out, lse, workspace)
PyObject* prefill_attn(PyObject* module, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 9) Py_RETURN_NONE;
  lsa_prefill_attn_params prm{};
  int32_t p[7];
  for (int i = 0; i < 7; ++i)
    if (!int_attr(a[0], prefill_names[i], p[i])) Py_RETURN_NONE;
  if (!scale_attr(a[0], prm.sm_scale)) Py_RETURN_NONE;
  prm = lsa_prefill_attn_params{p[0], p[1], p[2], p[3], p[4], p[5], p[6], prm.sm_scale};
  const int64_t H = p[0], nk = p[1], d_qk = p[2], d_v = p[3];
  Tensors ts;
  const at::Tensor *q = ts.get(a[1]), *k = ts.get(a[2]), *v = ts.get(a[3]);
  if (q == nullptr || k == nullptr || v == nullptr || q->dim() != 3 || k->dim() != 3) Py_RETURN_NONE;
  const int64_t n = q->size(0), n_kv = k->size(0);
  int64_t qs = 0, ks = 0, vs = 0, n_seq = 0;
  ts.tokens(a[1], n, H, d_qk, qs);
  ts.tokens(a[2], n_kv, nk, d_qk, ks);
  ts.tokens(a[3], n_kv, nk, d_v, vs);
  const at::Tensor* cu_q = ts.offsets(a[4], n_seq);
  if (!ts.ok) Py_RETURN_NONE;
  const at::Tensor* cu_kv = ts.whole(a[5], at::kInt, {n_seq + 1}, true);
  ts.need(cu_kv != nullptr || n_kv == n);
  Outputs y(ts, a[6], a[7], a[8], n, H, d_v);
  if (!ts.ok) Py_RETURN_NONE;
  const c10::DeviceGuard guard(c10::Device(c10::kCUDA, ts.device));
  void* stream;
  if (!stream_of(ts.device, stream)) return nullptr;
  lsa_status st;
  {
    Unlocked unlocked;
    y.make(q, a[7] == Py_True, lsa_prefill_attn_workspace_size(&prm, (int32_t)n_seq, n, n_kv), n, H, d_v);
    st = lsa_prefill_attn(&prm, (int32_t)n_seq, n, n_kv, at_of(q), qs, at_of(k), ks, at_of(v), vs, at_of<int32_t>(cu_q), at_of<int32_t>(cu_kv),
                          at_of(y.out), at_of<float>(y.lse), at_of(y.workspace), y.workspace == nullptr ? 0 : y.workspace->nbytes(), stream);
  }
  if (st != LSA_OK) return not_done(module, st, "lsa_prefill_attn");
  return tuple_of({y.out, y.lse});
  END_HANDLE_TH_ERRORS
}

// chunk_attn(prm, q, k_cache, v_cache, cu_q, ctx_len, page_table, k_scale, v_scale, out, lse, workspace)
PyObject* chunk_attn(PyObject* module, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 12) Py_RETURN_NONE;
  int32_t p[8], max_pages;
  float sm_scale;
  for (int i = 0; i < 8; ++i)
    if (!int_attr(a[0], attn_names[i], p[i])) Py_RETURN_NONE;
  if (!scale_attr(a[0], sm_scale)) Py_RETURN_NONE;
  const int64_t H = p[0], nk = p[1], d_qk = p[2], d_v = p[3];
  const bool fp8 = p[5] != 0;
  lsa_decode_attn_params prm{p[0], p[1], p[2], p[3], p[4], fp8 ? LSA_KEY_FP8_E4M3FN : LSA_KEY_BF16, p[6], p[7], sm_scale};
  Tensors ts;
  const at::Tensor* q = ts.get(a[1]);
  if (q == nullptr || q->dim() != 3) Py_RETURN_NONE;
  const int64_t n = q->size(0);
  ts.whole(a[1], at::kBFloat16, {n, H, d_qk});
  int64_t n_phys = -1, page = 0, n_seq = 0;
  const at::Tensor* k = ts.cache(a[2], fp8, nk, d_qk, n_phys, page);
  if (!ts.ok) Py_RETURN_NONE;
  const at::Tensor* v = ts.cache(a[3], fp8, nk, d_v, n_phys, page);
  const at::Tensor* k_scale = ts.scales(a[7], fp8, n_phys, nk, page);
  const at::Tensor* v_scale = ts.scales(a[8], fp8, n_phys, nk, page);
  const at::Tensor* cu_q = ts.offsets(a[4], n_seq);
  if (!ts.ok) Py_RETURN_NONE;
  const at::Tensor* ctx_len = ts.whole(a[5], at::kInt, {n_seq});
  const at::Tensor* table = ts.table(a[6], max_pages);
  ts.need((table == nullptr || table->size(0) == n_seq) && page <= INT32_MAX);
  Outputs y(ts, a[9], a[10], a[11], n, H, d_v);
  if (!ts.ok) Py_RETURN_NONE;
  const c10::DeviceGuard guard(c10::Device(c10::kCUDA, ts.device));
  void* stream;
  if (!stream_of(ts.device, stream)) return nullptr;
  lsa_status st;
  {
    Unlocked unlocked;
    y.make(q, a[10] == Py_True, lsa_chunk_attn_workspace_size(&prm, (int32_t)n_seq, n, max_pages, (int32_t)page), n, H, d_v);
    st = lsa_chunk_attn(&prm, (int32_t)n_seq, n, at_of(q), at_of(k), at_of<float>(k_scale), at_of(v), at_of<float>(v_scale), at_of<int32_t>(cu_q),
                        at_of<int32_t>(ctx_len), at_of<int32_t>(table), max_pages, (int32_t)page, n_phys, at_of(y.out), at_of<float>(y.lse),
                        at_of(y.workspace), y.workspace == nullptr ? 0 : y.workspace->nbytes(), stream);
  }
  if (st != LSA_OK) return not_done(module, st, "lsa_chunk_attn");
  return tuple_of({y.out, y.lse});
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"cache_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append<false>)), METH_FASTCALL, nullptr},
    {"norm_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(append<true>)), METH_FASTCALL, nullptr},
    {"cache_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cache_read)), METH_FASTCALL, nullptr},
    {"prefill_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(prefill_attn)), METH_FASTCALL, nullptr},
    {"chunk_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(chunk_attn)), METH_FASTCALL, nullptr},
    {"decode_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode_attn)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef definition = {PyModuleDef_HEAD_INIT, "_serve", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serve() {
  PyObject* c = PyImport_ImportModule("torch._C");
  if (c == nullptr) return nullptr;
  raw_stream = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
  Py_DECREF(c);
  if (raw_stream == nullptr) return nullptr;
  auto intern = [](PyObject** to, const char* const* names, int n) {
    for (int i = 0; i < n; ++i)
      if ((to[i] = PyUnicode_InternFromString(names[i])) == nullptr) return false;
    return true;
  };
  if (!intern(append_names, kAppendNames, 8) || !intern(attn_names, kAttnNames, 8) || !intern(read_names, kReadNames, 4) ||
      !intern(prefill_names, kPrefillNames, 7))
    return nullptr;
  if ((sm_scale_name = PyUnicode_InternFromString("sm_scale")) == nullptr) return nullptr;
  return PyModule_Create(&definition);
}
