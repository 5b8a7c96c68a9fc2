// Marshals the arguments of the operators on bounded, shared and paged caches and of the log probabilities: torch tensors in, the C
// entry points of include/lazyllm.h out, their status back.  It does what the ctypes layer does for the other calls (checks of types, sizes and
// devices, addresses, pitches) in one call from Python: with a dozen tensors per operator and a few microseconds of device
// time, checking them one by one in Python costs more than the operator (14.8 us a call for the step, 9.7 for the verification).
// No arithmetic, no state but the entry points' addresses.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include "lazyllm.h"

namespace {

struct Fail {};  // a Python error is set

[[noreturn]] void fail(const char *name, const char *what) {
  PyErr_Format(PyExc_ValueError, "%s: %s", name, what);
  throw Fail();
}

// For the handlers: no C++ exception leaves an entry point.
PyObject *raised() {
  try {
    throw;
  } catch (const Fail &) {
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

// What one call's arguments have in common.
struct Call {
  PyObject *const *args;
  Py_ssize_t n, next = 0;
  int64_t device = 0;
  void *stream = nullptr;

  Call(PyObject *const *args, Py_ssize_t n, Py_ssize_t want) : args(args), n(n) {
    if (n != want) {
      PyErr_Format(PyExc_TypeError, "%zd arguments are wanted, got %zd", want, n);
      throw Fail();
    }
    device = integer("device");
    stream = reinterpret_cast<void *>(static_cast<intptr_t>(integer("stream")));
  }
  int64_t integer(const char *name) {
    const long long v = PyLong_AsLongLong(args[next++]);
    if (v == -1 && PyErr_Occurred()) throw Fail();
    (void)name;
    return v;
  }
  int32_t int32(const char *name) {
    const int64_t v = integer(name);
    if (v < INT32_MIN || v > INT32_MAX) fail(name, "does not fit 32 bits");
    return static_cast<int32_t>(v);
  }
  const at::Tensor &tensor(const char *name) {
    PyObject *o = args[next++];
    if (!THPVariable_Check(o)) {
      PyErr_Format(PyExc_TypeError, "%s: a tensor is wanted", name);
      throw Fail();
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device) fail(name, "a tensor on the current CUDA device is wanted");
    return t;
  }
  bool none() { return args[next] == Py_None ? (++next, true) : false; }
  // A contiguous tensor of a type and a number of elements (-1: any).
  template <typename T>
  T *dense(const char *name, at::ScalarType type, int64_t count, int64_t *got = nullptr) {
    const at::Tensor &t = tensor(name);
    if (t.scalar_type() != type) fail(name, "another element type is wanted");
    if (!t.is_contiguous()) fail(name, "a contiguous tensor is wanted");
    if (count >= 0 && t.numel() != count) fail(name, "its size does not agree with the other arguments");
    if (got) *got = t.numel();
    return static_cast<T *>(t.data_ptr());
  }
  // A matrix of rows of `width` elements, each contiguous: its address, rows and pitch.
  void *rows(const char *name, at::ScalarType type, int64_t width, int64_t *count, int32_t *pitch) {
    const at::Tensor &t = tensor(name);
    if (t.scalar_type() != type) fail(name, "another element type is wanted");
    if (t.dim() != 2 || t.size(1) != width || (t.size(0) > 0 && width > 1 && t.stride(1) != 1))
      fail(name, "contiguous rows of another width are wanted");
    const int64_t p = t.size(0) > 1 ? t.stride(0) : width;
    if (p < width || p > INT32_MAX) fail(name, "rows overlap or lie too far apart");
    *count = t.size(0);
    *pitch = static_cast<int32_t>(p);
    return t.data_ptr();
  }
};

int32_t fits(int64_t v, const char *name) {
  if (v > INT32_MAX) fail(name, "too large");
  return static_cast<int32_t>(v);
}
int32_t code_of(at::ScalarType t) {
  if (t == at::kBFloat16) return LAZY_BF16;
  if (t == at::kFloat) return LAZY_F32;
  fail("dtype", "bfloat16 or float32 is wanted");
}
at::ScalarType type_of(PyObject *o) {
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, "a tensor is wanted");
    throw Fail();
  }
  return THPVariable_Unpack(o).scalar_type();
}

decltype(&lazy_k_attention_mass) f_mass;
decltype(&lazy_k_evict) f_evict;
decltype(&lazy_k_evict_step) f_step;
decltype(&lazy_k_attention_prefix) f_prefix;
decltype(&lazy_k_verify) f_verify;
decltype(&lazy_k_paged_append) f_append;
decltype(&lazy_k_attention_paged) f_paged;
decltype(&lazy_k_token_logprobs) f_logprobs;

// Caches [n_seqs, cap, n_kv_heads, head_dim].
struct Cache {
  void *k, *v;
  int64_t n_seqs, cap, heads, dim;
  Cache(Call &c, at::ScalarType type) {
    const at::Tensor &t = THPVariable_Check(c.args[c.next]) ? THPVariable_Unpack(c.args[c.next]) : c.tensor("kc");
    if (t.dim() != 4) fail("kc", "[n_seqs, cap, n_kv_heads, head_dim] is wanted");
    n_seqs = t.size(0), cap = t.size(1), heads = t.size(2), dim = t.size(3);
    k = c.dense<void>("kc", type, t.numel());
    v = c.dense<void>("vc", type, t.numel());
  }
};

// Pages [n_pages, page_size, n_kv_heads, head_dim] of k and v with equal strides, then the table and the lengths: four arguments.
struct Pages : lazy_pages {
  int64_t heads = 0, dim = 0, n_seqs = 0;
  Pages(Call &c, at::ScalarType type) {
    const at::Tensor &tk = c.tensor("k_pages"), &tv = c.tensor("v_pages");
    if (tk.scalar_type() != type || tv.scalar_type() != type) fail("k_pages, v_pages", "the type of the rows is wanted");
    if (tk.dim() != 4 || tk.sizes() != tv.sizes()) fail("k_pages, v_pages", "[n_pages, page_size, n_kv_heads, head_dim] is wanted");
    if (tk.strides() != tv.strides() || (tk.numel() > 0 && tk.size(3) > 1 && tk.stride(3) != 1))
      fail("k_pages, v_pages", "equal strides and contiguous heads are wanted");
    heads = tk.size(2), dim = tk.size(3);
    k = tk.data_ptr(), v = tv.data_ptr();
    // a stride that is never used may be anything
    page_stride = tk.size(0) > 1 ? tk.stride(0) : 0;
    slot_stride = tk.size(1) > 1 ? tk.stride(1) : 0;
    head_stride = tk.size(2) > 1 ? tk.stride(2) : 0;
    n_pages = fits(tk.size(0), "k_pages"), page_size = fits(tk.size(1), "k_pages");
    const at::Tensor &t = c.tensor("page_table");
    if (t.scalar_type() != at::kInt || t.dim() != 2 || (t.numel() > 0 && t.size(1) > 1 && t.stride(1) != 1))
      fail("page_table", "int32 [n_seqs, pages] with contiguous rows is wanted");
    n_seqs = t.size(0);
    table_pages = fits(t.size(1), "page_table");
    ld_table = t.size(0) > 1 ? fits(t.stride(0), "page_table") : table_pages;
    table = static_cast<int32_t *>(t.data_ptr());
    len = c.dense<int32_t>("kv_len", at::kInt, n_seqs);
  }
};

// (device, stream, q, k, cu_seqlens, scratch, out, max_len, n_heads, n_kv_heads, head_dim, window)
PyObject *attention_mass(PyObject *, PyObject *const *args, Py_ssize_t n) try {
  Call c(args, n, 12);
  const at::ScalarType type = type_of(args[2]);
  const int64_t H = PyLong_AsLongLong(args[8]), Hkv = PyLong_AsLongLong(args[9]), dh = PyLong_AsLongLong(args[10]);
  if (PyErr_Occurred()) throw Fail();
  int64_t nq, nk, seqs, floats;
  int32_t ldq, ldk;
  const void *q = c.rows("q", type, H * dh, &nq, &ldq), *k = c.rows("k", type, Hkv * dh, &nk, &ldk);
  if (nq != nk) fail("k", "as many rows as q are wanted");
  const int32_t *cu = c.dense<int32_t>("cu_seqlens", at::kInt, -1, &seqs);
  float *scratch = c.dense<float>("scratch", at::kFloat, -1, &floats), *out = c.dense<float>("out", at::kFloat, Hkv * nq);
  const int32_t max_len = c.int32("max_len"), h = c.int32("n_heads"), hk = c.int32("n_kv_heads"), d = c.int32("head_dim"),
                window = c.int32("window");
  return PyLong_FromLong(f_mass(c.stream, code_of(type), q, ldq, k, ldk, cu, fits(seqs - 1, "cu_seqlens"), max_len,
                                fits(nq, "q"), h, hk, d, window, scratch, floats, out));
} catch (...) {
  return raised();
}

// (device, stream, k, v, pos, mass, cu_seqlens, scratch, kc, vc, cmass, cpos, clen, max_len, budget, n_recent)
PyObject *evict(PyObject *, PyObject *const *args, Py_ssize_t n) try {
  Call c(args, n, 16);
  const at::ScalarType type = type_of(args[2]);
  if (!THPVariable_Check(args[8]) || THPVariable_Unpack(args[8]).dim() != 4) fail("kc", "[n_seqs, cap, n_kv_heads, head_dim] is wanted");
  const at::Tensor &kc = THPVariable_Unpack(args[8]);
  const int64_t width = kc.size(2) * kc.size(3);
  int64_t nk, nv, seqs, ints;
  int32_t ldk, ldv;
  const void *k = c.rows("k", type, width, &nk, &ldk), *v = c.rows("v", type, width, &nv, &ldv);
  if (nk != nv || ldk != ldv) fail("v", "rows and pitch of k are wanted");
  const int32_t *pos = c.dense<int32_t>("pos", at::kInt, nk);
  const float *mass = c.dense<float>("mass", at::kFloat, kc.size(2) * nk);
  const int32_t *cu = c.dense<int32_t>("cu_seqlens", at::kInt, -1, &seqs);
  int32_t *scratch = c.dense<int32_t>("scratch", at::kInt, -1, &ints);
  const Cache cache(c, type);
  if (cache.n_seqs != seqs - 1) fail("kc", "a cache per sequence is wanted");
  const int64_t heads = cache.n_seqs * cache.heads;
  float *cmass = c.dense<float>("cmass", at::kFloat, heads * cache.cap);
  int32_t *cpos = c.dense<int32_t>("cpos", at::kInt, heads * cache.cap), *clen = c.dense<int32_t>("clen", at::kInt, heads);
  const int32_t max_len = c.int32("max_len"), budget = c.int32("budget"), recent = c.int32("n_recent");
  return PyLong_FromLong(f_evict(c.stream, code_of(type), k, v, ldk, pos, mass, cu, fits(cache.n_seqs, "kc"), max_len,
                                 fits(nk, "k"), fits(cache.heads, "kc"), fits(cache.dim, "kc"), budget, recent, scratch, ints,
                                 cache.k, cache.v, cmass, cpos, clen, fits(cache.cap, "kc")));
} catch (...) {
  return raised();
}

// (device, stream, kc, vc, q, k_new, v_new, pos_new, cmass, mass_out, cpos, pos_out, clen, len_out, scratch, o, slot, gone,
//  n_heads, budget, n_recent)
PyObject *evict_step(PyObject *, PyObject *const *args, Py_ssize_t n) try {
  Call c(args, n, 21);
  const at::ScalarType type = type_of(args[4]);
  const Cache cache(c, type);
  const int64_t S = cache.n_seqs, H = PyLong_AsLongLong(args[18]), heads = S * cache.heads, slots = heads * cache.cap;
  if (PyErr_Occurred()) throw Fail();
  int64_t nq, nk, nv, floats;
  int32_t ldq, ldk, ldv;
  const void *q = c.rows("q", type, H * cache.dim, &nq, &ldq);
  const void *k = c.rows("k_new", type, cache.heads * cache.dim, &nk, &ldk);
  const void *v = c.rows("v_new", type, cache.heads * cache.dim, &nv, &ldv);
  if (nq != S || nk != S || nv != S || ldk != ldv) fail("q, k_new, v_new", "a row per sequence, k_new and v_new of one pitch");
  const int32_t *pos_new = c.dense<int32_t>("pos_new", at::kInt, S);
  const float *mass_in = c.dense<float>("cmass", at::kFloat, slots);
  float *mass_out = c.dense<float>("mass_out", at::kFloat, slots);
  const int32_t *pos_in = c.dense<int32_t>("cpos", at::kInt, slots);
  int32_t *pos_out = c.dense<int32_t>("pos_out", at::kInt, slots);
  const int32_t *len_in = c.dense<int32_t>("clen", at::kInt, heads);
  int32_t *len_out = c.dense<int32_t>("len_out", at::kInt, heads);
  float *scratch = c.dense<float>("scratch", at::kFloat, -1, &floats);
  void *o = c.dense<void>("o", type, S * H * cache.dim);
  int32_t *slot = c.dense<int32_t>("slot", at::kInt, heads), *gone = c.dense<int32_t>("gone", at::kInt, heads);
  const int32_t h = c.int32("n_heads"), budget = c.int32("budget"), recent = c.int32("n_recent");
  return PyLong_FromLong(f_step(c.stream, code_of(type), q, ldq, k, v, ldk, pos_new, cache.k, cache.v, fits(cache.cap, "kc"),
                                mass_in, mass_out, pos_in, pos_out, len_in, len_out, fits(S, "kc"), h, fits(cache.heads, "kc"),
                                fits(cache.dim, "kc"), budget, recent, scratch, floats, o, slot, gone));
} catch (...) {
  return raised();
}

// (device, stream, q, cu_q, k_pre, v_pre, k, v, kv_idx, cu_kv, scratch, out, max_q, max_kv, n_heads, n_kv_heads, head_dim)
PyObject *attention_prefix(PyObject *, PyObject *const *args, Py_ssize_t n) try {
  Call c(args, n, 17);
  const at::ScalarType type = type_of(args[2]);
  const int64_t H = PyLong_AsLongLong(args[14]), Hkv = PyLong_AsLongLong(args[15]), dh = PyLong_AsLongLong(args[16]);
  if (PyErr_Occurred()) throw Fail();
  int64_t rows, seqs, n_pre, n_vpre, n_k, n_v, n_kv, floats;
  int32_t ldq, ldp, ldvp, ldk, ldv;
  const void *q = c.rows("q", type, H * dh, &rows, &ldq);
  const int32_t *cu_q = c.dense<int32_t>("cu_q", at::kInt, -1, &seqs);
  const void *kp = c.rows("k_pre", type, Hkv * dh, &n_pre, &ldp), *vp = c.rows("v_pre", type, Hkv * dh, &n_vpre, &ldvp);
  if (n_pre != n_vpre || ldp != ldvp) fail("v_pre", "rows and pitch of k_pre are wanted");
  const void *k = c.rows("k", type, Hkv * dh, &n_k, &ldk), *v = c.rows("v", type, Hkv * dh, &n_v, &ldv);
  if (n_k != n_v || ldk != ldv) fail("v", "rows and pitch of k are wanted");
  const int32_t *idx = c.dense<int32_t>("kv_idx", at::kInt, -1, &n_kv), *cu_kv = c.dense<int32_t>("cu_kv", at::kInt, seqs);
  float *scratch = c.dense<float>("scratch", at::kFloat, -1, &floats);
  void *out = c.dense<void>("out", type, rows * H * dh);
  const int32_t max_q = c.int32("max_q"), max_kv = c.int32("max_kv"), h = c.int32("n_heads"), hk = c.int32("n_kv_heads"),
                d = c.int32("head_dim");
  return PyLong_FromLong(f_prefix(c.stream, code_of(type), q, ldq, cu_q, fits(rows, "q"), fits(seqs - 1, "cu_q"), max_q, kp, vp,
                                  ldp, fits(n_pre, "k_pre"), k, v, ldk, fits(n_k, "k"), idx, cu_kv, fits(n_kv, "kv_idx"), max_kv,
                                  h, hk, d, scratch, floats, out));
} catch (...) {
  return raised();
}

// (device, stream, p, q or None, draft, cu_draft, u_accept, u_sample, n_accept, tokens, max_draft)
PyObject *verify(PyObject *, PyObject *const *args, Py_ssize_t n) try {
  Call c(args, n, 11);
  type_of(args[2]);
  const at::Tensor &pt = THPVariable_Unpack(args[2]);
  if (pt.dim() != 2) fail("p", "[n_draft + n_seqs, vocab] is wanted");
  const int64_t vocab = pt.size(1);
  int64_t np, nq = -1, n_draft, seqs;
  int32_t ldp, ldq = 0;
  const float *p = static_cast<float *>(c.rows("p", at::kFloat, vocab, &np, &ldp)), *q = nullptr;
  if (!c.none()) q = static_cast<float *>(c.rows("q", at::kFloat, vocab, &nq, &ldq));
  const int32_t *draft = c.dense<int32_t>("draft", at::kInt, -1, &n_draft), *cu = c.dense<int32_t>("cu_draft", at::kInt, -1, &seqs);
  seqs -= 1;
  if (np != n_draft + seqs) fail("p", "a row per draft and one more per sequence are wanted");
  if (nq >= 0 && nq != n_draft) fail("q", "a row per draft is wanted");
  const float *ua = c.dense<float>("u_accept", at::kFloat, n_draft), *us = c.dense<float>("u_sample", at::kFloat, seqs);
  int64_t n_tokens;
  int32_t *acc = c.dense<int32_t>("n_accept", at::kInt, seqs), *tokens = c.dense<int32_t>("tokens", at::kInt, -1, &n_tokens);
  const int32_t max_draft = c.int32("max_draft");
  if (n_tokens != seqs * (max_draft + 1LL)) fail("tokens", "[n_seqs, max_draft + 1] is wanted");
  return PyLong_FromLong(f_verify(c.stream, p, ldp, n_draft ? q : nullptr, n_draft ? ldq : 0, draft, cu, fits(seqs, "cu_draft"),
                                  fits(n_draft, "draft"), max_draft, fits(vocab, "p"), ua, us, acc, tokens));
} catch (...) {
  return raised();
}

// (device, stream, q, k, v, pos, rope_table, g_q or None, g_k or None, cu_q or None, k_pages, v_pages, page_table, kv_len, q_out,
//  k_out or None, eps)
PyObject *paged_append(PyObject *, PyObject *const *args, Py_ssize_t n) try {
  Call c(args, n, 17);
  const at::ScalarType type = type_of(args[2]);
  if (!THPVariable_Check(args[10]) || THPVariable_Unpack(args[10]).dim() != 4)
    fail("k_pages", "[n_pages, page_size, n_kv_heads, head_dim] is wanted");
  const at::Tensor &kp = THPVariable_Unpack(args[10]), &tq = THPVariable_Unpack(args[2]);
  const int64_t dh = kp.size(3), width = kp.size(2) * dh;
  if (tq.dim() != 2 || dh < 1 || tq.size(1) % dh) fail("q", "[n, n_heads * head_dim] is wanted");
  const int64_t wq = tq.size(1);
  int64_t nq, nk, nv, n_out, n_table, n_seqs = 0;
  int32_t ldq, ldk, ldv, ldo, ldko = 0;
  const void *q = c.rows("q", type, wq, &nq, &ldq), *k = c.rows("k", type, width, &nk, &ldk), *v = c.rows("v", type, width, &nv, &ldv);
  if (nk != nq || nv != nq || ldk != ldv) fail("k, v", "as many rows as q, of one pitch, are wanted");
  const int32_t *pos = c.dense<int32_t>("pos", at::kInt, nq);
  const float *rope = c.dense<float>("rope_table", at::kFloat, -1, &n_table);
  if (dh < 1 || n_table % dh) fail("rope_table", "[max_pos, head_dim / 2, 2] is wanted");
  const void *gq = c.none() ? nullptr : c.dense<void>("g_q", type, dh), *gk = c.none() ? nullptr : c.dense<void>("g_k", type, dh);
  const int32_t *cu = nullptr;
  const bool one_each = c.none();
  if (!one_each) cu = c.dense<int32_t>("cu_q", at::kInt, -1, &n_seqs);
  const Pages pages(c, type);
  if (!one_each && n_seqs - 1 != pages.n_seqs) fail("cu_q", "a boundary more than sequences is wanted");
  if (one_each && nq != pages.n_seqs) fail("q", "a row per sequence is wanted without cu_q");
  void *q_out = c.rows("q_out", type, wq, &n_out, &ldo), *k_out = nullptr;
  if (n_out != nq) fail("q_out", "as many rows as q are wanted");
  if (!c.none()) {
    k_out = c.rows("k_out", type, width, &n_out, &ldko);
    if (n_out != nq) fail("k_out", "as many rows as k are wanted");
  }
  const double eps = PyFloat_AsDouble(args[c.next]);
  if (eps == -1.0 && PyErr_Occurred()) throw Fail();
  return PyLong_FromLong(f_append(c.stream, code_of(type), q, ldq, k, v, ldk, pos, rope, fits(n_table / dh, "rope_table"), gq, gk,
                                  static_cast<float>(eps), cu, fits(nq, "q"), fits(pages.n_seqs, "page_table"), &pages,
                                  fits(wq / dh, "q"), fits(pages.heads, "k_pages"), fits(dh, "k_pages"), q_out, ldo, k_out, ldko));
} catch (...) {
  return raised();
}

// (device, stream, q, cu_q or None, k_pages, v_pages, page_table, kv_len, scratch, out, max_q, max_kv)
PyObject *attention_paged(PyObject *, PyObject *const *args, Py_ssize_t n) try {
  Call c(args, n, 12);
  const at::ScalarType type = type_of(args[2]);
  const at::Tensor &tq = THPVariable_Unpack(args[2]);
  if (tq.dim() != 2) fail("q", "[n, n_heads * head_dim] is wanted");
  const int64_t wq = tq.size(1);
  int64_t nq, n_seqs = 0, floats;
  int32_t ldq;
  const void *q = c.rows("q", type, wq, &nq, &ldq);
  const int32_t *cu = nullptr;
  const bool one_each = c.none();
  if (!one_each) cu = c.dense<int32_t>("cu_q", at::kInt, -1, &n_seqs);
  const Pages pages(c, type);
  if (!one_each && n_seqs - 1 != pages.n_seqs) fail("cu_q", "a boundary more than sequences is wanted");
  if (one_each && nq != pages.n_seqs) fail("q", "a row per sequence is wanted without cu_q");
  if (pages.dim < 1 || wq % pages.dim) fail("q", "[n, n_heads * head_dim] is wanted");
  float *scratch = c.dense<float>("scratch", at::kFloat, -1, &floats);
  void *out = c.dense<void>("out", type, nq * wq);
  const int32_t max_q = c.int32("max_q"), max_kv = c.int32("max_kv");
  return PyLong_FromLong(f_paged(c.stream, code_of(type), q, ldq, cu, fits(nq, "q"), fits(pages.n_seqs, "page_table"), max_q, &pages,
                                 max_kv, fits(wq / pages.dim, "q"), fits(pages.heads, "k_pages"), fits(pages.dim, "k_pages"), scratch,
                                 floats, out));
} catch (...) {
  return raised();
}

// (device, stream, logits, tokens, logprob, entropy, rank, top_id, top_logprob, n_top)
PyObject *token_logprobs(PyObject *, PyObject *const *args, Py_ssize_t n) try {
  Call c(args, n, 10);
  const at::ScalarType type = type_of(args[2]);
  const at::Tensor &t = c.tensor("logits");
  if (t.dim() != 2 || (t.numel() > 0 && t.size(1) > 1 && t.stride(1) != 1)) fail("logits", "[n, vocab] with contiguous rows is wanted");
  const int64_t rows = t.size(0), vocab = t.size(1), ld = rows > 1 ? t.stride(0) : vocab;
  if (ld < vocab) fail("logits", "rows overlap");
  const int32_t *tokens = c.dense<int32_t>("tokens", at::kInt, rows);
  float *logprob = c.dense<float>("logprob", at::kFloat, rows), *entropy = c.dense<float>("entropy", at::kFloat, rows);
  int32_t *rank = c.dense<int32_t>("rank", at::kInt, rows);
  const int64_t n_top = PyLong_AsLongLong(args[9]);
  if (PyErr_Occurred()) throw Fail();
  if (n_top < 0 || n_top > LAZY_MAX_TOP) fail("n_top", "0 to 64 are wanted");
  int32_t *id = c.dense<int32_t>("top_id", at::kInt, rows * n_top);
  float *top = c.dense<float>("top_logprob", at::kFloat, rows * n_top);
  return PyLong_FromLong(f_logprobs(c.stream, code_of(type), t.data_ptr(), ld, tokens, fits(rows, "logits"), fits(vocab, "logits"),
                                    static_cast<int32_t>(n_top), logprob, entropy, rank, id, top));
} catch (...) {
  return raised();
}

// bind(attention_mass, evict, evict_step, attention_prefix, verify, paged_append, attention_paged, token_logprobs): the entry points'
// addresses.
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n) {
  constexpr int COUNT = 8;
  void *f[COUNT];
  if (n != COUNT) {
    PyErr_SetString(PyExc_TypeError, "eight addresses are wanted");
    return nullptr;
  }
  for (int i = 0; i < COUNT; ++i) {
    f[i] = PyLong_AsVoidPtr(args[i]);
    if (!f[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is null");
      return nullptr;
    }
  }
  f_mass = reinterpret_cast<decltype(f_mass)>(f[0]);
  f_evict = reinterpret_cast<decltype(f_evict)>(f[1]);
  f_step = reinterpret_cast<decltype(f_step)>(f[2]);
  f_prefix = reinterpret_cast<decltype(f_prefix)>(f[3]);
  f_verify = reinterpret_cast<decltype(f_verify)>(f[4]);
  f_append = reinterpret_cast<decltype(f_append)>(f[5]);
  f_paged = reinterpret_cast<decltype(f_paged)>(f[6]);
  f_logprobs = reinterpret_cast<decltype(f_logprobs)>(f[7]);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind)), METH_FASTCALL, nullptr},
    {"attention_mass", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(attention_mass)), METH_FASTCALL, nullptr},
    {"evict", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(evict)), METH_FASTCALL, nullptr},
    {"evict_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(evict_step)), METH_FASTCALL, nullptr},
    {"attention_prefix", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(attention_prefix)), METH_FASTCALL, nullptr},
    {"verify", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(verify)), METH_FASTCALL, nullptr},
    {"paged_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(paged_append)), METH_FASTCALL, nullptr},
    {"attention_paged", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(attention_paged)), METH_FASTCALL, nullptr},
    {"token_logprobs", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(token_logprobs)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "lazycall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_lazycall() { return PyModule_Create(&module); }
