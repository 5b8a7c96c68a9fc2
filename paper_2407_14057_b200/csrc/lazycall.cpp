// Marshals the arguments of the operators on bounded and shared caches: torch tensors in, the C entry points of
// include/lazyllm.h out, their status back.  It does what the ctypes layer does for the other calls (checks of types, sizes and
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

// bind(attention_mass, evict, evict_step, attention_prefix, verify): the entry points' addresses.
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n) {
  void *f[5];
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "five addresses are wanted");
    return nullptr;
  }
  for (int i = 0; i < 5; ++i) {
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
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind)), METH_FASTCALL, nullptr},
    {"attention_mass", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(attention_mass)), METH_FASTCALL, nullptr},
    {"evict", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(evict)), METH_FASTCALL, nullptr},
    {"evict_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(evict_step)), METH_FASTCALL, nullptr},
    {"attention_prefix", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(attention_prefix)), METH_FASTCALL, nullptr},
    {"verify", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(verify)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "lazycall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_lazycall() { return PyModule_Create(&module); }
