// CPython module between the Python entry points and the C ABI: the checks, the output allocation, the current
// stream and the call, for the arguments that a program passes in the usual case.  Anything else -- a wrong type, a
// wrong shape, a status other than RTOPK_OK -- makes the functions return None, and the Python code behind the same entry
// point then raises what it always raised (or makes the call without scratch memory, whose launch writes every output, should
// a launch of a split call have been refused).
//
// Why native: at the sizes of a sampled mini-batch the kernel takes 3 us and the Python form of these steps (ten
// attribute reads, two torch.empty, a stream lookup, a ctypes call of eight arguments) took 10 us.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/Context.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <ATen/record_function.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/hip/HIPGuard.h>
#include <c10/hip/HIPStream.h>

#include <cstdint>
#include <exception>
#include <limits>

#include "rtopk.h"

namespace {

using at::Tensor;

// A tensor argument; nullptr where it is none.
const Tensor* tensor_of(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

// A whole number that fits 32 bits: a Python int, or whatever counts as an index (NumPy's integers).  What does not, or
// raises, is left to the Python code, with no exception set.
bool int32_of(PyObject* o, int32_t& v) {
  PyObject* made = nullptr;
  if (!PyLong_Check(o)) {
    if (!PyIndex_Check(o) || !(made = PyNumber_Index(o))) {
      PyErr_Clear();
      return false;
    }
    o = made;
  }
  int overflow = 0;
  const long long x = PyLong_AsLongLongAndOverflow(o, &overflow);
  Py_XDECREF(made);
  if (overflow != 0 || x < std::numeric_limits<int32_t>::min() || x > std::numeric_limits<int32_t>::max()) return false;
  v = (int32_t)x;
  return true;
}

// A number as a float: a Python float or int, or whatever converts to one.
bool float_of(PyObject* o, float& v) {
  const double x = PyFloat_Check(o) ? PyFloat_AS_DOUBLE(o) : (PyUnicode_Check(o) ? -1.0 : PyFloat_AsDouble(o));
  if (x == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  v = (float)x;
  return !PyUnicode_Check(o);
}

bool is_matrix(const Tensor& t, at::ScalarType type) {
  return t.is_cuda() && t.scalar_type() == type && t.dim() == 2 && t.is_contiguous();
}

bool is_shape(const Tensor& t, at::ScalarType type, int64_t rows, int64_t cols) {
  return is_matrix(t, type) && t.size(0) == rows && t.size(1) == cols;
}

// Whether a call is plain: no dispatch key beyond the default ones is switched on for the thread (modes, function transforms,
// tracing ...), no profiler listens, and new memory is not to be filled.
bool is_plain() {
  return (c10::impl::tls_local_dispatch_key_set().included_ - c10::default_included_set).empty() && !at::hasCallbacks() &&
         !at::globalContext().deterministicAlgorithms();
}

// A new tensor on the device.  at::empty goes through the dispatcher twice, which is most of its 0.65 us; a plain call makes the
// tensor directly, by the same allocator (64 x 256, k = 32, two outputs, a call among others: 5.15 -> 4.70 us, the medians of four
// runs of either in turn, each within 0.05).
Tensor new_tensor(at::IntArrayRef shape, at::ScalarType type, c10::Device device, bool plain) {
  if (!plain) return at::empty(shape, at::TensorOptions().dtype(type).device(device));
  return Tensor(at::detail::empty_cuda(shape, type, device, std::nullopt));
}

// An output: the caller's, if it fits, or a new one.  `object` is a new reference to what the caller gets back.
struct Output {
  Tensor tensor;
  PyObject* object = nullptr;
  ~Output() { Py_XDECREF(object); }
  bool set(PyObject* given, at::ScalarType type, at::IntArrayRef shape, c10::Device device, bool plain) {
    if (given != Py_None) {
      const Tensor* t = tensor_of(given);
      if (!t || !t->is_cuda() || t->scalar_type() != type || !t->is_contiguous() || t->sizes() != shape) return false;
      tensor = *t;
      object = Py_NewRef(given);
      return true;
    }
    tensor = new_tensor(shape, type, device, plain);
    object = THPVariable_Wrap(tensor);
    return object != nullptr;
  }
  PyObject* release() {
    PyObject* o = object;
    object = nullptr;
    return o;
  }
};

void* stream_of(const Tensor& t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }

// f() with C++ exceptions turned into Python's.  Without memory for an output the caller gets None, so that it makes the
// allocation itself and the user sees torch's own exception.
template <typename F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const c10::OutOfMemoryError& e) {
    Py_RETURN_NONE;
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// call() without the interpreter lock.
template <typename F>
int unlocked(F call) {
  PyThreadState* state = PyEval_SaveThread();
  const int status = call();  // a C function: does not throw
  PyEval_RestoreThread(state);
  return status;
}

PyObject* none() { Py_RETURN_NONE; }

PyObject* pair(Output& a, Output& b) {
  PyObject* t = PyTuple_New(2);
  if (!t) return nullptr;
  PyTuple_SET_ITEM(t, 0, a.release());
  PyTuple_SET_ITEM(t, 1, b.release());
  return t;
}

// Scratch memory for a shape that can use it (rtopk_workspace_bytes), from torch's allocator: stream-ordered, so it may
// go back as soon as the call has enqueued its work on the current stream.  Where there is no memory for it the call does
// without.
struct Scratch {
  Tensor tensor;
  void* data = nullptr;
  int64_t bytes = 0;
  Scratch(const Tensor& x, int32_t k, int32_t variant, int32_t max_iter, bool plain) {
    bytes = rtopk_workspace_bytes(x.size(0), (int32_t)x.size(1), k, variant, max_iter);
    if (bytes > 0) {
      try {
        tensor = new_tensor({bytes}, at::kByte, x.device(), plain);
        data = tensor.data_ptr();
      } catch (const c10::OutOfMemoryError&) {
        bytes = 0;
      }
    }
  }
};

// select(which, x, k, max_iter, out_vals, out_idx): the entry points that return pairs.  which: 0 fp32, 1 fp32 with
// byte-wide columns, 2 the k smallest, 3 half, 4 bfloat16; plus 8 for exact mode (max_iter is then not looked at).
PyObject* select(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int32_t which, k, max_iter;
    if (n != 6 || !int32_of(args[0], which) || !int32_of(args[2], k) || !int32_of(args[3], max_iter) || k < 0) return none();
    const bool exact = (which & 8) != 0;
    which &= 7;
    const Tensor* x = tensor_of(args[1]);
    const at::ScalarType vt = which == 3 ? at::kHalf : (which == 4 ? at::kBFloat16 : at::kFloat);
    const at::ScalarType it = which == 1 ? at::kByte : at::kInt;
    if (!x || !is_matrix(*x, vt)) return none();
    const int64_t N = x->size(0), M = x->size(1);
    if (M > std::numeric_limits<int32_t>::max()) return none();
    const bool plain = is_plain();
    Output v, i;
    if (!v.set(args[4], vt, {N, k}, x->device(), plain) || !i.set(args[5], it, {N, k}, x->device(), plain))
      return PyErr_Occurred() ? nullptr : none();
    const void* in = x->data_ptr();
    void *ov = v.tensor.data_ptr(), *oi = i.tensor.data_ptr(), *s = stream_of(*x);
    const int32_t m = (int32_t)M;
    const int32_t variant = (exact ? RTOPK_EXACT : RTOPK_EARLY) + (which == 2 ? RTOPK_SMALLEST : 0);
    Scratch w(*x, which == 0 || which == 2 ? k : 0, variant, max_iter, plain);  // (none for k = 0)
    const int status = unlocked([&]() -> int {
      if (w.bytes > 0)
        return rtopk_select_ws(static_cast<const float*>(in), N, m, k, variant, max_iter, 0.0f, static_cast<float*>(ov),
                               static_cast<int32_t*>(oi), nullptr, w.data, w.bytes, s);
      const float* f = static_cast<const float*>(in);
      const uint16_t* h = static_cast<const uint16_t*>(in);
      float* fv = static_cast<float*>(ov);
      uint16_t* hv = static_cast<uint16_t*>(ov);
      int32_t* ii = static_cast<int32_t*>(oi);
      uint8_t* bi = static_cast<uint8_t*>(oi);
      switch (which) {
        case 0: return exact ? rtopk_rowwise_exact(f, N, m, k, fv, ii, s) : rtopk_rowwise(f, N, m, k, max_iter, fv, ii, s);
        case 1: return exact ? rtopk_rowwise_exact_u8(f, N, m, k, fv, bi, s) : rtopk_rowwise_u8(f, N, m, k, max_iter, fv, bi, s);
        case 2: return exact ? rtopk_rowwise_exact_smallest(f, N, m, k, fv, ii, s) : rtopk_rowwise_smallest(f, N, m, k, max_iter, fv, ii, s);
        case 3: return exact ? rtopk_rowwise_exact_f16(h, N, m, k, hv, ii, s) : rtopk_rowwise_f16(h, N, m, k, max_iter, hv, ii, s);
        case 4: return exact ? rtopk_rowwise_exact_bf16(h, N, m, k, hv, ii, s) : rtopk_rowwise_bf16(h, N, m, k, max_iter, hv, ii, s);
        default: return RTOPK_ERR_BAD_SHAPE;
      }
    });
    return status == RTOPK_OK ? pair(v, i) : none();
  });
}

// select_eps(x, k, eps_rel, out_vals, out_idx, out_iters, want_iters)
PyObject* select_eps(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int32_t k;
    float eps;
    if (n != 7 || !int32_of(args[1], k) || k < 0 || !float_of(args[2], eps)) return none();
    const int iters = args[5] != Py_None ? 1 : PyObject_IsTrue(args[6]);
    if (iters < 0) return nullptr;
    const Tensor* x = tensor_of(args[0]);
    if (!x || !is_matrix(*x, at::kFloat)) return none();
    const int64_t N = x->size(0), M = x->size(1);
    if (M > std::numeric_limits<int32_t>::max()) return none();
    const bool plain = is_plain();
    Output v, i, t;
    if (!v.set(args[3], at::kFloat, {N, k}, x->device(), plain) || !i.set(args[4], at::kInt, {N, k}, x->device(), plain) ||
        (iters != 0 && !t.set(args[5], at::kInt, {N}, x->device(), plain)))
      return PyErr_Occurred() ? nullptr : none();
    const float* in = static_cast<const float*>(x->data_ptr());
    float* ov = static_cast<float*>(v.tensor.data_ptr());
    int32_t* oi = static_cast<int32_t*>(i.tensor.data_ptr());
    int32_t* ot = iters != 0 ? static_cast<int32_t*>(t.tensor.data_ptr()) : nullptr;
    void* s = stream_of(*x);
    Scratch w(*x, k, RTOPK_EPS, 0, plain);
    const int status = unlocked([&] {
      return rtopk_select_ws(in, N, (int32_t)M, k, RTOPK_EPS, 0, eps, ov, oi, ot, w.data, w.bytes, s);
    });
    if (status != RTOPK_OK) return none();
    if (iters == 0) return pair(v, i);
    PyObject* r = PyTuple_New(3);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, v.release());
    PyTuple_SET_ITEM(r, 1, i.release());
    PyTuple_SET_ITEM(r, 2, t.release());
    return r;
  });
}

// dense(x, k, max_iter, out)
PyObject* dense(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int32_t k, max_iter;
    if (n != 4 || !int32_of(args[1], k) || !int32_of(args[2], max_iter)) return none();
    const Tensor* x = tensor_of(args[0]);
    if (!x || !is_matrix(*x, at::kFloat)) return none();
    const int64_t N = x->size(0), M = x->size(1);
    if (M > std::numeric_limits<int32_t>::max()) return none();
    const bool plain = is_plain();
    Output y;
    if (!y.set(args[3], at::kFloat, {N, M}, x->device(), plain)) return PyErr_Occurred() ? nullptr : none();
    const float* in = static_cast<const float*>(x->data_ptr());
    float* out = static_cast<float*>(y.tensor.data_ptr());
    void* s = stream_of(*x);
    const int status = unlocked([&] { return rtopk_maxk_dense(in, N, (int32_t)M, k, max_iter, out, s); });
    return status == RTOPK_OK ? y.release() : none();
  });
}

// scatter(grad_vals, idx, M, grad_in) and gather(grad_out, idx, grad_vals)
PyObject* scatter(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int32_t M;
    if (n != 4 || !int32_of(args[2], M) || M < 0) return none();
    const Tensor *g = tensor_of(args[0]), *idx = tensor_of(args[1]);
    if (!g || !idx) return none();
    const bool u8 = idx->scalar_type() == at::kByte;
    if (!is_matrix(*idx, u8 ? at::kByte : at::kInt) || (u8 && M > 256)) return none();
    const int64_t N = idx->size(0), k = idx->size(1);
    if (k > std::numeric_limits<int32_t>::max() || !is_shape(*g, at::kFloat, N, k)) return none();
    const bool plain = is_plain();
    Output y;
    if (!y.set(args[3], at::kFloat, {N, M}, idx->device(), plain)) return PyErr_Occurred() ? nullptr : none();
    const float* gv = static_cast<const float*>(g->data_ptr());
    const void* ix = idx->data_ptr();
    float* out = static_cast<float*>(y.tensor.data_ptr());
    void* s = stream_of(*idx);
    const int status = unlocked([&] {
      return u8 ? rtopk_maxk_backward_u8(gv, static_cast<const uint8_t*>(ix), N, M, (int32_t)k, out, s)
                : rtopk_maxk_backward(gv, static_cast<const int32_t*>(ix), N, M, (int32_t)k, out, s);
    });
    return status == RTOPK_OK ? y.release() : none();
  });
}

PyObject* gather(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 3) return none();
    const Tensor *g = tensor_of(args[0]), *idx = tensor_of(args[1]);
    if (!g || !idx || !is_matrix(*g, at::kFloat)) return none();
    const int64_t N = g->size(0), M = g->size(1);
    const bool u8 = idx->scalar_type() == at::kByte;
    if (!is_matrix(*idx, u8 ? at::kByte : at::kInt) || (u8 && M > 256) || idx->size(0) != N) return none();
    const int64_t k = idx->size(1);
    if (k > std::numeric_limits<int32_t>::max() || M > std::numeric_limits<int32_t>::max()) return none();
    const bool plain = is_plain();
    Output y;
    if (!y.set(args[2], at::kFloat, {N, k}, idx->device(), plain)) return PyErr_Occurred() ? nullptr : none();
    const float* go = static_cast<const float*>(g->data_ptr());
    const void* ix = idx->data_ptr();
    float* out = static_cast<float*>(y.tensor.data_ptr());
    void* s = stream_of(*idx);
    const int status = unlocked([&] {
      return u8 ? rtopk_maxk_backward_gather_u8(go, static_cast<const uint8_t*>(ix), N, (int32_t)M, (int32_t)k, out, s)
                : rtopk_maxk_backward_gather(go, static_cast<const int32_t*>(ix), N, (int32_t)M, (int32_t)k, out, s);
    });
    return status == RTOPK_OK ? y.release() : none();
  });
}

// ---- operators on rows of logits ----

// Rows of logits (or their gradient): a matrix whose rows are contiguous, any distance apart that keeps them from overlapping.
struct Rows {
  void* data = nullptr;
  int64_t N = 0, stride = 0;
  int32_t M = 0, dtype = 0;
  at::ScalarType type = at::kFloat;
  bool set(const Tensor* t) {
    if (!t || !t->is_cuda() || t->dim() != 2 || t->size(1) > std::numeric_limits<int32_t>::max()) return false;
    type = t->scalar_type();
    if (type != at::kFloat && type != at::kHalf && type != at::kBFloat16) return false;
    dtype = type == at::kFloat ? RTOPK_F32 : (type == at::kHalf ? RTOPK_F16 : RTOPK_BF16);
    N = t->size(0);
    M = (int32_t)t->size(1);
    stride = N > 1 ? t->stride(0) : M;
    data = t->data_ptr();
    return (t->stride(1) == 1 || M <= 1) && stride >= M;
  }
};

bool is_vector(const Tensor* t, at::ScalarType type, int64_t n, c10::Device device) {
  return t && t->device() == device && t->scalar_type() == type && t->dim() == 1 && t->size(0) == n && t->is_contiguous();
}

// Given tokens: [N] or [N, G], 32 or 64 bits.
struct Tokens {
  const void* data = nullptr;
  int32_t bytes = 0, G = 1;
  bool set(const Tensor* t, int64_t N, c10::Device device) {
    if (!t || t->device() != device || !t->is_contiguous() || t->dim() < 1 || t->dim() > 2 || t->size(0) != N) return false;
    if (t->scalar_type() != at::kInt && t->scalar_type() != at::kLong) return false;
    if (t->dim() == 2 && t->size(1) > 1024) return false;
    bytes = t->scalar_type() == at::kLong ? 8 : 4;
    G = t->dim() == 2 ? (int32_t)t->size(1) : 1;
    data = t->data_ptr();
    return true;
  }
};

// The teacher's list: values and columns [N, k].
struct Teacher {
  const void* vals = nullptr;
  const int32_t* cols = nullptr;
  int32_t dtype = 0, k = 0, log_probs = 0;
  bool set(PyObject* v, PyObject* c, PyObject* lp, int64_t N, c10::Device device) {
    Rows r;
    const Tensor *tv = tensor_of(v), *tc = tensor_of(c);
    if (!r.set(tv) || !tv->is_contiguous() || r.N != N || tv->device() != device) return false;
    if (!tc || tc->device() != device || !is_shape(*tc, at::kInt, N, r.M)) return false;
    const int truth = PyObject_IsTrue(lp);
    if (truth < 0) {
      PyErr_Clear();
      return false;
    }
    vals = r.data;
    cols = static_cast<const int32_t*>(tc->data_ptr());
    dtype = r.dtype;
    k = r.M;
    log_probs = truth;
    return true;
  }
};

// Scratch memory as above.
struct LogitsScratch {
  Tensor tensor;
  void* data = nullptr;
  int64_t bytes = 0;
  LogitsScratch(const Tensor& x, const Rows& r, int32_t k, bool plain) {
    bytes = rtopk_logits_workspace_bytes(r.N, r.M, r.dtype, k);
    if (bytes > 0) {
      try {
        tensor = new_tensor({bytes}, at::kByte, x.device(), plain);
        data = tensor.data_ptr();
      } catch (const c10::OutOfMemoryError&) {
        bytes = 0;
      }
    }
  }
};

// The gradient: the caller's rows, or new ones.
struct Gradient {
  Output made;
  Rows rows;
  bool set(PyObject* given, const Tensor& x, const Rows& r, bool plain) {
    if (given != Py_None) {
      const Tensor* t = tensor_of(given);
      if (!rows.set(t) || t->device() != x.device() || rows.type != r.type || rows.N != r.N || rows.M != r.M) return false;
      made.object = Py_NewRef(given);
      return true;
    }
    return made.set(Py_None, r.type, {r.N, (int64_t)r.M}, x.device(), plain) && rows.set(&made.tensor);
  }
};

template <typename... O>
PyObject* tuple_of(O&... outputs) {
  PyObject* t = PyTuple_New(sizeof...(outputs));
  if (!t) return nullptr;
  Py_ssize_t i = 0;
  (PyTuple_SET_ITEM(t, i++, outputs.release()), ...);
  return t;
}

PyObject* failed() { return PyErr_Occurred() ? nullptr : none(); }

float* floats(Output& o) { return static_cast<float*>(o.tensor.data_ptr()); }

// token_logprobs(logits, tokens, k, temperature, out_logprobs, out_entropy, out_lse, out_top_logprobs, out_top_cols)
PyObject* token_logprobs(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int32_t k;
    float temperature;
    const Tensor* x = n == 9 ? tensor_of(args[0]) : nullptr;
    const Tensor* given = x ? tensor_of(args[1]) : nullptr;
    Rows r;
    Tokens t;
    if (!r.set(x) || !t.set(given, r.N, x->device()) || !int32_of(args[2], k) || k < 0 || !float_of(args[3], temperature)) return none();
    if (k == 0 && (args[7] != Py_None || args[8] != Py_None)) return none();
    const bool plain = is_plain();
    Output lp, h, lse, tl, tc;
    if (!lp.set(args[4], at::kFloat, given->sizes(), x->device(), plain) || !h.set(args[5], at::kFloat, {r.N}, x->device(), plain) ||
        !lse.set(args[6], at::kFloat, {r.N}, x->device(), plain))
      return failed();
    if (k > 0 && (!tl.set(args[7], at::kFloat, {r.N, k}, x->device(), plain) || !tc.set(args[8], at::kInt, {r.N, k}, x->device(), plain)))
      return failed();
    float *p_lp = floats(lp), *p_h = floats(h), *p_lse = floats(lse), *p_tl = k > 0 ? floats(tl) : nullptr;
    int32_t* p_tc = k > 0 ? static_cast<int32_t*>(tc.tensor.data_ptr()) : nullptr;
    void* s = stream_of(*x);
    LogitsScratch w(*x, r, k, plain);
    const int status = unlocked([&] {
      return rtopk_token_logprobs(r.data, r.dtype, r.N, r.M, r.stride, t.data, t.bytes, t.G, k, temperature, p_lp, p_h, p_lse, p_tl, p_tc, w.data,
                                  w.bytes, s);
    });
    if (status != RTOPK_OK) return none();
    return k > 0 ? tuple_of(lp, h, lse, tl, tc) : tuple_of(lp, h, lse);
  });
}

// token_logprobs_backward(grad_logprobs, logits, tokens, lse, temperature, grad_entropy, entropy, grad_logits)
PyObject* token_logprobs_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    float temperature;
    const Tensor* x = n == 8 ? tensor_of(args[1]) : nullptr;
    const Tensor* given = x ? tensor_of(args[2]) : nullptr;
    Rows r;
    Tokens t;
    if (!r.set(x) || !t.set(given, r.N, x->device()) || !float_of(args[4], temperature)) return none();
    const Tensor *g = tensor_of(args[0]), *lse = tensor_of(args[3]);
    if (!g || g->device() != x->device() || g->scalar_type() != at::kFloat || !g->is_contiguous() || g->sizes() != given->sizes()) return none();
    if (!is_vector(lse, at::kFloat, r.N, x->device())) return none();
    const float *p_gh = nullptr, *p_h = nullptr;
    if (args[5] != Py_None) {
      const Tensor *gh = tensor_of(args[5]), *h = tensor_of(args[6]);
      if (!is_vector(gh, at::kFloat, r.N, x->device()) || !is_vector(h, at::kFloat, r.N, x->device())) return none();
      p_gh = static_cast<const float*>(gh->data_ptr());
      p_h = static_cast<const float*>(h->data_ptr());
    }
    Gradient d;
    if (!d.set(args[7], *x, r, is_plain())) return failed();
    const float *p_g = static_cast<const float*>(g->data_ptr()), *p_lse = static_cast<const float*>(lse->data_ptr());
    void* s = stream_of(*x);
    const int status = unlocked([&] {
      return rtopk_token_logprobs_backward(p_g, p_gh, r.data, r.dtype, r.N, r.M, r.stride, t.data, t.bytes, t.G, p_lse, p_h, temperature,
                                           d.rows.data, d.rows.stride, s);
    });
    return status == RTOPK_OK ? d.made.release() : none();
  });
}

// distill(logits, teacher_vals, teacher_cols, temperature, log_probs, out_loss, out_lse)
PyObject* distill(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    float temperature;
    const Tensor* x = n == 7 ? tensor_of(args[0]) : nullptr;
    Rows r;
    Teacher t;
    if (!r.set(x) || !float_of(args[3], temperature) || !t.set(args[1], args[2], args[4], r.N, x->device())) return none();
    const bool plain = is_plain();
    Output loss, lse;
    if (!loss.set(args[5], at::kFloat, {r.N}, x->device(), plain) || !lse.set(args[6], at::kFloat, {r.N}, x->device(), plain)) return failed();
    float *p_loss = floats(loss), *p_lse = floats(lse);
    void* s = stream_of(*x);
    LogitsScratch w(*x, r, 0, plain);
    const int status = unlocked([&] {
      return rtopk_distill(r.data, r.dtype, r.N, r.M, r.stride, t.vals, t.dtype, t.cols, t.k, t.log_probs, temperature, p_loss, p_lse, w.data,
                           w.bytes, s);
    });
    return status == RTOPK_OK ? tuple_of(loss, lse) : none();
  });
}

// distill_backward(grad_loss, logits, teacher_vals, teacher_cols, lse, temperature, log_probs, grad_logits)
PyObject* distill_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    float temperature;
    const Tensor* x = n == 8 ? tensor_of(args[1]) : nullptr;
    Rows r;
    Teacher t;
    if (!r.set(x) || !float_of(args[5], temperature) || !t.set(args[2], args[3], args[6], r.N, x->device())) return none();
    const Tensor *g = tensor_of(args[0]), *lse = tensor_of(args[4]);
    if (!is_vector(g, at::kFloat, r.N, x->device()) || !is_vector(lse, at::kFloat, r.N, x->device())) return none();
    Gradient d;
    if (!d.set(args[7], *x, r, is_plain())) return failed();
    const float *p_g = static_cast<const float*>(g->data_ptr()), *p_lse = static_cast<const float*>(lse->data_ptr());
    void* s = stream_of(*x);
    const int status = unlocked([&] {
      return rtopk_distill_backward(p_g, r.data, r.dtype, r.N, r.M, r.stride, t.vals, t.dtype, t.cols, t.k, t.log_probs, p_lse, temperature,
                                    d.rows.data, d.rows.stride, s);
    });
    return status == RTOPK_OK ? d.made.release() : none();
  });
}

// distill_with_grad(weights, logits, teacher_vals, teacher_cols, temperature, log_probs, out_loss, grad_logits)
PyObject* distill_with_grad(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    float temperature;
    const Tensor* x = n == 8 ? tensor_of(args[1]) : nullptr;
    Rows r;
    Teacher t;
    if (!r.set(x) || !float_of(args[4], temperature) || !t.set(args[2], args[3], args[5], r.N, x->device())) return none();
    const Tensor* g = tensor_of(args[0]);
    if (!is_vector(g, at::kFloat, r.N, x->device())) return none();
    const bool plain = is_plain();
    Output loss;
    Gradient d;
    if (!loss.set(args[6], at::kFloat, {r.N}, x->device(), plain) || !d.set(args[7], *x, r, plain)) return failed();
    const float* p_g = static_cast<const float*>(g->data_ptr());
    float* p_loss = floats(loss);
    void* s = stream_of(*x);
    LogitsScratch w(*x, r, 0, plain);
    const int status = unlocked([&] {
      return rtopk_distill_with_grad(p_g, r.data, r.dtype, r.N, r.M, r.stride, t.vals, t.dtype, t.cols, t.k, t.log_probs, temperature, p_loss,
                                     d.rows.data, d.rows.stride, w.data, w.bytes, s);
    });
    return status == RTOPK_OK ? tuple_of(loss, d.made) : none();
  });
}

// Scratch memory of n bytes, if there is any.
struct Memory {
  Tensor tensor;
  void* data = nullptr;
  int64_t bytes = 0;
  Memory(int64_t n, c10::Device device, bool plain) {
    if (n <= 0) return;
    try {
      tensor = new_tensor({n}, at::kByte, device, plain);
      data = tensor.data_ptr();
      bytes = n;
    } catch (const c10::OutOfMemoryError&) {
    }
  }
};

// Random numbers and temperatures: a number for all, or a tensor with one for each.
struct Random {
  const float *uniforms = nullptr, *temperatures = nullptr;
  double temperature = 1.0;
  bool set(PyObject* u, PyObject* t, at::IntArrayRef shape, int64_t B, c10::Device device) {
    if (const Tensor* per = tensor_of(t)) {
      if (!is_vector(per, at::kFloat, B, device)) return false;
      temperatures = static_cast<const float*>(per->data_ptr());
    } else {
      if (!PyFloat_Check(t) && !PyLong_Check(t)) return false;
      temperature = PyFloat_AsDouble(t);
      if (temperature == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
      }
    }
    if (u == Py_None) return !temperatures && temperature == 0.0;
    const Tensor* x = tensor_of(u);
    if (!x || x->device() != device || x->scalar_type() != at::kFloat || !x->is_contiguous() || x->sizes() != shape) return false;
    uniforms = static_cast<const float*>(x->data_ptr());
    return true;
  }
};

// sample_tokens(logits, uniforms, temperature, out_tokens)
PyObject* sample_tokens(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const Tensor* x = n == 4 ? tensor_of(args[0]) : nullptr;
    Rows r;
    Random u;
    if (!r.set(x) || !u.set(args[1], args[2], {r.N}, r.N, x->device())) return none();
    const Tensor* given = tensor_of(args[3]);
    const at::ScalarType type = given && given->scalar_type() == at::kInt ? at::kInt : at::kLong;
    const bool plain = is_plain();
    Output out;
    if (!out.set(args[3], type, {r.N}, x->device(), plain) || out.tensor.device() != x->device()) return failed();
    void* p = out.tensor.data_ptr();
    void* s = stream_of(*x);
    Memory w(rtopk_verify_workspace_bytes(r.N, 0, r.M, r.dtype, 0), x->device(), plain);
    const c10::hip::HIPGuard on(x->device().index());
    const int status = unlocked([&] {
      return rtopk_sample_tokens(r.data, r.dtype, r.N, r.M, r.stride, u.uniforms, u.temperatures, u.temperature, p, type == at::kInt ? 4 : 8, w.data,
                                 w.bytes, s);
    });
    return status == RTOPK_OK ? out.release() : none();
  });
}

// Rows of logits of sequences, [B, positions, M].
struct Sequences {
  void* data = nullptr;
  int64_t B = 0, P = 0, seq = 0, pos = 0;
  int32_t M = 0, dtype = 0;
  bool set(const Tensor* t) {
    if (!t || !t->is_cuda() || t->dim() != 3 || t->size(2) > std::numeric_limits<int32_t>::max()) return false;
    const at::ScalarType type = t->scalar_type();
    if (type != at::kFloat && type != at::kHalf && type != at::kBFloat16) return false;
    dtype = type == at::kFloat ? RTOPK_F32 : (type == at::kHalf ? RTOPK_F16 : RTOPK_BF16);
    B = t->size(0);
    P = t->size(1);
    M = (int32_t)t->size(2);
    seq = B > 1 ? t->stride(0) : M;
    pos = P > 1 ? t->stride(1) : M;
    data = t->data_ptr();
    return (t->stride(2) == 1 || M <= 1) && seq >= M && pos >= M;
  }
};

// verify_drafts(target_logits, drafts, uniforms, draft_logits, temperature, out_tokens, out_accepted)
PyObject* verify_drafts(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const Tensor* x = n == 7 ? tensor_of(args[0]) : nullptr;
    const Tensor* d = x ? tensor_of(args[1]) : nullptr;
    Sequences t, q;
    Random u;
    if (!t.set(x) || t.P < 1 || t.P > 1024 || !d || d->device() != x->device() || !d->is_contiguous() || d->dim() != 2 || d->size(0) != t.B ||
        d->size(1) != t.P - 1 || (d->scalar_type() != at::kInt && d->scalar_type() != at::kLong))
      return none();
    if (!u.set(args[2], args[4], {t.B, t.P}, t.B, x->device())) return none();
    if (args[3] != Py_None) {
      const Tensor* y = tensor_of(args[3]);
      if (!q.set(y) || y->device() != x->device() || q.dtype != t.dtype || q.B != t.B || q.P != t.P - 1 || q.M != t.M) return none();
    }
    const bool plain = is_plain();
    Output out, accepted;
    if (!out.set(args[5], d->scalar_type(), {t.B, t.P}, x->device(), plain) || out.tensor.device() != x->device() ||
        !accepted.set(args[6], at::kInt, {t.B}, x->device(), plain) || accepted.tensor.device() != x->device())
      return failed();
    const void* p_d = d->data_ptr();
    const int bytes = d->scalar_type() == at::kInt ? 4 : 8;
    void* p_out = out.tensor.data_ptr();
    int32_t* p_accepted = static_cast<int32_t*>(accepted.tensor.data_ptr());
    void* s = stream_of(*x);
    const int G = (int)(t.P - 1);
    Memory w(rtopk_verify_workspace_bytes(t.B, G, t.M, t.dtype, q.data ? 1 : 0), x->device(), plain);
    const c10::hip::HIPGuard on(x->device().index());
    const int status = unlocked([&] {
      return rtopk_verify_drafts(t.data, q.data, t.dtype, t.B, G, t.M, t.seq, t.pos, q.seq, q.pos, p_d, bytes, u.uniforms, u.temperatures, u.temperature,
                                 p_out, p_accepted, w.data, w.bytes, s);
    });
    return status == RTOPK_OK ? tuple_of(out, accepted) : none();
  });
}

// A router's picks: columns [N, k], 32 bits or bytes.
struct Picks {
  const void* data = nullptr;
  int32_t bytes = 0, k = 0;
  bool set(const Tensor* t, int64_t N, c10::Device device) {
    if (!t || t->device() != device || !t->is_contiguous() || t->dim() != 2 || t->size(0) != N || t->size(1) > 1024) return false;
    if (t->scalar_type() != at::kInt && t->scalar_type() != at::kByte) return false;
    bytes = t->scalar_type() == at::kInt ? 4 : 1;
    k = (int32_t)t->size(1);
    data = t->data_ptr();
    return true;
  }
};

// balance_loss(logits, cols, groups, out_loss, out_z, out_probs, out_counts, out_rows)
PyObject* balance_loss(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int32_t groups;
    const Tensor* x = n == 8 ? tensor_of(args[0]) : nullptr;
    Rows r;
    Picks c;
    if (!r.set(x) || !c.set(tensor_of(args[1]), r.N, x->device()) || !int32_of(args[2], groups) || groups < 1) return none();
    const c10::Device device = x->device();
    const bool plain = is_plain();
    Output loss, z, probs, counts, rows;
    if (!loss.set(args[3], at::kFloat, {groups}, device, plain) || !z.set(args[4], at::kFloat, {groups}, device, plain) ||
        !probs.set(args[5], at::kFloat, {groups, r.M}, device, plain) || !counts.set(args[6], at::kInt, {groups, r.M}, device, plain) ||
        !rows.set(args[7], at::kInt, {groups}, device, plain))
      return failed();
    for (const Output* o : {&loss, &z, &probs, &counts, &rows})
      if (o->tensor.device() != device) return none();
    float *p_loss = floats(loss), *p_z = floats(z), *p_probs = floats(probs);
    int32_t *p_counts = static_cast<int32_t*>(counts.tensor.data_ptr()), *p_rows = static_cast<int32_t*>(rows.tensor.data_ptr());
    void* s = stream_of(*x);
    Memory w(rtopk_balance_workspace_bytes(r.N, r.M, r.dtype, c.k, groups), device, plain);
    const c10::hip::HIPGuard on(device.index());
    const int status = unlocked([&] {
      return rtopk_balance_loss(r.data, r.dtype, r.N, r.M, r.stride, c.data, c.bytes, c.k, groups, p_loss, p_z, p_probs, p_counts, p_rows, w.data, w.bytes, s);
    });
    return status == RTOPK_OK ? tuple_of(loss, z, probs, counts, rows) : none();
  });
}

// balance_loss_backward(grad_loss, logits, cols, counts, rows, grad_z, grad_vals, grad_logits)
PyObject* balance_loss_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    const Tensor* x = n == 8 ? tensor_of(args[1]) : nullptr;
    const Tensor* counts = x ? tensor_of(args[3]) : nullptr;
    Rows r;
    Picks c;
    if (!r.set(x) || !c.set(tensor_of(args[2]), r.N, x->device()) || !counts || counts->dim() != 2 || counts->size(0) < 1 || counts->size(0) > INT32_MAX) return none();
    const c10::Device device = x->device();
    const int32_t groups = (int32_t)counts->size(0);
    const Tensor *g = tensor_of(args[0]), *rows = tensor_of(args[4]);
    if (counts->device() != device || !is_shape(*counts, at::kInt, groups, r.M) || !is_vector(rows, at::kInt, groups, device) ||
        !is_vector(g, at::kFloat, groups, device))
      return none();
    const float *p_g = static_cast<const float*>(g->data_ptr()), *p_z = nullptr, *p_v = nullptr;
    if (args[5] != Py_None) {
      const Tensor* z = tensor_of(args[5]);
      if (!is_vector(z, at::kFloat, groups, device)) return none();
      p_z = static_cast<const float*>(z->data_ptr());
    }
    if (args[6] != Py_None) {
      const Tensor* v = tensor_of(args[6]);
      if (!v || v->device() != device || !is_shape(*v, at::kFloat, r.N, c.k)) return none();
      p_v = static_cast<const float*>(v->data_ptr());
    }
    Gradient d;
    if (!d.set(args[7], *x, r, is_plain())) return failed();
    const int32_t *p_counts = static_cast<const int32_t*>(counts->data_ptr()), *p_rows = static_cast<const int32_t*>(rows->data_ptr());
    void* s = stream_of(*x);
    const c10::hip::HIPGuard on(device.index());
    const int status = unlocked([&] {
      return rtopk_balance_loss_backward(p_g, p_z, p_v, r.data, r.dtype, r.N, r.M, r.stride, c.data, c.bytes, c.k, groups, p_counts, p_rows, d.rows.data,
                                         d.rows.stride, s);
    });
    return status == RTOPK_OK ? d.made.release() : none();
  });
}

template <typename F>
PyCFunction fast(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef kMethods[] = {
    {"select", fast(select), METH_FASTCALL, nullptr},   {"select_eps", fast(select_eps), METH_FASTCALL, nullptr},
    {"dense", fast(dense), METH_FASTCALL, nullptr},     {"scatter", fast(scatter), METH_FASTCALL, nullptr},
    {"gather", fast(gather), METH_FASTCALL, nullptr},   {"token_logprobs", fast(token_logprobs), METH_FASTCALL, nullptr},
    {"token_logprobs_backward", fast(token_logprobs_backward), METH_FASTCALL, nullptr},
    {"distill", fast(distill), METH_FASTCALL, nullptr}, {"distill_backward", fast(distill_backward), METH_FASTCALL, nullptr},
    {"distill_with_grad", fast(distill_with_grad), METH_FASTCALL, nullptr},
    {"sample_tokens", fast(sample_tokens), METH_FASTCALL, nullptr}, {"verify_drafts", fast(verify_drafts), METH_FASTCALL, nullptr},
    {"balance_loss", fast(balance_loss), METH_FASTCALL, nullptr},
    {"balance_loss_backward", fast(balance_loss_backward), METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr},
};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_rtopk_torch", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rtopk_torch(void) { return PyModule_Create(&kModule); }
