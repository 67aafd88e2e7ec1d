// Marshalling of the Python binding: each function takes the tensors and
// numbers of one entry point of libdsde, checks the tensors (device, type,
// contiguity, size), fetches their device pointers and the current stream, and
// calls the entry point without the interpreter lock.  The same checks in
// Python (40 tensors for a fused step, about half a microsecond each, and
// ctypes' conversion of 45 arguments) took 21 us of host time, as long as the
// step's kernels take in small batches.
#include <Python.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPStream.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>
#include <vector>

#include "dsde.h"

namespace {

PyObject *g_error = nullptr;  // paper_2509_01083_amd.DsdeError

// The entry points, looked up in the library that the package has loaded
// (set_library), which need not be the one beside this file.
#define DSDE_ENTRIES(X)                                                                                         \
  X(dsde_status_string)                                                                                         \
  X(dsde_verify) X(dsde_step) X(dsde_step_static) X(dsde_kld_signal) X(dsde_next_sl) X(dsde_calibration_update) \
  X(dsde_sample) X(dsde_top_logits) X(dsde_distill_loss) X(dsde_distill_grad) X(dsde_distill_step)              \
  X(dsde_kv_map_next) X(dsde_kv_write) X(dsde_kv_attention)                                                          \
  X(dsde_shard_stats) X(dsde_shard_accept) X(dsde_shard_accept_step) X(dsde_shard_draw_mass) X(dsde_shard_draw_pick)
struct Library {
#define X(name) decltype(&::name) name;
  DSDE_ENTRIES(X)
#undef X
} g_lib;

struct Failed {};  // a Python exception is set

[[noreturn]] void fail(const std::string &text) {
  PyErr_SetString(g_error ? g_error : PyExc_RuntimeError, text.c_str());
  throw Failed{};
}

// The arguments of one call, taken in order.
struct Args {
  PyObject *const *at;
  PyObject *const *end;

  PyObject *next() {
    if (at == end) {
      PyErr_SetString(PyExc_TypeError, "too few arguments");
      throw Failed{};
    }
    return *at++;
  }
  int64_t integer() {
    // any object with __index__; wraps like a C conversion (the library checks the ranges)
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(next());
    if (v == ~0ull && PyErr_Occurred()) throw Failed{};
    return int64_t(v);
  }
  int32_t int32() { return int32_t(integer()); }
  float real() {
    const double v = PyFloat_AsDouble(next());
    if (v == -1.0 && PyErr_Occurred()) throw Failed{};
    return float(v);
  }
  bool flag() { return PyObject_IsTrue(next()) > 0; }
  // The raw stream: an integer handle, or None for torch's current stream.
  void *stream() {
    PyObject *o = next();
    if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
    void *p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Failed{};
    return p;
  }
  void done() {
    if (at != end) {
      PyErr_SetString(PyExc_TypeError, "too many arguments");
      throw Failed{};
    }
  }
};

constexpr int kAny = -1;
constexpr int kErr = -2;  // error bits: int32 or uint32
constexpr int kI32 = int(at::ScalarType::Int), kI64 = int(at::ScalarType::Long), kU8 = int(at::ScalarType::Byte);
constexpr int kF32 = int(at::ScalarType::Float), kF64 = int(at::ScalarType::Double);

const char *type_name(int type) {
  return type == kI32 || type == kErr ? "torch.int32"
         : type == kI64 ? "torch.int64"
         : type == kU8  ? "torch.uint8"
         : type == kF32 ? "torch.float32"
                        : "torch.float64";
}

// Device pointer of a contiguous GPU tensor of `type` with at least `n`
// elements; NULL for None.
void *ptr(PyObject *o, int type, int64_t n, const char *name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) fail(std::string(name) + " must be a GPU tensor");
  const at::Tensor &t = THPVariable_Unpack(o);
  if (!t.is_cuda()) fail(std::string(name) + " must be a GPU tensor");
  const at::ScalarType is = t.scalar_type();
  if (type != kAny && int(is) != type &&
      !(type == kErr && (is == at::ScalarType::Int || is == at::ScalarType::UInt32))) {
    std::string got = "another type";
    if (PyObject *d = PyObject_GetAttrString(o, "dtype")) {
      if (PyObject *s = PyObject_Str(d)) {
        if (const char *c = PyUnicode_AsUTF8(s)) got = c;
        Py_DECREF(s);
      }
      Py_DECREF(d);
    }
    PyErr_Clear();
    fail(std::string(name) + " must be " + type_name(type) + ", got " + got);
  }
  if (!t.is_contiguous()) fail(std::string(name) + " must be contiguous");
  if (t.numel() < n)
    fail(std::string(name) + " has " + std::to_string(t.numel()) + " elements, needs " + std::to_string(n));
  return t.data_ptr();
}
template <typename T>
T *take(Args &a, int type, int64_t n, const char *name) {
  return static_cast<T *>(ptr(a.next(), type, n, name));
}
int64_t size_of(PyObject *o, int64_t dim, const char *name) {
  if (!THPVariable_Check(o)) fail(std::string(name) + " must be a GPU tensor");
  const at::Tensor &t = THPVariable_Unpack(o);
  if (t.dim() <= dim) fail(std::string(name) + " has too few dimensions");
  return t.size(dim);
}
// Raises the version of a tensor that the call writes, as torch's own operations in place do: a
// backward that has saved it then refuses it.  (Inference tensors have no version.)
void written(PyObject *o) {
  if (o == Py_None) return;
  const at::Tensor &t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// Outputs are taken from the caller's dict, or other mapping, by key.  A
// mapping's item is a new reference, dropped once its pointer is known (as
// with the inputs, the caller keeps the tensor itself alive).  `versioned`: outputs that a
// graph may hold, as the teacher's entries of a distillation.
template <typename T>
T *out(PyObject *dict, const char *key, int type, int64_t n, bool versioned = false) {
  const auto take = [&](PyObject *o) {
    T *p = static_cast<T *>(ptr(o, type, n, key));
    if (versioned) written(o);
    return p;
  };
  if (PyDict_CheckExact(dict)) {
    PyObject *o = PyDict_GetItemString(dict, key);
    if (!o) {
      PyErr_SetString(PyExc_KeyError, key);
      throw Failed{};
    }
    return take(o);
  }
  struct Ref {
    PyObject *o;
    ~Ref() { Py_XDECREF(o); }
  };
  const Ref k{PyUnicode_FromString(key)};
  const Ref o{k.o ? PyObject_GetItem(dict, k.o) : nullptr};
  if (!o.o) throw Failed{};
  return take(o.o);
}

int32_t logits_type(const at::Tensor &t) {
  if (t.scalar_type() == at::ScalarType::BFloat16) return DSDE_BF16;
  if (t.scalar_type() == at::ScalarType::Float) return DSDE_FP32;
  fail("logits must be bfloat16 or float32");
}

// The target and draft rows of a call.
struct Rows {
  const void *target, *draft;
  int32_t dtype;
  int64_t V, N;
};
// A draft that does not match the target is refused: the kernels index both with
// the target's element size and width.  `empty` refuses one without rows too,
// which nothing reads.
Rows take_rows(Args &a, int64_t B, const char *what, bool empty = true) {
  PyObject *t = a.next(), *d = a.next();
  const int64_t rows = size_of(t, 0, "target"), V = size_of(t, 1, "target");
  const at::Tensor &tt = THPVariable_Unpack(t);
  Rows r;
  r.dtype = logits_type(tt);
  r.V = V;
  r.N = d == Py_None ? 0 : size_of(d, 0, "draft");
  if (d != Py_None && (empty || r.N > 0)) {
    const at::Tensor &dt = THPVariable_Unpack(d);
    if (dt.scalar_type() != tt.scalar_type() || (r.N > 0 && size_of(d, 1, "draft") != V))
      fail(std::string("draft ") + what + " must match the target's dtype and vocabulary");
  }
  if (rows != r.N + B)
    fail("target has " + std::to_string(rows) + " rows, expected N + B = " + std::to_string(r.N + B));
  r.target = ptr(t, kAny, 0, "target");
  r.draft = r.N > 0 ? ptr(d, kAny, 0, "draft") : nullptr;
  return r;
}

// Per-sequence and per-position inputs in the order of the entry points.
struct Batch {
  const int32_t *sl, *cu_sl, *tokens;
  const float *temperature, *u_acc, *u_res;
};
Batch take_batch(PyObject *const *p, int64_t B, int64_t N) {
  Batch x;
  x.sl = static_cast<const int32_t *>(ptr(p[0], kI32, B, "sl"));
  x.cu_sl = static_cast<const int32_t *>(ptr(p[1], kI32, B + 1, "cu_sl"));
  x.tokens = N > 0 ? static_cast<const int32_t *>(ptr(p[2], kI32, N, "draft_tokens")) : nullptr;
  x.temperature = static_cast<const float *>(ptr(p[3], kF32, B, "temperature"));
  x.u_acc = N > 0 ? static_cast<const float *>(ptr(p[4], kF32, N, "u_acc")) : nullptr;
  x.u_res = static_cast<const float *>(ptr(p[5], kF32, B, "u_res"));
  return x;
}

// The outputs every verification call has.
struct VerifyOut {
  int32_t *accepted, *tokens;
  float *kld, *entropy;
  double *row_lse;
};
VerifyOut take_verify_out(PyObject *dict, PyObject *row_lse, bool entropy, int64_t B, int64_t N, int32_t k_max) {
  VerifyOut o;
  o.accepted = out<int32_t>(dict, "accepted", kI32, B);
  o.tokens = out<int32_t>(dict, "tokens", kI32, B * (k_max + 1));
  o.kld = N > 0 ? out<float>(dict, "kld", kF32, N) : nullptr;
  o.row_lse = static_cast<double *>(ptr(row_lse, kF64, 2 * N, "row_lse"));
  o.entropy = entropy && N > 0 ? out<float>(dict, "draft_entropy", kF32, N) : nullptr;
  return o;
}

// The ring, the signal's and the rule's parameters and outputs of the fused calls.
struct Signal {
  float *hist;
  int32_t *head, *count;
  const float *sl_max;
  int32_t W, n_short, n_long;
  float delta, eps, sl_min;
  int32_t sl_hi;
  const int32_t *budget;
  float *mu_last, *var_short, *var_long, *wvir, *sf, *sl_hat, *sl_cap;
  int32_t *sl_next;
};
Signal take_signal(Args &a, PyObject *dict, int64_t B) {
  Signal s;
  PyObject *hist = a.next();
  const int64_t W = size_of(hist, 1, "hist");
  s.W = int32_t(W);
  s.hist = static_cast<float *>(ptr(hist, kF32, B * W, "hist"));
  s.head = take<int32_t>(a, kI32, B, "head");
  s.count = take<int32_t>(a, kI32, B, "count");
  s.sl_max = take<float>(a, kF32, B, "sl_max");
  s.n_short = a.int32();
  s.n_long = a.int32();
  s.delta = a.real();
  s.eps = a.real();
  s.sl_min = a.real();
  s.sl_hi = a.int32();
  s.budget = take<int32_t>(a, kI32, B, "budget");
  s.mu_last = out<float>(dict, "mu_last", kF32, B);
  s.var_short = out<float>(dict, "var_short", kF32, B);
  s.var_long = out<float>(dict, "var_long", kF32, B);
  s.wvir = out<float>(dict, "wvir", kF32, B);
  s.sf = out<float>(dict, "sf", kF32, B);
  s.sl_hat = out<float>(dict, "sl_hat", kF32, B);
  s.sl_cap = out<float>(dict, "sl_cap", kF32, 1);
  s.sl_next = out<int32_t>(dict, "sl_next", kI32, B);
  return s;
}

void *take_workspace(Args &a, size_t *bytes) {
  PyObject *o = a.next();
  void *p = ptr(o, kU8, 0, "workspace");
  *bytes = o == Py_None ? 0 : size_t(THPVariable_Unpack(o).numel());
  return p;
}

template <typename F>
void call(F f) {
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS rc = f();
  Py_END_ALLOW_THREADS if (rc != DSDE_OK)
      fail(std::string("libdsde: ") + g_lib.dsde_status_string(rc) + " (status " + std::to_string(rc) + ")");
}

// Runs one function body; C++ exceptions become Python ones.
template <typename F>
PyObject *guarded(PyObject *const *args, Py_ssize_t n, F f) {
  try {
    Args a{args, args + n};
    f(a);
    Py_RETURN_NONE;
  } catch (const Failed &) {
  } catch (const std::exception &e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

// verify(target, draft, sl, cu_sl, draft_tokens, temperature, u_acc, u_res, k_max, pad_id, out, row_lse,
//        draft_entropy, workspace, stream)
PyObject *py_verify(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    if (n < 8) a.at = a.end;
    PyObject *const *batch = args + 2;
    const int64_t B = n < 8 ? 0 : size_of(batch[0], 0, "sl");
    const Rows r = take_rows(a, B, "logits");
    const Batch x = take_batch(batch, B, r.N);
    a.at += 6;
    const int32_t k_max = a.int32(), pad = a.int32();
    PyObject *dict = a.next(), *lse = a.next();
    const VerifyOut o = take_verify_out(dict, lse, a.flag(), B, r.N, k_max);
    uint32_t *err = out<uint32_t>(dict, "seq_err", kErr, B);
    size_t bytes;
    void *ws = take_workspace(a, &bytes), *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_verify(r.target, r.draft, r.dtype, r.V, int32_t(B), r.N, k_max, x.sl, x.cu_sl, x.tokens,
                         x.temperature, x.u_acc, x.u_res, pad, o.accepted, o.tokens, o.kld, err, o.row_lse, o.entropy,
                         ws, bytes, stream);
    });
  });
}

// step(target, draft, sl, cu_sl, draft_tokens, temperature, u_acc, u_res, k_max, pad_id, out, row_lse,
//      draft_entropy, hist, head, count, sl_max, n_short, n_long, delta, eps, sl_min, sl_hi, budget, workspace,
//      stream); workspace False: dsde_step_static
PyObject *py_step(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    if (n < 8) a.at = a.end;
    PyObject *const *batch = args + 2;
    const int64_t B = n < 8 ? 0 : size_of(batch[0], 0, "sl");
    const Rows r = take_rows(a, B, "logits", false);
    const Batch x = take_batch(batch, B, r.N);
    a.at += 6;
    const int32_t k_max = a.int32(), pad = a.int32();
    PyObject *dict = a.next(), *lse = a.next();
    const VerifyOut o = take_verify_out(dict, lse, a.flag(), B, r.N, k_max);
    const Signal s = take_signal(a, dict, B);
    uint32_t *err = out<uint32_t>(dict, "seq_err", kErr, B);
    const bool fixed = a.at < a.end && *a.at == Py_False;
    size_t bytes = 0;
    void *ws = nullptr;
    if (fixed)
      a.next();
    else
      ws = take_workspace(a, &bytes);
    void *stream = a.stream();
    a.done();
    call([&] {
      if (fixed)
        return g_lib.dsde_step_static(r.target, r.draft, r.dtype, r.V, int32_t(B), r.N, k_max, x.sl, x.cu_sl, x.tokens,
                                x.temperature, x.u_acc, x.u_res, pad, o.accepted, o.tokens, o.kld, o.row_lse,
                                o.entropy, s.hist, s.head, s.count, s.W, s.n_short, s.n_long, s.delta, s.eps,
                                s.mu_last, s.var_short, s.var_long, s.wvir, s.sf, s.sl_max, s.sl_min, s.sl_hi,
                                s.budget, s.sl_hat, s.sl_cap, s.sl_next, err, stream);
      return g_lib.dsde_step(r.target, r.draft, r.dtype, r.V, int32_t(B), r.N, k_max, x.sl, x.cu_sl, x.tokens,
                       x.temperature, x.u_acc, x.u_res, pad, o.accepted, o.tokens, o.kld, o.row_lse, o.entropy, s.hist,
                       s.head, s.count, s.W, s.n_short, s.n_long, s.delta, s.eps, s.mu_last, s.var_short, s.var_long,
                       s.wvir, s.sf, s.sl_max, s.sl_min, s.sl_hi, s.budget, s.sl_hat, s.sl_cap, s.sl_next, err, ws,
                       bytes, stream);
    });
  });
}

// kld_signal(sl, cu_sl, kld, hist, head, count, n_short, n_long, delta, eps, out, stream)
PyObject *py_kld_signal(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    PyObject *sl_o = a.next(), *cu_o = a.next(), *kld_o = a.next(), *hist_o = a.next();
    const int64_t B = size_of(sl_o, 0, "sl"), N = size_of(kld_o, 0, "kld"), W = size_of(hist_o, 1, "hist");
    const auto *sl = static_cast<const int32_t *>(ptr(sl_o, kI32, B, "sl"));
    const auto *cu = static_cast<const int32_t *>(ptr(cu_o, kI32, B + 1, "cu_sl"));
    const auto *kld = N > 0 ? static_cast<const float *>(ptr(kld_o, kF32, N, "kld")) : nullptr;
    auto *hist = static_cast<float *>(ptr(hist_o, kF32, B * W, "hist"));
    int32_t *head = take<int32_t>(a, kI32, B, "head"), *count = take<int32_t>(a, kI32, B, "count");
    const int32_t n_short = a.int32(), n_long = a.int32();
    const float delta = a.real(), eps = a.real();
    PyObject *d = a.next();
    float *mu = out<float>(d, "mu_last", kF32, B), *vs = out<float>(d, "var_short", kF32, B);
    float *vl = out<float>(d, "var_long", kF32, B), *wvir = out<float>(d, "wvir", kF32, B);
    float *sf = out<float>(d, "sf", kF32, B);
    uint32_t *err = out<uint32_t>(d, "seq_err", kErr, B);
    void *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_kld_signal(int32_t(B), N, sl, cu, kld, hist, head, count, int32_t(W), n_short, n_long, delta, eps, mu,
                             vs, vl, wvir, sf, err, stream);
    });
  });
}

// next_sl(sf, wvir, sl_max, sl_min, sl_hi, budget, out, stream)
PyObject *py_next_sl(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    PyObject *sf_o = a.next();
    const int64_t B = size_of(sf_o, 0, "sf");
    const auto *sf = static_cast<const float *>(ptr(sf_o, kF32, B, "sf"));
    const float *wvir = take<float>(a, kF32, B, "wvir"), *sl_max = take<float>(a, kF32, B, "sl_max");
    const float sl_min = a.real();
    const int32_t sl_hi = a.int32();
    const int32_t *budget = take<int32_t>(a, kI32, B, "budget");
    PyObject *d = a.next();
    float *hat = out<float>(d, "sl_hat", kF32, B), *cap = out<float>(d, "sl_cap", kF32, 1);
    int32_t *next = out<int32_t>(d, "sl_next", kI32, B);
    uint32_t *err = out<uint32_t>(d, "seq_err", kErr, B);
    void *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_next_sl(int32_t(B), sf, wvir, sl_max, sl_min, sl_hi, budget, hat, cap, next, err, stream);
    });
  });
}

// calibration_update(sl, cu_sl, accepted, kld, seq_err, state, stream)
PyObject *py_calibration_update(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    PyObject *sl_o = a.next(), *cu_o = a.next(), *acc_o = a.next(), *kld_o = a.next(), *err_o = a.next();
    PyObject *d = a.next();
    const int64_t B = size_of(sl_o, 0, "sl"), N = size_of(kld_o, 0, "kld");
    const auto *sl = static_cast<const int32_t *>(ptr(sl_o, kI32, B, "sl"));
    const auto *cu = static_cast<const int32_t *>(ptr(cu_o, kI32, B + 1, "cu_sl"));
    const auto *acc = static_cast<const int32_t *>(ptr(acc_o, kI32, B, "accepted"));
    const auto *kld = N > 0 ? static_cast<const float *>(ptr(kld_o, kF32, N, "kld")) : nullptr;
    const auto *err = static_cast<const uint32_t *>(ptr(err_o, kErr, B, "seq_err"));
    int32_t *a_max = out<int32_t>(d, "a_max", kI32, B);
    double *sum = out<double>(d, "kld_sum", kF64, B);
    int64_t *cnt = out<int64_t>(d, "kld_count", kI64, B);
    float *kmax = out<float>(d, "kld_max", kF32, B);
    void *stream = a.stream();
    a.done();
    call([&] { return g_lib.dsde_calibration_update(int32_t(B), N, sl, cu, acc, kld, err, a_max, sum, cnt, kmax, stream); });
  });
}

// shard_stats(target, draft, v_begin, V, sl, cu_sl, draft_tokens, temperature, k_max, workspace, part, seq_err, stream)
PyObject *py_shard_stats(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    if (n < 8) a.at = a.end;
    const int64_t B = n < 8 ? 0 : size_of(args[4], 0, "sl");
    const Rows r = take_rows(a, B, "slice");
    const int64_t v_begin = a.integer(), V = a.integer();
    const int32_t *sl = take<int32_t>(a, kI32, B, "sl"), *cu = take<int32_t>(a, kI32, B + 1, "cu_sl");
    PyObject *tok_o = a.next();
    const auto *tok = r.N > 0 ? static_cast<const int32_t *>(ptr(tok_o, kI32, r.N, "draft_tokens")) : nullptr;
    const float *temp = take<float>(a, kF32, B, "temperature");
    const int32_t k_max = a.int32();
    size_t bytes;
    void *ws = take_workspace(a, &bytes);
    PyObject *part_o = a.next();
    void *part = r.N > 0 ? ptr(part_o, kU8, r.N * int64_t(sizeof(dsde_shard_partial)), "part") : nullptr;
    uint32_t *err = take<uint32_t>(a, kErr, B, "seq_err");
    void *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_shard_stats(r.target, r.draft, r.dtype, r.V, v_begin, V, int32_t(B), r.N, k_max, sl, cu, tok, temp,
                              static_cast<dsde_shard_partial *>(part), err, ws, bytes, stream);
    });
  });
}

// shard_accept(fused, parts, V, sl, cu_sl, draft_tokens, temperature, u_acc, u_res, k_max, pad_id, out, row_lse,
//              draft_entropy, seq_err[, hist, head, count, sl_max, n_short, n_long, delta, eps, sl_min, sl_hi, budget],
//              stream); parts packed [G, N, 64]
PyObject *py_shard_accept(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    const bool fused = a.flag();
    PyObject *parts_o = a.next();
    const int64_t G = size_of(parts_o, 0, "parts"), V = a.integer();
    if (a.end - a.at < 6) a.at = a.end;
    PyObject *const *batch = a.at;
    PyObject *sl_o = a.next();
    const int64_t B = size_of(sl_o, 0, "sl");
    const int64_t N = batch[2] == Py_None ? 0 : size_of(batch[2], 0, "draft_tokens");
    a.at = batch + 6;
    const Batch x = take_batch(batch, B, N);
    const auto *parts = N > 0 ? static_cast<const dsde_shard_partial *>(
                                    ptr(parts_o, kU8, G * N * int64_t(sizeof(dsde_shard_partial)), "parts"))
                              : nullptr;
    const int32_t k_max = a.int32(), pad = a.int32();
    PyObject *dict = a.next(), *lse = a.next();
    const VerifyOut o = take_verify_out(dict, lse, a.flag(), B, N, k_max);
    auto *jobs = out<dsde_draw_job>(dict, "jobs", kU8, B * int64_t(sizeof(dsde_draw_job)));
    uint32_t *err = take<uint32_t>(a, kErr, B, "seq_err");
    Signal s{};
    if (fused) s = take_signal(a, dict, B);
    void *stream = a.stream();
    a.done();
    call([&] {
      if (!fused)
        return g_lib.dsde_shard_accept(int32_t(G), parts, V, int32_t(B), N, k_max, x.sl, x.cu_sl, x.tokens, x.temperature,
                                 x.u_acc, x.u_res, pad, o.accepted, o.tokens, o.kld, o.row_lse, o.entropy, jobs, err,
                                 stream);
      return g_lib.dsde_shard_accept_step(int32_t(G), parts, V, int32_t(B), N, k_max, x.sl, x.cu_sl, x.tokens, x.temperature,
                                    x.u_acc, x.u_res, pad, o.accepted, o.tokens, o.kld, o.row_lse, o.entropy, jobs,
                                    s.hist, s.head, s.count, s.W, s.n_short, s.n_long, s.delta, s.eps, s.mu_last,
                                    s.var_short, s.var_long, s.wvir, s.sf, s.sl_max, s.sl_min, s.sl_hi, s.budget,
                                    s.sl_hat, s.sl_cap, s.sl_next, err, stream);
    });
  });
}

// shard_draw_mass(target, draft, v_begin, part, jobs, k_max, workspace, mass, stream)
PyObject *py_shard_draw_mass(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    if (n < 5) a.at = a.end;
    const int64_t B = n < 5 ? 0 : size_of(args[4], 0, "jobs");
    const Rows r = take_rows(a, B, "slice");
    const int64_t v_begin = a.integer();
    PyObject *part_o = a.next();
    void *part = r.N > 0 ? ptr(part_o, kU8, r.N * int64_t(sizeof(dsde_shard_partial)), "part") : nullptr;
    auto *jobs = take<dsde_draw_job>(a, kU8, B * int64_t(sizeof(dsde_draw_job)), "jobs");
    const int32_t k_max = a.int32();
    size_t bytes;
    void *ws = take_workspace(a, &bytes);
    auto *mass = take<dsde_shard_mass>(a, kU8, B * int64_t(sizeof(dsde_shard_mass)), "mass");
    void *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_shard_draw_mass(r.target, r.draft, r.dtype, r.V, v_begin, int32_t(B), r.N, k_max,
                                  static_cast<const dsde_shard_partial *>(part), jobs, mass, ws, bytes, stream);
    });
  });
}

// shard_draw_pick(g, masses, target, draft, v_begin, jobs, k_max, pad_id, accepted, tokens, drawn, seq_err, workspace,
//                 stream)
PyObject *py_shard_draw_pick(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    const int32_t g = a.int32();
    PyObject *masses_o = a.next();
    if (n < 6) a.at = a.end;
    const int64_t G = size_of(masses_o, 0, "masses"), B = n < 6 ? 0 : size_of(args[5], 0, "jobs");
    const Rows r = take_rows(a, B, "slice");
    const auto *masses = static_cast<const dsde_shard_mass *>(
        ptr(masses_o, kU8, G * B * int64_t(sizeof(dsde_shard_mass)), "masses"));
    const int64_t v_begin = a.integer();
    auto *jobs = take<dsde_draw_job>(a, kU8, B * int64_t(sizeof(dsde_draw_job)), "jobs");
    const int32_t k_max = a.int32(), pad = a.int32();
    int32_t *accepted = take<int32_t>(a, kI32, B, "accepted");
    int32_t *tokens = take<int32_t>(a, kI32, B * (k_max + 1), "tokens"), *drawn = take<int32_t>(a, kI32, B, "drawn");
    uint32_t *err = take<uint32_t>(a, kErr, B, "seq_err");
    size_t bytes;
    void *ws = take_workspace(a, &bytes), *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_shard_draw_pick(int32_t(G), g, masses, r.target, r.draft, r.dtype, r.V, v_begin, int32_t(B), r.N,
                                  k_max, jobs, pad, accepted, tokens, drawn, err, ws, bytes, stream);
    });
  });
}

// Strided rows [R, V] of logits: any row stride, each row dense.
struct LogitRows {
  void *data;
  int64_t R, V, stride;
  int32_t dtype;
};
LogitRows take_strided(Args &a, const char *name) {
  PyObject *o = a.next();
  size_of(o, 1, name);
  const at::Tensor &t = THPVariable_Unpack(o);
  LogitRows r;
  r.dtype = logits_type(t);
  if (t.dim() != 2) fail(std::string(name) + " must be [rows, vocabulary]");
  if (!t.is_cuda()) fail(std::string(name) + " must be a GPU tensor");
  r.R = t.size(0);
  r.V = t.size(1);
  r.stride = r.R > 1 ? t.stride(0) : r.V;
  if (r.R > 0 && r.V > 1 && t.stride(1) != 1) fail(std::string(name) + " must have dense rows");
  if (r.R > 1 && r.stride < r.V) fail(std::string(name) + " must have rows that do not overlap");
  r.data = t.data_ptr();
  return r;
}

// sample(logits, temperature, top_k, top_p, min_p, u, pad_id, out, workspace, stream); logprob and kept where out has them
PyObject *py_sample(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    const LogitRows z = take_strided(a, "logits");
    const auto *T = take<float>(a, kF32, z.R, "temperature");
    const auto *k = take<int32_t>(a, kI32, z.R, "top_k");
    const auto *p = take<float>(a, kF32, z.R, "top_p"), *m = take<float>(a, kF32, z.R, "min_p");
    const auto *u = take<float>(a, kF32, z.R, "u");
    const int32_t pad = a.int32();
    PyObject *dict = a.next();
    auto *tokens = out<int32_t>(dict, "tokens", kI32, z.R, true);
    auto *lp = PyMapping_HasKeyString(dict, "logprob") ? out<float>(dict, "logprob", kF32, z.R, true) : nullptr;
    auto *kept = PyMapping_HasKeyString(dict, "kept") ? out<int32_t>(dict, "kept", kI32, z.R, true) : nullptr;
    auto *err = out<uint32_t>(dict, "row_err", kErr, z.R, true);
    size_t bytes;
    void *ws = take_workspace(a, &bytes), *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_sample(z.data, z.stride, z.dtype, z.V, z.R, T, k, p, m, u, pad, tokens, lp, kept, err, ws,
                               bytes, stream);
    });
  });
}

// top_logits(logits, k, temperature, out, workspace, stream)
PyObject *py_top_logits(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    const LogitRows z = take_strided(a, "logits");
    const int32_t k = a.int32();
    const float T = a.real();
    PyObject *dict = a.next();
    auto *values = out<float>(dict, "values", kF32, z.R * k, true);
    auto *ids = out<int32_t>(dict, "ids", kI32, z.R * k, true);
    auto *lse = out<float>(dict, "lse", kF32, z.R, true);
    auto *err = out<uint32_t>(dict, "row_err", kErr, z.R, true);
    size_t bytes;
    void *ws = take_workspace(a, &bytes), *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_top_logits(z.data, z.stride, z.dtype, z.V, z.R, k, T, values, ids, lse, err, ws, bytes, stream);
    });
  });
}

// The teacher of a distillation: ids [N, K], teacher [N, K], teacher_lse [N] or None.
struct Teacher {
  int32_t K;
  const int32_t *ids;
  const float *logits;
};
Teacher take_teacher(Args &a, int64_t N) {
  Teacher x;
  PyObject *ids = a.next(), *logits = a.next();
  const int64_t K = size_of(ids, 1, "ids");
  for (PyObject *o : {ids, logits}) {
    const char *name = o == ids ? "ids" : "teacher";
    if (size_of(o, 0, name) != N || size_of(o, 1, name) != K || THPVariable_Unpack(o).dim() != 2)
      fail("ids and teacher must be [N, K] for logits of N rows");
  }
  x.K = int32_t(K);
  x.ids = static_cast<const int32_t *>(ptr(ids, kI32, N * K, "ids"));
  x.logits = static_cast<const float *>(ptr(logits, kF32, N * K, "teacher"));
  return x;
}
LogitRows take_gradient(Args &a, const LogitRows &z) {
  const LogitRows g = take_strided(a, "grad");
  if (g.R != z.R || g.V != z.V || g.dtype != z.dtype) fail("grad must have the logits' shape and type");
  written(a.at[-1]);
  return g;
}

// distill_loss(logits, ids, teacher, teacher_lse, temperature, out, workspace, stream)
PyObject *py_distill_loss(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    const LogitRows z = take_strided(a, "logits");
    const Teacher x = take_teacher(a, z.R);
    const auto *lse = take<float>(a, kF32, z.R, "teacher_lse");
    const float T = a.real();
    PyObject *dict = a.next();
    auto *loss = out<float>(dict, "loss", kF32, z.R, true);
    auto *record = out<dsde_distill_row>(dict, "record", kU8, z.R * int64_t(sizeof(dsde_distill_row)), true);
    auto *err = out<uint32_t>(dict, "row_err", kErr, z.R, true);
    size_t bytes;
    void *ws = take_workspace(a, &bytes), *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_distill_loss(z.data, z.stride, z.dtype, z.V, z.R, x.K, x.ids, x.logits, lse, T, loss, record,
                                     err, ws, bytes, stream);
    });
  });
}

// distill_grad(logits, ids, teacher, temperature, record, weight, grad, stream)
PyObject *py_distill_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    const LogitRows z = take_strided(a, "logits");
    const Teacher x = take_teacher(a, z.R);
    const float T = a.real();
    const auto *record = take<dsde_distill_row>(a, kU8, z.R * int64_t(sizeof(dsde_distill_row)), "record");
    const auto *weight = take<float>(a, kF32, z.R, "weight");
    const LogitRows g = take_gradient(a, z);
    void *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_distill_grad(z.data, z.stride, z.dtype, z.V, z.R, x.K, x.ids, x.logits, T, record, weight,
                                     g.data, g.stride, stream);
    });
  });
}

// distill_step(logits, ids, teacher, teacher_lse, temperature, weight, loss, grad, row_err, workspace, stream)
PyObject *py_distill_step(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    const LogitRows z = take_strided(a, "logits");
    const Teacher x = take_teacher(a, z.R);
    const auto *lse = take<float>(a, kF32, z.R, "teacher_lse");
    const float T = a.real();
    const auto *weight = take<float>(a, kF32, z.R, "weight");
    auto *loss = take<float>(a, kF32, z.R, "loss");
    written(a.at[-1]);
    const LogitRows g = take_gradient(a, z);
    auto *err = take<uint32_t>(a, kErr, z.R, "row_err");
    written(a.at[-1]);
    size_t bytes;
    void *ws = take_workspace(a, &bytes), *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_distill_step(z.data, z.stride, z.dtype, z.V, z.R, x.K, x.ids, x.logits, lse, T, weight, loss,
                                     g.data, g.stride, err, ws, bytes, stream);
    });
  });
}

// The cache's calls: their tensors lie on one device, which is made the current one for the call (its
// current stream too, where no stream is given).
struct OneDevice {
  c10::OptionalDeviceGuard guard;
  int device = -1;
  std::vector<PyObject *> items;  // taken from mappings, held for the call

  ~OneDevice() {
    for (PyObject *o : items) Py_DECREF(o);
  }
  PyObject *item(PyObject *dict, const char *key) {
    PyObject *o = PyMapping_GetItemString(dict, key);
    if (!o) throw Failed{};
    items.push_back(o);
    return o;
  }

  void see(PyObject *o, const char *name) {
    if (o == Py_None || !THPVariable_Check(o)) return;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) return;  // refused where its pointer is taken
    if (device < 0)
      guard.reset_device(t.device()), device = t.get_device();
    else if (t.get_device() != device)
      fail(std::string(name) + " must be on the device of the other tensors");
  }
};
// An array of a call: on the call's device, contiguous; `write`: raises its version.
template <typename T>
T *take_on(Args &a, OneDevice &dev, int type, int64_t n, const char *name, bool write = false) {
  PyObject *o = a.next();
  dev.see(o, name);
  T *p = static_cast<T *>(ptr(o, type, n, name));
  if (write) written(o);
  return p;
}
template <typename T>
T *out_on(PyObject *dict, OneDevice &dev, const char *key, int type, int64_t n) {
  PyObject *o = dev.item(dict, key);
  dev.see(o, key);
  T *p = static_cast<T *>(ptr(o, type, n, key));
  written(o);
  return p;
}

// The cache's calls go forward only: where a gradient is being recorded, a tensor that wants one would lose it unsaid.
void forward_only(PyObject *o, const char *name) {
  if (o != Py_None && THPVariable_Check(o) && c10::GradMode::is_enabled() && THPVariable_Unpack(o).requires_grad())
    fail(std::string(name) + " requires a gradient, which the cache's calls do not give: call them under torch.no_grad()");
}

// Rows [T, heads, dim] with dense heads.
struct HeadRows {
  void *data;
  int64_t T, heads, dim, token_stride, head_stride;
  at::ScalarType type;
};
HeadRows head_rows(PyObject *o, OneDevice &dev, const char *name) {
  size_of(o, 2, name);
  const at::Tensor &t = THPVariable_Unpack(o);
  if (t.dim() != 3) fail(std::string(name) + " must be [rows, heads, dim]");
  forward_only(o, name);
  if (t.scalar_type() != at::ScalarType::BFloat16 && t.scalar_type() != at::ScalarType::Float)
    fail(std::string(name) + " must be bfloat16 or float32");
  if (!t.is_cuda()) fail(std::string(name) + " must be a GPU tensor");
  dev.see(o, name);
  HeadRows r{t.data_ptr(), t.size(0), t.size(1), t.size(2), t.size(0) > 1 ? t.stride(0) : 0,
             t.size(1) > 1 ? t.stride(1) : 0, t.scalar_type()};
  if (t.numel() > 0 && r.dim > 1 && t.stride(2) != 1) fail(std::string(name) + " must have dense heads");
  const int64_t e = t.element_size();
  if (t.numel() > 0 && (reinterpret_cast<uintptr_t>(r.data) % 16 != 0 || r.token_stride * e % 16 != 0 || r.head_stride * e % 16 != 0))
    fail(std::string(name) + " must have heads that start at multiples of 16 bytes");
  return r;
}
int32_t row_type(const HeadRows &r) { return r.type == at::ScalarType::BFloat16 ? DSDE_BF16 : DSDE_FP32; }

// A cache of two tensors [pages, heads, page_size, dim] of one layout, and its scales.
dsde_kv_cache take_cache(Args &a, OneDevice &dev, bool write) {
  PyObject *o[2] = {a.next(), a.next()};
  const char *names[2] = {"k_cache", "v_cache"};
  dsde_kv_cache c{};
  for (int i = 0; i < 2; ++i) {
    size_of(o[i], 3, names[i]);
    const at::Tensor &t = THPVariable_Unpack(o[i]);
    if (t.dim() != 4) fail(std::string(names[i]) + " must be [pages, heads, page_size, dim]");
    forward_only(o[i], names[i]);
    const at::ScalarType is = t.scalar_type();
    if (is != at::ScalarType::BFloat16 && is != at::ScalarType::Float && is != at::ScalarType::Float8_e4m3fn)
      fail(std::string(names[i]) + " must be bfloat16, float32 or float8_e4m3fn");
    if (!t.is_cuda()) fail(std::string(names[i]) + " must be a GPU tensor");
    dev.see(o[i], names[i]);
    int64_t size[4], stride[4];
    for (int d = 0; d < 4; ++d) {
      size[d] = t.size(d);
      stride[d] = size[d] > 1 ? t.stride(d) : 0;
    }
    if (size[0] < 1 || size[0] > 0x7fffffff || size[1] < 1 || size[1] > DSDE_MAX_HEADS) fail(std::string(names[i]) + " has too few or too many pages or heads");
    if (size[2] < 16 || size[2] > 1024 || (size[2] & (size[2] - 1)) != 0) fail("page_size must be a power of two in 16..1024");
    if (size[3] < 16 || size[3] > DSDE_MAX_DIM || size[3] % 16 != 0) fail("dim must be a multiple of 16 in 16..256");
    if (stride[3] != 1) fail(std::string(names[i]) + " must have dense heads");
    const int32_t type = is == at::ScalarType::BFloat16 ? DSDE_BF16 : is == at::ScalarType::Float ? DSDE_FP32 : DSDE_E4M3;
    const int64_t e = t.element_size();
    if (reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 != 0 || stride[0] * e % 16 != 0 || stride[1] * e % 16 != 0 || stride[2] * e % 16 != 0)
      fail(std::string(names[i]) + " must have rows that start at multiples of 16 bytes");
    if (i == 0) {
      c = dsde_kv_cache{t.data_ptr(), nullptr, type, int32_t(size[0]), int32_t(size[2]), int32_t(size[1]), int32_t(size[3]),
                        stride[0], stride[1], stride[2], nullptr, nullptr};
    } else {
      if (c.dtype != type || c.pages != size[0] || c.heads != size[1] || c.page_size != size[2] || c.dim != size[3] ||
          c.page_stride != stride[0] || c.head_stride != stride[1] || c.token_stride != stride[2])
        fail("k_cache and v_cache must have one type, shape and layout");
      c.v = t.data_ptr();
    }
    if (write) written(o[i]);
  }
  const auto scale = [&](const char *name) {
    if (a.at != a.end) forward_only(*a.at, name);
    return take_on<float>(a, dev, kF32, c.heads, name);
  };
  c.k_scale = scale("k_scale");
  c.v_scale = scale("v_scale");
  if ((c.dtype == DSDE_E4M3) != (c.k_scale != nullptr) || (c.dtype == DSDE_E4M3) != (c.v_scale != nullptr))
    fail("k_scale and v_scale belong to a cache of float8_e4m3fn, and both to each");
  return c;
}
void check_rows(const dsde_kv_cache &c, const HeadRows &r, const char *name) {
  if (r.dim != c.dim) fail(std::string(name) + " must have the cache's dim");
  if (row_type(r) != (c.dtype == DSDE_E4M3 ? DSDE_BF16 : c.dtype))
    fail(std::string(name) + " must be of the cache's type, or bfloat16 for a cache of float8_e4m3fn");
}

// kv_map(sl, extra, kv_len, accepted, last_err, pool, page_size, rows, out, workspace, stream)
PyObject *py_kv_map(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    OneDevice dev;
    if (n < 1) a.next();
    const int64_t B = size_of(args[0], 0, "sl");
    const auto *sl = take_on<int32_t>(a, dev, kI32, B, "sl");
    const int32_t extra = a.int32();
    const auto *kv_len = take_on<int32_t>(a, dev, kI32, B, "kv_len"), *accepted = take_on<int32_t>(a, dev, kI32, B, "accepted");
    const auto *last_err = take_on<uint32_t>(a, dev, kErr, B, "last_err");
    PyObject *pool = a.next();
    const int64_t page = a.integer(), rows = a.integer();
    PyObject *table_o = dev.item(pool, "table"), *free_o = dev.item(pool, "free");
    const int64_t width = size_of(table_o, 1, "table"), pages = size_of(free_o, 0, "free");
    if (THPVariable_Unpack(table_o).dim() != 2 || size_of(table_o, 0, "table") != B) fail("table must be [B, width]");
    if (width > 0x7fffffff || pages > 0x7fffffff || page < 1 || page > 1024 || rows < 0 || B > 0x7fffffff)
      fail("kv_map: a size is out of range");
    auto *table = out_on<int32_t>(pool, dev, "table", kI32, B * width), *held = out_on<int32_t>(pool, dev, "held", kI32, B);
    auto *stack = out_on<int32_t>(pool, dev, "free", kI32, pages), *n_free = out_on<int32_t>(pool, dev, "n_free", kI32, 1);
    PyObject *dict = a.next();
    auto *base = out_on<int32_t>(dict, dev, "base", kI32, B), *context = out_on<int32_t>(dict, dev, "context", kI32, B);
    auto *cu = out_on<int32_t>(dict, dev, "cu_rows", kI32, B + 1);
    auto *slots = rows > 0 ? out_on<int32_t>(dict, dev, "slots", kI32, rows) : nullptr;
    auto *positions = rows > 0 ? out_on<int32_t>(dict, dev, "positions", kI32, rows) : nullptr;
    auto *err = out_on<uint32_t>(dict, dev, "seq_err", kErr, B);
    if (a.at != a.end) dev.see(*a.at, "workspace");
    size_t bytes;
    void *ws = take_workspace(a, &bytes), *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_kv_map_next(int32_t(B), int32_t(page), int32_t(pages), int32_t(width), rows, sl, extra, kv_len,
                                    accepted, last_err, table, held, stack, n_free, base, context, cu, slots, positions, err,
                                    ws, bytes, stream);
    });
  });
}

// kv_write(k, v, slots, k_cache, v_cache, k_scale, v_scale, row_err, stream)
PyObject *py_kv_write(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    OneDevice dev;
    const HeadRows k = head_rows(a.next(), dev, "k"), v = head_rows(a.next(), dev, "v");
    const auto *slots = take_on<int32_t>(a, dev, kI32, k.T, "slots");
    const dsde_kv_cache c = take_cache(a, dev, true);
    check_rows(c, k, "k");
    check_rows(c, v, "v");
    if (k.T != v.T || k.heads != c.heads || v.heads != c.heads) fail("k and v must be [rows, heads, dim] of the cache's heads");
    auto *err = take_on<uint32_t>(a, dev, kErr, k.T, "row_err", true);
    void *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_kv_write(&c, k.data, k.token_stride, k.head_stride, v.data, v.token_stride, v.head_stride, row_type(k),
                                 k.T, slots, err, stream);
    });
  });
}

// kv_attention(q, k_cache, v_cache, k_scale, v_scale, table, context, cu_rows, max_rows, scale, window, out, workspace,
//              stream); lse where out has it
PyObject *py_kv_attention(PyObject *, PyObject *const *args, Py_ssize_t n) {
  return guarded(args, n, [&](Args &a) {
    OneDevice dev;
    const HeadRows q = head_rows(a.next(), dev, "q");
    const dsde_kv_cache c = take_cache(a, dev, false);
    check_rows(c, q, "q");
    if (q.heads < 1 || q.heads % c.heads != 0) fail("q must have a multiple of the cache's heads");
    PyObject *table_o = a.next();
    dev.see(table_o, "table");
    const int64_t B = size_of(table_o, 0, "table"), width = size_of(table_o, 1, "table");
    if (THPVariable_Unpack(table_o).dim() != 2 || B > 0x7fffffff || width > 0x7fffffff) fail("table must be [B, width]");
    const auto *table = static_cast<const int32_t *>(ptr(table_o, kI32, B * width, "table"));
    const auto *context = take_on<int32_t>(a, dev, kI32, B, "context"), *cu = take_on<int32_t>(a, dev, kI32, B + 1, "cu_rows");
    const int32_t max_rows = a.int32();
    const float scale = a.real();
    const int64_t window = a.integer();
    if (window < 0 || window > 0x7fffffff) fail("window must be in 0..2^31-1");
    PyObject *dict = a.next();
    PyObject *out_o = dev.item(dict, "out");
    const HeadRows o = head_rows(out_o, dev, "out");
    if (o.T != q.T || o.heads != q.heads || o.dim != q.dim || o.type != q.type) fail("out must have the queries' shape and type");
    written(out_o);
    auto *lse = PyMapping_HasKeyString(dict, "lse") ? out_on<float>(dict, dev, "lse", kF32, q.T * q.heads) : nullptr;
    auto *err = out_on<uint32_t>(dict, dev, "seq_err", kErr, B);
    if (a.at != a.end) dev.see(*a.at, "workspace");
    size_t bytes;
    void *ws = take_workspace(a, &bytes), *stream = a.stream();
    a.done();
    call([&] {
      return g_lib.dsde_kv_attention(&c, q.data, q.token_stride, q.head_stride, row_type(q), int32_t(q.heads), q.T, int32_t(B),
                                     max_rows, table, int32_t(width), context, cu, scale, int32_t(window), o.data,
                                     o.token_stride, o.head_stride, lse, err, ws, bytes, stream);
    });
  });
}

// set_error(type): the exception the checks raise
PyObject *py_set_error(PyObject *, PyObject *type) {
  Py_INCREF(type);
  Py_XDECREF(g_error);
  g_error = type;
  Py_RETURN_NONE;
}

// set_library(handle): takes the entry points from a library's dlopen handle
PyObject *py_set_library(PyObject *, PyObject *handle) {
  void *h = PyLong_AsVoidPtr(handle);
  if (!h) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no library handle");
    return nullptr;
  }
  Library lib;
#define X(name)                                                                      \
  if (!(lib.name = reinterpret_cast<decltype(lib.name)>(dlsym(h, #name)))) {         \
    PyErr_SetString(g_error ? g_error : PyExc_RuntimeError, "libdsde lacks " #name); \
    return nullptr;                                                                  \
  }
  DSDE_ENTRIES(X)
#undef X
  g_lib = lib;
  Py_RETURN_NONE;
}

using Fast = PyObject *(*)(PyObject *, PyObject *const *, Py_ssize_t);
PyMethodDef entry(const char *name, Fast f) {
  return PyMethodDef{name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {entry("verify", py_verify),
                           entry("step", py_step),
                           entry("kld_signal", py_kld_signal),
                           entry("next_sl", py_next_sl),
                           entry("calibration_update", py_calibration_update),
                           entry("shard_stats", py_shard_stats),
                           entry("shard_accept", py_shard_accept),
                           entry("shard_draw_mass", py_shard_draw_mass),
                           entry("shard_draw_pick", py_shard_draw_pick),
                           entry("sample", py_sample),
                           entry("top_logits", py_top_logits),
                           entry("distill_loss", py_distill_loss),
                           entry("distill_grad", py_distill_grad),
                           entry("distill_step", py_distill_step),
                           entry("kv_map", py_kv_map),
                           entry("kv_write", py_kv_write),
                           entry("kv_attention", py_kv_attention),
                           {"set_error", py_set_error, METH_O, nullptr},
                           {"set_library", py_set_library, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&g_module); }
