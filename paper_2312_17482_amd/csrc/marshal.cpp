// The calls of binding.py that a training or serving step makes many times, in native code: tensors in, C ABI out.  Host
// code only.  With small batches the host's time per call is what bounds a step: in Python a call cost 1.5 to 4 us on top of
// the launch, most of it for looking at tensors (data_ptr, shape, stride) one method call at a time.
//
// Two objects (`Calls`, and `Fp8Calls` with the 8-bit calls) per imported binding, each of which holds the addresses of the C functions, the binding's error class and how to
// find the current stream.  Their methods take what the binding documents, by position or by name, and do what the C ABI does
// not: defaults, allocation of what is not given, and the checks of shapes and strides that are left once a tensor is a pointer.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <algorithm>
#include <climits>
#include <cstdint>
#include <functional>
#include <utility>

#include "mosaic_attn.h"

namespace {

// Thrown with the Python error set.
struct Raised {};

[[noreturn]] void raise(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw Raised();
}
void require(bool ok, const char* text) {
  if (!ok) raise(PyExc_AssertionError, text);
}

// What every object of calls holds.
struct Host {
  PyObject_HEAD
  PyObject* error;        // the binding's exception class: (status, message)
  PyObject* device;       // () -> current device
  PyObject* raw_stream;   // (device) -> stream handle, or None
  PyObject* stream;       // () -> stream handle, where there is no raw_stream
  decltype(&mb_last_error) last_error;
};

struct Calls : Host {
  decltype(&mb_unpad_index) unpad_index;
  decltype(&mb_unpad) unpad;
  decltype(&mb_pad) pad;
  decltype(&mb_zero_padding) zero_padding;
  decltype(&mb_alibi_attn_fwd) attn_fwd;
  decltype(&mb_alibi_attn_fwd_workspace_bytes) attn_fwd_bytes;
  decltype(&mb_alibi_attn_bwd) attn_bwd;
  decltype(&mb_alibi_attn_bwd_workspace_bytes) attn_bwd_bytes;
  decltype(&mb_add_layernorm_fwd) layernorm_fwd;
  decltype(&mb_add_layernorm_bwd) layernorm_bwd;
  decltype(&mb_add_layernorm_bwd_workspace_bytes) layernorm_bwd_bytes;
  decltype(&mb_geglu_fwd) geglu_fwd;
  decltype(&mb_geglu_bwd) geglu_bwd;
  decltype(&mb_geglu_bwd_workspace_bytes) geglu_bwd_bytes;
  decltype(&mb_linear_fwd) linear_fwd;
};

// The 8-bit calls.
struct Fp8Calls : Host {
  decltype(&mb_fp8_quant) quant;
  decltype(&mb_fp8_dequant) dequant;
  decltype(&mb_fp8_quant_weight) quant_weight;
  decltype(&mb_linear_fp8_fwd) linear;
  decltype(&mb_linear_fp8_wgrad) wgrad;
  decltype(&mb_linear_fp8_wgrad_workspace_bytes) wgrad_bytes;
  decltype(&mb_geglu_fp8_act) act;
  decltype(&mb_gelu_gate_fp8_bwd) gate_bwd;
};

// ---------------------------------------------------------------------------------------------------- arguments
// The parameters of a call: keywords arrive as interned strings, so that looking for one is comparing pointers.
template <int N>
struct Names {
  const char* text[N];
  PyObject* interned[N];
  template <typename... T>
  explicit Names(T... t) : text{t...}, interned{PyUnicode_InternFromString(t)...} {
    static_assert(sizeof...(T) == N, "as many names as parameters");
  }
  int find(PyObject* key) const {
    for (int i = 0; i < N; ++i)
      if (key == interned[i]) return i;
    for (int i = 0; i < N; ++i)
      if (PyUnicode_CompareWithASCIIString(key, text[i]) == 0) return i;
    return N;
  }
};
template <typename... T>
Names(T...) -> Names<sizeof...(T)>;

// What x.name() gives: the calls below take a bare pointer from any object that has the method.
PyObject* asked(PyObject* x, const char* name) {
  PyObject* r = PyObject_CallMethod(x, name, nullptr);
  if (!r) throw Raised();
  return r;
}

// The arguments of a call by their place in `names` (nullptr where not given).
template <int N>
struct Args {
  PyObject* v[N] = {};
  Args(const char* call, const Names<N>& names, int required, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
    if (n > N) {
      PyErr_Format(PyExc_TypeError, "%s() takes %d arguments but %zd were given", call, N, n);
      throw Raised();
    }
    for (Py_ssize_t i = 0; i < n; ++i) v[i] = args[i];
    const Py_ssize_t nk = kw ? PyTuple_GET_SIZE(kw) : 0;
    for (Py_ssize_t j = 0; j < nk; ++j) {
      PyObject* key = PyTuple_GET_ITEM(kw, j);
      const int at = names.find(key);
      if (at == N) {
        PyErr_Format(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", call, key);
        throw Raised();
      }
      if (v[at]) {
        PyErr_Format(PyExc_TypeError, "%s() got multiple values for argument '%s'", call, names.text[at]);
        throw Raised();
      }
      v[at] = args[n + j];
    }
    for (int i = 0; i < required; ++i)
      if (!v[i]) {
        PyErr_Format(PyExc_TypeError, "%s() missing required argument '%s'", call, names.text[i]);
        throw Raised();
      }
  }
  bool given(int i) const { return v[i] && v[i] != Py_None; }
  const at::Tensor& tensor(int i) const {
    if (!THPVariable_Check(v[i])) {
      PyErr_Format(PyExc_TypeError, "argument %d must be a tensor, not %s", i + 1, Py_TYPE(v[i])->tp_name);
      throw Raised();
    }
    return THPVariable_Unpack(v[i]);
  }
  void* ptr(int i) const {
    if (!given(i)) return nullptr;
    if (THPVariable_Check(v[i])) return THPVariable_Unpack(v[i]).data_ptr();
    PyObject* r = asked(v[i], "data_ptr");
    void* p = r == Py_None ? nullptr : PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    if (!p && PyErr_Occurred()) throw Raised();
    return p;
  }
  int64_t numel(int i) const {
    if (THPVariable_Check(v[i])) return THPVariable_Unpack(v[i]).numel();
    PyObject* r = asked(v[i], "numel");
    const int64_t n = PyLong_AsLongLong(r);
    Py_DECREF(r);
    if (n == -1 && PyErr_Occurred()) throw Raised();
    return n;
  }
  bool contiguous(int i) const {
    if (THPVariable_Check(v[i])) return THPVariable_Unpack(v[i]).is_contiguous();
    PyObject* r = asked(v[i], "is_contiguous");
    const int yes = PyObject_IsTrue(r);
    Py_DECREF(r);
    if (yes < 0) throw Raised();
    return yes;
  }
  int integer(int i) const {   // as ctypes converts to a C int
    PyObject* x = PyNumber_Index(v[i]);
    if (!x) throw Raised();
    const unsigned long u = PyLong_AsUnsignedLongMask(x);
    Py_DECREF(x);
    if (u == (unsigned long)-1 && PyErr_Occurred()) throw Raised();
    return (int)u;
  }
  int integer_or(int i, int64_t otherwise) const { return given(i) ? integer(i) : (int)otherwise; }
  float number(int i) const {
    PyObject* x = PyNumber_Float(v[i]);
    if (!x) throw Raised();
    const double d = PyFloat_AS_DOUBLE(x);
    Py_DECREF(x);
    return (float)d;
  }
};

// A result: the object that was given, or a tensor made here.
struct Result {
  PyObject* object = nullptr;   // borrowed, if given
  at::Tensor made;
  void* ptr = nullptr;
  template <typename A, typename Make>
  Result(const A& a, int i, Make make) {
    if (a.given(i)) {
      object = a.v[i];
      ptr = a.ptr(i);
    } else {
      made = make();
      ptr = made.data_ptr();
    }
  }
  template <typename A>
  const at::Tensor& tensor(const A& a, int i) const { return object ? a.tensor(i) : made; }
  template <typename A>
  size_t numel(const A& a, int i) const { return (size_t)(object ? a.numel(i) : made.numel()); }
  PyObject* take() {
    if (object) {
      Py_INCREF(object);
      return object;
    }
    return THPVariable_Wrap(std::move(made));
  }
};

template <typename... R>
PyObject* tuple_of(R&&... results) {
  PyObject* t = PyTuple_New(sizeof...(results));
  if (!t) throw Raised();
  Py_ssize_t i = 0;
  auto put = [&](PyObject* x) {
    if (!x) {
      Py_DECREF(t);
      throw Raised();
    }
    PyTuple_SET_ITEM(t, i++, x);
  };
  (put(results), ...);
  return t;
}

int dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return MB_BF16;
  if (t.scalar_type() == at::kFloat) return MB_F32;
  const std::string text = std::string("unsupported dtype ") + c10::toString(t.scalar_type());
  raise(PyExc_TypeError, text.c_str());
}

// [T, H, D] view with dense (H, D): the token stride in elements.
int64_t row_stride(const at::Tensor& t) {
  require(t.dim() == 3 && t.stride(2) == 1 && t.stride(1) == t.size(2), "need [T, H, D] with dense (H, D)");
  return t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1) * t.size(2));
}

at::Tensor new_like(const at::Tensor& like, at::IntArrayRef sizes, at::ScalarType type) {
  return at::empty(sizes, like.options().dtype(type).requires_grad(false));
}
at::Tensor new_bytes(const at::Tensor& like, size_t n) { return new_like(like, {(int64_t)n}, at::kByte); }

void* current_stream(const Host* s) {
  PyObject* handle;
  if (s->raw_stream == Py_None) {
    handle = PyObject_CallNoArgs(s->stream);
  } else {
    PyObject* device = PyObject_CallNoArgs(s->device);
    if (!device) throw Raised();
    handle = PyObject_CallOneArg(s->raw_stream, device);
    Py_DECREF(device);
  }
  if (!handle) throw Raised();
  void* p = handle == Py_None ? nullptr : PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  if (!p && PyErr_Occurred()) throw Raised();
  return p;
}

// Runs the C function without the interpreter's lock, as ctypes does.
template <typename F, typename... A>
void run(const Host* s, F function, A... args) {
  mb_status status;
  Py_BEGIN_ALLOW_THREADS
  status = function(args...);
  Py_END_ALLOW_THREADS
  if (status == MB_OK) return;
  PyObject* e = PyObject_CallFunction(s->error, "is", (int)status, s->last_error());
  if (e) {
    PyErr_SetObject(s->error, e);
    Py_DECREF(e);
  }
  throw Raised();
}

// ---------------------------------------------------------------------------------------------------- the calls
using Self = const Calls*;
using Argv = PyObject* const*;

PyObject* unpad_index(Self s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("mask");
  const Args<1> a("mb_unpad_index", names, 1, argv, n, kw);
  const at::Tensor& mask = a.tensor(0);
  require(mask.scalar_type() == at::kInt && mask.dim() == 2 && mask.is_contiguous(), "need a contiguous [B, L] int32 mask");
  const int64_t B = mask.size(0), L = mask.size(1);
  auto make = [&](int64_t count) { return new_like(mask, {count}, at::kInt); };
  at::Tensor seqlens = B > 0 ? make(B) : make(1).slice(0, 0, 0), cu = make(B + 1),
             indices = B * L > 0 ? make(B * L) : make(1).slice(0, 0, 0), meta = make(2);
  void* const stream = current_stream(s);
  run(s, s->unpad_index, (const int32_t*)mask.data_ptr(), (int)B, (int)L, (int32_t*)seqlens.data_ptr(),
      (int32_t*)cu.data_ptr(), (int32_t*)indices.data_ptr(), (int32_t*)meta.data_ptr(), stream);
  return tuple_of(THPVariable_Wrap(std::move(seqlens)), THPVariable_Wrap(std::move(cu)), THPVariable_Wrap(std::move(indices)),
                  THPVariable_Wrap(std::move(meta)));
}

PyObject* unpad(Self s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("padded", "indices", "T_cap", "meta", "out");
  const Args<5> a("mb_unpad", names, 4, argv, n, kw);
  const at::Tensor& padded = a.tensor(0);
  require(padded.dim() == 2 && padded.is_contiguous(), "padded must be a contiguous matrix");
  const int64_t W = padded.size(1);
  const int T_cap = a.integer(2);
  Result out(a, 4, [&] { return new_like(padded, {T_cap, W}, padded.scalar_type()); });
  const at::Tensor& o = out.tensor(a, 4);
  require(o.is_contiguous() && o.dim() >= 2 && o.size(1) == W && o.size(0) >= T_cap, "out must be contiguous, [>= T_cap, W]");
  const mb_dtype dt = (mb_dtype)dtype_code(padded);
  void* const stream = current_stream(s);
  run(s, s->unpad, padded.data_ptr(), (const int32_t*)a.ptr(1), T_cap, (const int32_t*)a.ptr(3), (int)W,
      dt, out.ptr, stream);
  return out.take();
}

PyObject* pad(Self s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("packed", "indices", "T_cap", "meta", "B", "L", "out");
  const Args<7> a("mb_pad", names, 6, argv, n, kw);
  const at::Tensor& packed = a.tensor(0);
  require(packed.dim() == 2 && packed.is_contiguous(), "packed must be a contiguous matrix");
  const int64_t W = packed.size(1);
  const int B = a.integer(4), L = a.integer(5);
  Result out(a, 6, [&] { return new_like(packed, {(int64_t)B * L, W}, packed.scalar_type()); });
  const at::Tensor& o = out.tensor(a, 6);
  require(o.is_contiguous() && o.dim() == 2 && o.size(0) == (int64_t)B * L && o.size(1) == W, "out must be contiguous, [B * L, W]");
  const mb_dtype dt = (mb_dtype)dtype_code(packed);
  void* const stream = current_stream(s);
  run(s, s->pad, packed.data_ptr(), (const int32_t*)a.ptr(1), a.integer(2), (const int32_t*)a.ptr(3), B, L, (int)W,
      dt, out.ptr, stream);
  return out.take();
}

PyObject* zero_padding(Self s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("padded", "indices", "T_cap", "meta", "B", "L");
  const Args<6> a("mb_zero_padding", names, 6, argv, n, kw);
  const at::Tensor& padded = a.tensor(0);
  const int B = a.integer(4), L = a.integer(5);
  require(padded.dim() == 2 && padded.is_contiguous() && padded.size(0) == (int64_t)B * L, "padded must be contiguous, [B * L, W]");
  const mb_dtype dt = (mb_dtype)dtype_code(padded);
  void* const stream = current_stream(s);
  run(s, s->zero_padding, (const int32_t*)a.ptr(1), a.integer(2), (const int32_t*)a.ptr(3), B, L, (int)padded.size(1),
      dt, padded.data_ptr(), stream);
  Py_INCREF(a.v[0]);
  return a.v[0];
}

// [T, H, D] of q: what an attention call takes its sizes from.
void attention_sizes(const at::Tensor& q, int64_t* R, int64_t* H, int64_t* D) {
  if (q.dim() != 3) raise(PyExc_ValueError, "q must be [T, H, D]");
  *R = q.size(0);
  *H = q.size(1);
  *D = q.size(2);
}

PyObject* attn_fwd(Self s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("q", "k", "v", "cu_seqlens", "max_seqlen", "slopes", "softmax_scale", "out", "lse",
                                      "token_rows", "T", "workspace", "key_lens", "plan");
  const Args<14> a("mb_alibi_attn_fwd", names, 7, argv, n, kw);
  const at::Tensor &q = a.tensor(0), &k = a.tensor(1), &v = a.tensor(2);
  int64_t R, H, D;
  attention_sizes(q, &R, &H, &D);
  const int T = a.integer_or(10, R), max_seqlen = a.integer(4), B = (int)(a.numel(3) - 1);
  Result out(a, 7, [&] { return new_like(q, {R, H, D}, q.scalar_type()); });
  Result lse(a, 8, [&] { return new_like(q, {H, T}, at::kFloat); });
  const mb_dtype dt = (mb_dtype)dtype_code(q);
  at::Tensor own;
  void* workspace = a.ptr(11);
  size_t workspace_bytes = a.given(11) ? (size_t)a.numel(11) : 0;
  if (!a.given(11) && !a.given(13)) {
    workspace_bytes = s->attn_fwd_bytes(B, T, max_seqlen, (int)H, (int)D, dt);
    if (workspace_bytes > 0) {
      own = new_bytes(q, workspace_bytes);
      workspace = own.data_ptr();
    }
  }
  void* const stream = current_stream(s);
  run(s, s->attn_fwd, (const void*)q.data_ptr(), (const void*)k.data_ptr(), (const void*)v.data_ptr(), row_stride(q),
      row_stride(k), row_stride(v), (const int32_t*)a.ptr(3), B, T, max_seqlen, (int)H, (int)D,
      (const float*)a.ptr(5), a.number(6), dt, out.ptr, row_stride(out.tensor(a, 7)), (float*)lse.ptr, workspace, workspace_bytes,
      (const int32_t*)a.ptr(12), (const int32_t*)a.ptr(9), (const void*)a.ptr(13), stream);
  return tuple_of(out.take(), lse.take());
}

PyObject* attn_bwd(Self s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("dout", "q", "k", "v", "o", "lse", "cu_seqlens", "max_seqlen", "slopes",
                                      "softmax_scale", "dq", "dk", "dv", "workspace", "token_rows", "T", "key_lens", "plan");
  const Args<18> a("mb_alibi_attn_bwd", names, 10, argv, n, kw);
  const at::Tensor &dout = a.tensor(0), &q = a.tensor(1), &k = a.tensor(2), &v = a.tensor(3), &o = a.tensor(4);
  int64_t R, H, D;
  attention_sizes(q, &R, &H, &D);
  const int T = a.integer_or(15, R), max_seqlen = a.integer(7), B = (int)(a.numel(6) - 1);
  auto make = [&] { return new_like(q, {R, H, D}, q.scalar_type()); };
  Result dq(a, 10, make), dk(a, 11, make), dv(a, 12, make);
  const mb_dtype dt = (mb_dtype)dtype_code(q);
  Result workspace(a, 13, [&] {
    return new_bytes(q, std::max<size_t>(s->attn_bwd_bytes(B, T, max_seqlen, (int)H, (int)D, dt), 16));
  });
  void* const stream = current_stream(s);
  run(s, s->attn_bwd, (const void*)dout.data_ptr(), (const void*)q.data_ptr(), (const void*)k.data_ptr(),
      (const void*)v.data_ptr(), (const void*)o.data_ptr(), (const float*)a.ptr(5), row_stride(dout), row_stride(q),
      row_stride(k), row_stride(v), row_stride(o), (const int32_t*)a.ptr(6), B, T, max_seqlen, (int)H, (int)D,
      (const float*)a.ptr(8), a.number(9), dt, dq.ptr, dk.ptr, dv.ptr, row_stride(dq.tensor(a, 10)), row_stride(dk.tensor(a, 11)),
      row_stride(dv.tensor(a, 12)), workspace.ptr, workspace.numel(a, 13), (const int32_t*)a.ptr(16),
      (const int32_t*)a.ptr(14), (const void*)a.ptr(17), stream);
  return tuple_of(dq.take(), dk.take(), dv.take());
}

PyObject* layernorm_fwd(Self s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("x", "r", "gamma", "beta", "eps", "T_cap", "meta", "y", "s", "mean", "rstd", "y_rows");
  const Args<12> a("mb_add_layernorm_fwd", names, 5, argv, n, kw);
  const at::Tensor& x = a.tensor(0);
  require(x.dim() == 2 && x.is_contiguous(), "x must be a contiguous matrix");
  require(!a.given(11) || a.given(7), "y_rows needs y");
  const int64_t rows = x.size(0), W = x.size(1);
  auto like = [&] { return new_like(x, {rows, W}, x.scalar_type()); };
  auto per_row = [&] { return new_like(x, {rows}, at::kFloat); };
  const bool add = a.given(1);
  Result y(a, 7, like);
  Result sum(a, add ? 8 : 0, like);   // without r the sum is x itself
  Result mean(a, 9, per_row), rstd(a, 10, per_row);
  const mb_dtype dt = (mb_dtype)dtype_code(x);
  void* const stream = current_stream(s);
  run(s, s->layernorm_fwd, (const void*)x.data_ptr(), (const void*)a.ptr(1), (const void*)a.ptr(2), (const void*)a.ptr(3),
      a.integer_or(5, rows), (const int32_t*)a.ptr(6), (int)W, a.number(4), dt, y.ptr,
      add ? sum.ptr : nullptr, (float*)mean.ptr, (float*)rstd.ptr, (const int32_t*)a.ptr(11), stream);
  return tuple_of(y.take(), sum.take(), mean.take(), rstd.take());
}

PyObject* layernorm_bwd(Self s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("dy", "s", "gamma", "mean", "rstd", "T_cap", "meta", "ds", "dgamma", "dbeta",
                                      "workspace", "dy_rows");
  const Args<12> a("mb_add_layernorm_bwd", names, 5, argv, n, kw);
  const at::Tensor& sum = a.tensor(1);
  if (sum.dim() != 2) raise(PyExc_ValueError, "s must be a matrix");
  const int64_t rows = sum.size(0), W = sum.size(1);
  auto column = [&] { return new_like(sum, {W}, at::kFloat); };
  Result ds(a, 7, [&] { return at::empty_like(sum, sum.options().requires_grad(false)); });
  Result dgamma(a, 8, column), dbeta(a, 9, column);
  Result workspace(a, 10, [&] { return new_bytes(sum, s->layernorm_bwd_bytes((int)W)); });
  const mb_dtype dt = (mb_dtype)dtype_code(sum);
  void* const stream = current_stream(s);
  run(s, s->layernorm_bwd, (const void*)a.ptr(0), (const void*)sum.data_ptr(), (const void*)a.ptr(2), (const float*)a.ptr(3),
      (const float*)a.ptr(4), a.integer_or(5, rows), (const int32_t*)a.ptr(6), (int)W, dt, ds.ptr,
      (float*)dgamma.ptr, (float*)dbeta.ptr, workspace.ptr, workspace.numel(a, 10), (const int32_t*)a.ptr(11),
      stream);
  return tuple_of(ds.take(), dgamma.take(), dbeta.take());
}

PyObject* geglu_fwd(Self s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("x", "w1v", "w2", "T_cap", "meta", "act", "y");
  const Args<7> a("mb_geglu_fwd", names, 3, argv, n, kw);
  const at::Tensor &x = a.tensor(0), &w1v = a.tensor(1), &w2 = a.tensor(2);
  require(x.dim() == 2 && x.is_contiguous() && w1v.is_contiguous() && w2.is_contiguous(), "x, w1v and w2 must be contiguous");
  require(w1v.dim() == 2 && w2.dim() == 2, "w1v and w2 must be matrices");
  const int64_t rows = x.size(0), hidden = x.size(1), inter = w2.size(1);
  require(w1v.size(0) == 2 * inter && w1v.size(1) == hidden && w2.size(0) == hidden, "w1v [2 inter, hidden], w2 [hidden, inter]");
  Result act(a, 5, [&] { return new_like(x, {rows, inter}, x.scalar_type()); });
  Result y(a, 6, [&] { return new_like(x, {rows, hidden}, x.scalar_type()); });
  const mb_dtype dt = (mb_dtype)dtype_code(x);
  void* const stream = current_stream(s);
  run(s, s->geglu_fwd, (const void*)x.data_ptr(), (const void*)w1v.data_ptr(), (const void*)w2.data_ptr(),
      a.integer_or(3, rows), (const int32_t*)a.ptr(4), (int)hidden, (int)inter, dt, act.ptr, y.ptr,
      stream);
  return tuple_of(y.take(), act.take());
}

PyObject* geglu_bwd(Self s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("dy", "x", "w1v", "w2", "act", "hg", "T_cap", "meta", "dx", "dw1v", "dw2", "workspace");
  const Args<12> a("mb_geglu_bwd", names, 5, argv, n, kw);
  require(!a.given(5) || a.contiguous(5), "hg must be contiguous");
  const at::Tensor &x = a.tensor(1), &w2 = a.tensor(3);
  if (x.dim() != 2) raise(PyExc_ValueError, "x must be a matrix");
  if (w2.dim() < 2) raise(PyExc_IndexError, "w2 must be a matrix");
  const int64_t rows = x.size(0), hidden = x.size(1), inter = w2.size(1);
  const int T_cap = a.integer_or(6, rows);
  const mb_dtype dt = (mb_dtype)dtype_code(x);
  Result dx(a, 8, [&] { return at::empty_like(x, x.options().requires_grad(false)); });
  Result dw1v(a, 9, [&] { return new_like(x, {2 * inter, hidden}, at::kFloat); });
  Result dw2(a, 10, [&] { return new_like(x, {hidden, inter}, at::kFloat); });
  Result workspace(a, 11, [&] {
    return new_bytes(x, std::max<size_t>(s->geglu_bwd_bytes(T_cap, (int)hidden, (int)inter, dt), 256));
  });
  void* const stream = current_stream(s);
  run(s, s->geglu_bwd, (const void*)a.ptr(0), (const void*)x.data_ptr(), (const void*)a.ptr(2), (const void*)w2.data_ptr(),
      (const void*)a.ptr(4), (const void*)a.ptr(5), T_cap, (const int32_t*)a.ptr(7), (int)hidden, (int)inter, dt, dx.ptr,
      (float*)dw1v.ptr, (float*)dw2.ptr, workspace.ptr, workspace.numel(a, 11), stream);
  return tuple_of(dx.take(), dw1v.take(), dw2.take());
}

PyObject* linear_fwd(Self s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("x", "wt", "T_cap", "meta", "y");
  const Args<5> a("mb_linear_fwd", names, 2, argv, n, kw);
  const at::Tensor &x = a.tensor(0), &wt = a.tensor(1);
  require(x.dim() == 2 && x.is_contiguous() && wt.is_contiguous() && wt.dim() >= 2 && wt.size(1) == x.size(1),
          "x and wt must be contiguous, with as many columns");
  const int64_t rows = x.size(0), n_in = x.size(1), n_out = wt.size(0);
  Result y(a, 4, [&] { return new_like(x, {rows, n_out}, x.scalar_type()); });
  const mb_dtype dt = (mb_dtype)dtype_code(x);
  void* const stream = current_stream(s);
  run(s, s->linear_fwd, (const void*)x.data_ptr(), (const void*)wt.data_ptr(), a.integer_or(2, rows), (const int32_t*)a.ptr(3),
      (int)n_in, (int)n_out, dt, y.ptr, stream);
  return y.take();
}

// ---------------------------------------------------------------------------------------------------- the 8-bit calls
using Self8 = const Fp8Calls*;
constexpr int64_t kBlock = 128;
int64_t blocks_of(int64_t width) { return (width + kBlock - 1) / kBlock; }

// Tensors of one call: on one device, which is the current one (its stream is what the call goes to).
template <typename... T>
void together(Self8 s, const at::Tensor& first, const T&... others) {
  require(((others.device() == first.device()) && ...), "all tensors must be on one device");
  if (!first.is_cuda()) return;
  PyObject* r = PyObject_CallNoArgs(s->device);
  if (!r) throw Raised();
  const long device = PyLong_AsLong(r);
  Py_DECREF(r);
  if (device == -1 && PyErr_Occurred()) throw Raised();
  require(device == first.get_device(), "the tensors must be on the current device");
}

void codes(const at::Tensor& q) {
  require(q.scalar_type() == at::kFloat8_e4m3fn && q.dim() == 2 && q.is_contiguous(), "8-bit values must be a contiguous float8_e4m3fn matrix");
}
// 8-bit rows (or, block = 128, a weight) and their scales.
void stored(const at::Tensor& q, const at::Tensor& s, int64_t block = 1) {
  codes(q);
  require(s.scalar_type() == at::kFloat8_e8m0fnu && s.dim() == 2 && s.is_contiguous() && s.size(0) == (q.size(0) + block - 1) / block &&
              s.size(1) == blocks_of(q.size(1)),
          "scales must be a contiguous float8_e8m0fnu matrix with one value for each block of 128");
}
at::Tensor new_codes(const at::Tensor& like, int64_t rows, int64_t width) { return new_like(like, {rows, width}, at::kFloat8_e4m3fn); }
at::Tensor new_scales(const at::Tensor& like, int64_t rows, int64_t width) {
  return new_like(like, {rows, blocks_of(width)}, at::kFloat8_e8m0fnu);
}
// [rows, W] view with dense rows: the row stride in elements.
int64_t matrix_stride(const at::Tensor& t) {
  require(t.dim() == 2 && (t.stride(1) == 1 || t.size(1) <= 1), "need a matrix with dense rows");
  return t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1));
}
// A size as the library takes it: one that is no int is too large for it in any case.
int size_of(int64_t n) { return (int)std::clamp<int64_t>(n, INT_MIN, INT_MAX); }
template <int N>
int rows_used(const Args<N>& a, int i, int64_t rows) {
  if (!a.given(i)) return size_of(rows);
  PyObject* x = PyNumber_Index(a.v[i]);
  if (!x) throw Raised();
  const long long T_cap = PyLong_AsLongLong(x);
  Py_DECREF(x);
  if (T_cap == -1 && PyErr_Occurred()) throw Raised();
  require(T_cap <= rows, "T_cap is more rows than there are");
  return size_of(T_cap);
}
// The row count on the device.  (A tensor; of an object that only has a pointer nothing more is known.)
template <int N>
const int32_t* meta_of(const Args<N>& a, int i, const at::Tensor& like) {
  if (a.given(i) && THPVariable_Check(a.v[i])) {
    const at::Tensor& m = a.tensor(i);
    require(m.scalar_type() == at::kInt && m.numel() > 0 && m.device() == like.device(), "meta must be int32, on the tensors' device");
  }
  return (const int32_t*)a.ptr(i);
}

PyObject* quant(Self8 s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("x", "T_cap", "meta", "q", "s");
  const Args<5> a("mb_fp8_quant", names, 1, argv, n, kw);
  const at::Tensor& x = a.tensor(0);
  const int64_t stride = matrix_stride(x), rows = x.size(0), W = x.size(1);
  const int T_cap = rows_used(a, 1, rows);
  const mb_dtype dt = (mb_dtype)dtype_code(x);
  Result q(a, 3, [&] { return new_codes(x, rows, W); });
  Result sc(a, 4, [&] { return new_scales(x, rows, W); });
  stored(q.tensor(a, 3), sc.tensor(a, 4));
  require(q.tensor(a, 3).size(0) >= T_cap && q.tensor(a, 3).size(1) == W, "q must have x's columns and as many rows as are used");
  together(s, x, q.tensor(a, 3), sc.tensor(a, 4));
  run(s, s->quant, (const void*)x.data_ptr(), stride, T_cap, meta_of(a, 2, x), size_of(W), dt, (uint8_t*)q.ptr, (uint8_t*)sc.ptr,
      current_stream(s));
  return tuple_of(q.take(), sc.take());
}

// A torch dtype argument, or bfloat16.
template <int N>
at::ScalarType type_or_bf16(const Args<N>& a, int i) {
  if (!a.given(i)) return at::kBFloat16;
  if (!THPDtype_Check(a.v[i])) raise(PyExc_TypeError, "dtype must be a torch.dtype");
  return reinterpret_cast<THPDtype*>(a.v[i])->scalar_type;
}

PyObject* dequant(Self8 s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("q", "s", "dtype", "T_cap", "meta", "out");
  const Args<6> a("mb_fp8_dequant", names, 2, argv, n, kw);
  const at::Tensor &q = a.tensor(0), &sc = a.tensor(1);
  stored(q, sc);
  const int64_t rows = q.size(0), W = q.size(1);
  const int T_cap = rows_used(a, 3, rows);
  Result out(a, 5, [&] { return new_like(q, {rows, W}, type_or_bf16(a, 2)); });
  const at::Tensor& o = out.tensor(a, 5);
  const int64_t stride = matrix_stride(o);
  require(o.size(0) >= T_cap && o.size(1) == W, "out must have q's columns and as many rows as are used");
  require(!a.given(2) || o.scalar_type() == type_or_bf16(a, 2), "out is of another dtype");
  together(s, q, sc, o);
  run(s, s->dequant, (const uint8_t*)q.data_ptr(), (const uint8_t*)sc.data_ptr(), T_cap, meta_of(a, 4, q), size_of(W),
      (mb_dtype)dtype_code(o), out.ptr, stride, current_stream(s));
  return out.take();
}

PyObject* quant_weight(Self8 s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("w", "transposed", "q", "s", "qt", "st");
  const Args<6> a("mb_fp8_quant_weight", names, 1, argv, n, kw);
  const at::Tensor& w = a.tensor(0);
  require(w.dim() == 2 && w.is_contiguous(), "w must be a contiguous matrix");
  const int64_t n_out = w.size(0), n_in = w.size(1);
  const int both = a.given(1) ? PyObject_IsTrue(a.v[1]) : 1;
  if (both < 0) throw Raised();
  const mb_dtype dt = (mb_dtype)dtype_code(w);
  const bool given_t = a.given(4) || a.given(5);
  require(both || !given_t, "qt and st are outputs of transposed=True");
  Result q(a, 2, [&] { return new_codes(w, n_out, n_in); });
  Result sc(a, 3, [&] { return new_scales(w, blocks_of(n_out), n_in); });
  Result qt(a, 4, [&] { return new_codes(w, both ? n_in : 0, n_out); });
  Result st(a, 5, [&] { return new_scales(w, both ? blocks_of(n_in) : 0, n_out); });
  stored(q.tensor(a, 2), sc.tensor(a, 3), kBlock);
  stored(qt.tensor(a, 4), st.tensor(a, 5), kBlock);
  require(q.tensor(a, 2).sizes() == w.sizes(), "q must have w's shape");
  require(!both || (qt.tensor(a, 4).size(0) == n_in && qt.tensor(a, 4).size(1) == n_out), "qt must have w's shape transposed");
  together(s, w, q.tensor(a, 2), sc.tensor(a, 3), qt.tensor(a, 4), st.tensor(a, 5));
  run(s, s->quant_weight, (const void*)w.data_ptr(), size_of(n_out), size_of(n_in), dt, (uint8_t*)q.ptr, (uint8_t*)sc.ptr,
      both ? (uint8_t*)qt.ptr : nullptr, both ? (uint8_t*)st.ptr : nullptr, current_stream(s));
  if (!both) return tuple_of(q.take(), sc.take());
  return tuple_of(q.take(), sc.take(), qt.take(), st.take());
}

PyObject* linear(Self8 s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("xq", "xs", "wq", "ws", "dtype", "T_cap", "meta", "y");
  const Args<8> a("mb_linear_fp8_fwd", names, 4, argv, n, kw);
  const at::Tensor &xq = a.tensor(0), &xs = a.tensor(1), &wq = a.tensor(2), &ws = a.tensor(3);
  stored(xq, xs);
  stored(wq, ws, kBlock);
  const int64_t rows = xq.size(0), n_in = xq.size(1), n_out = wq.size(0);
  require(wq.size(1) == n_in, "the weight must have as many columns as the rows");
  const int T_cap = rows_used(a, 5, rows);
  Result y(a, 7, [&] { return new_like(xq, {rows, n_out}, type_or_bf16(a, 4)); });
  const at::Tensor& o = y.tensor(a, 7);
  const int64_t stride = matrix_stride(o);
  require(o.size(0) >= T_cap && o.size(1) == n_out, "y must have the weight's rows as columns and as many rows as are used");
  require(!a.given(4) || o.scalar_type() == type_or_bf16(a, 4), "y is of another dtype");
  together(s, xq, xs, wq, ws, o);
  run(s, s->linear, (const uint8_t*)xq.data_ptr(), (const uint8_t*)xs.data_ptr(), (const uint8_t*)wq.data_ptr(),
      (const uint8_t*)ws.data_ptr(), T_cap, meta_of(a, 6, xq), size_of(n_in), size_of(n_out), (mb_dtype)dtype_code(o), y.ptr, stride,
      current_stream(s));
  return y.take();
}

PyObject* wgrad(Self8 s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("dy", "xq", "xs", "dys", "T_cap", "meta", "dw", "workspace");
  const Args<8> a("mb_linear_fp8_wgrad", names, 3, argv, n, kw);
  const at::Tensor &dy = a.tensor(0), &xq = a.tensor(1), &xs = a.tensor(2);
  const bool eight = a.given(3);
  stored(xq, xs);
  if (eight) stored(dy, a.tensor(3));
  else require(dy.scalar_type() == at::kBFloat16, "dy must be bfloat16, or 8-bit rows with dys");
  const int64_t stride = matrix_stride(dy), rows = xq.size(0), n_in = xq.size(1), n_out = dy.size(1);
  const int T_cap = rows_used(a, 4, std::min(rows, dy.size(0)));
  require(a.given(4) || dy.size(0) == rows, "dy must have as many rows as the stored ones");
  Result dw(a, 6, [&] { return new_like(xq, {n_out, n_in}, at::kFloat); });
  const at::Tensor& o = dw.tensor(a, 6);
  require(o.scalar_type() == at::kFloat && o.dim() == 2 && o.is_contiguous() && o.size(0) == n_out && o.size(1) == n_in,
          "dw must be a contiguous float32 matrix [columns of dy, columns of x]");
  const size_t need = a.given(7) ? 0 : s->wgrad_bytes(T_cap, size_of(n_in), size_of(n_out));
  Result workspace(a, 7, [&] { return new_bytes(xq, need); });
  if (a.given(7) && THPVariable_Check(a.v[7]))
    require(a.tensor(7).device() == xq.device() && a.tensor(7).is_contiguous(), "workspace must be contiguous, on the tensors' device");
  if (eight) together(s, dy, a.tensor(3), xq, xs, o);
  else together(s, dy, xq, xs, o);
  run(s, s->wgrad, (const void*)dy.data_ptr(), eight ? (const uint8_t*)a.ptr(3) : nullptr, eight ? n_out : stride,
      (const uint8_t*)xq.data_ptr(), (const uint8_t*)xs.data_ptr(), T_cap, meta_of(a, 5, xq), size_of(n_in), size_of(n_out), (float*)dw.ptr,
      workspace.ptr, workspace.numel(a, 7), current_stream(s));
  return dw.take();
}

PyObject* geglu_act(Self8 s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("xq", "xs", "w1vq", "w1vs", "T_cap", "meta", "actq", "acts");
  const Args<8> a("mb_geglu_fp8_act", names, 4, argv, n, kw);
  const at::Tensor &xq = a.tensor(0), &xs = a.tensor(1), &wq = a.tensor(2), &ws = a.tensor(3);
  stored(xq, xs);
  stored(wq, ws, kBlock);
  const int64_t rows = xq.size(0), hidden = xq.size(1), inter = wq.size(0) / 2;
  require(wq.size(1) == hidden && wq.size(0) % 2 == 0, "w1vq must be [2 * inter, columns of xq]");
  const int T_cap = rows_used(a, 4, rows);
  Result q(a, 6, [&] { return new_codes(xq, rows, inter); });
  Result sc(a, 7, [&] { return new_scales(xq, rows, inter); });
  stored(q.tensor(a, 6), sc.tensor(a, 7));
  require(q.tensor(a, 6).size(0) >= T_cap && q.tensor(a, 6).size(1) == inter, "actq must have inter columns and as many rows as are used");
  together(s, xq, xs, wq, ws, q.tensor(a, 6), sc.tensor(a, 7));
  run(s, s->act, (const uint8_t*)xq.data_ptr(), (const uint8_t*)xs.data_ptr(), (const uint8_t*)wq.data_ptr(),
      (const uint8_t*)ws.data_ptr(), T_cap, meta_of(a, 5, xq), size_of(hidden), size_of(inter), (uint8_t*)q.ptr, (uint8_t*)sc.ptr,
      current_stream(s));
  return tuple_of(q.take(), sc.take());
}

PyObject* gate_bwd(Self8 s, Argv argv, Py_ssize_t n, PyObject* kw) {
  static const Names names("da", "hg", "hgs", "T_cap", "meta", "dhgq", "dhgs");
  const Args<7> a("mb_gelu_gate_fp8_bwd", names, 2, argv, n, kw);
  const at::Tensor &da = a.tensor(0), &hg = a.tensor(1);
  const bool eight = a.given(2);
  require(da.scalar_type() == at::kBFloat16 && da.dim() == 2 && da.is_contiguous(), "da must be a contiguous bfloat16 matrix");
  if (eight) stored(hg, a.tensor(2));
  else require(hg.scalar_type() == at::kBFloat16 && hg.dim() == 2 && hg.is_contiguous(), "hg must be contiguous bfloat16, or 8-bit rows with hgs");
  const int64_t rows = da.size(0), inter = da.size(1);
  require(hg.size(0) == rows && hg.size(1) == 2 * inter, "hg must be [rows of da, 2 * inter]");
  const int T_cap = rows_used(a, 3, rows);
  Result q(a, 5, [&] { return new_codes(da, rows, 2 * inter); });
  Result sc(a, 6, [&] { return new_scales(da, rows, 2 * inter); });
  stored(q.tensor(a, 5), sc.tensor(a, 6));
  require(q.tensor(a, 5).size(0) >= T_cap && q.tensor(a, 5).size(1) == 2 * inter, "dhgq must have 2 * inter columns and as many rows as are used");
  if (eight) together(s, da, hg, a.tensor(2), q.tensor(a, 5), sc.tensor(a, 6));
  else together(s, da, hg, q.tensor(a, 5), sc.tensor(a, 6));
  run(s, s->gate_bwd, (const void*)da.data_ptr(), (const void*)hg.data_ptr(), eight ? (const uint8_t*)a.ptr(2) : nullptr, T_cap,
      meta_of(a, 4, da), size_of(inter), (uint8_t*)q.ptr, (uint8_t*)sc.ptr, current_stream(s));
  return tuple_of(q.take(), sc.take());
}

// ---------------------------------------------------------------------------------------------------- the object
// No C++ exception leaves a method.
template <typename C, PyObject* (*F)(const C*, Argv, Py_ssize_t, PyObject*)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n, PyObject* kw) {
  HANDLE_TH_ERRORS
  try {
    return F(reinterpret_cast<const C*>(self), args, n, kw);
  } catch (const Raised&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
template <typename C, PyObject* (*F)(const C*, Argv, Py_ssize_t, PyObject*)>
PyCFunction method() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<C, F>));
}
#define MB_METHOD(name, f, doc) {name, method<Calls, f>(), METH_FASTCALL | METH_KEYWORDS, doc}
#define MB_METHOD8(name, f, doc) {name, method<Fp8Calls, f>(), METH_FASTCALL | METH_KEYWORDS, doc}

PyMethodDef methods[] = {
    MB_METHOD("mb_unpad_index", unpad_index,
              "mb_unpad_index($self, mask)\n--\n\n"
              "mask [B, L] int32 on the GPU -> (seqlens [B], cu_seqlens [B+1], indices [B*L] (first T valid), meta [2])."),
    MB_METHOD("mb_unpad", unpad,
              "mb_unpad($self, padded, indices, T_cap, meta, out=None)\n--\n\n"
              "padded [B*L, W] (any leading shape flattened by the caller) -> packed [T_cap, W]; rows < T written."),
    MB_METHOD("mb_pad", pad,
              "mb_pad($self, packed, indices, T_cap, meta, B, L, out=None)\n--\n\n"
              "packed [>=T, W] -> padded [B*L, W], zero at padded positions."),
    MB_METHOD("mb_zero_padding", zero_padding,
              "mb_zero_padding($self, padded, indices, T_cap, meta, B, L)\n--\n\n"
              "Zero the rows of padded [B*L, W] that `indices` does not list."),
    MB_METHOD("mb_alibi_attn_fwd", attn_fwd,
              "mb_alibi_attn_fwd($self, q, k, v, cu_seqlens, max_seqlen, slopes, softmax_scale, out=None, lse=None, "
              "token_rows=None, T=None, workspace=None, key_lens=None, plan=None)\n--\n\n"
              "q, k, v: [T, H, D] views (token stride free).  Returns (o [T, H, D], lse [H, T] float32).\n"
              "With token_rows the views are over a padded batch ([B*L, H, D]) and T (the lse pitch) must be given."),
    MB_METHOD("mb_alibi_attn_bwd", attn_bwd,
              "mb_alibi_attn_bwd($self, dout, q, k, v, o, lse, cu_seqlens, max_seqlen, slopes, softmax_scale, dq=None, "
              "dk=None, dv=None, workspace=None, token_rows=None, T=None, key_lens=None, plan=None)\n--\n\n"
              "Returns (dq, dk, dv), each [T, H, D] (padded-batch views when token_rows is given)."),
    MB_METHOD("mb_add_layernorm_fwd", layernorm_fwd,
              "mb_add_layernorm_fwd($self, x, r, gamma, beta, eps, T_cap=None, meta=None, y=None, s=None, mean=None, "
              "rstd=None, y_rows=None)\n--\n\n"
              "x, r: [rows, W] (r may be None).  Returns (y, s, mean, rstd); s is x itself when r is None.\n"
              "With y_rows, y must be given: a padded batch whose row y_rows[t] receives the result of token t."),
    MB_METHOD("mb_add_layernorm_bwd", layernorm_bwd,
              "mb_add_layernorm_bwd($self, dy, s, gamma, mean, rstd, T_cap=None, meta=None, ds=None, dgamma=None, "
              "dbeta=None, workspace=None, dy_rows=None)\n--\n\n"
              "Returns (ds [rows, W], dgamma [W] float32, dbeta [W] float32).\n"
              "With dy_rows, dy is a padded batch and token t's row is dy[dy_rows[t]]."),
    MB_METHOD("mb_geglu_fwd", geglu_fwd,
              "mb_geglu_fwd($self, x, w1v, w2, T_cap=None, meta=None, act=None, y=None)\n--\n\n"
              "x [rows, hidden]; w1v [2*inter, hidden] (W1 transposed over V transposed); w2 [hidden, inter] (W2\n"
              "transposed).  Returns (y [rows, hidden], act [rows, inter])."),
    MB_METHOD("mb_geglu_bwd", geglu_bwd,
              "mb_geglu_bwd($self, dy, x, w1v, w2, act, hg=None, T_cap=None, meta=None, dx=None, dw1v=None, dw2=None, "
              "workspace=None)\n--\n\n"
              "Returns (dx [rows, hidden], dw1v [2*inter, hidden] float32, dw2 [hidden, inter] float32).  hg: the stored\n"
              "[rows, 2*inter] projections of the unfused forward, or None to have them computed again."),
    MB_METHOD("mb_linear_fwd", linear_fwd,
              "mb_linear_fwd($self, x, wt, T_cap=None, meta=None, y=None)\n--\n\n"
              "y = x @ wt.T for x [rows, n_in], wt [n_out, n_in]."),
    {nullptr, nullptr, 0, nullptr}};

PyMethodDef methods8[] = {
    MB_METHOD8("mb_fp8_quant", quant,
               "mb_fp8_quant($self, x, T_cap=None, meta=None, q=None, s=None)\n--\n\n"
               "x [rows, W] bfloat16 or float32, dense rows -> (q [rows, W] float8_e4m3fn, s [rows, ceil(W/128)] float8_e8m0fnu)."),
    MB_METHOD8("mb_fp8_dequant", dequant,
               "mb_fp8_dequant($self, q, s, dtype=None, T_cap=None, meta=None, out=None)\n--\n\n"
               "8-bit rows -> [rows, W] bfloat16 (or dtype float32)."),
    MB_METHOD8("mb_fp8_quant_weight", quant_weight,
               "mb_fp8_quant_weight($self, w, transposed=True, q=None, s=None, qt=None, st=None)\n--\n\n"
               "w [n_out, n_in] -> (q, s, qt, st): 8-bit values with a scale for each 128 x 128 block, and the same transposed;\n"
               "(q, s) alone with transposed=False."),
    MB_METHOD8("mb_linear_fp8_fwd", linear,
               "mb_linear_fp8_fwd($self, xq, xs, wq, ws, dtype=None, T_cap=None, meta=None, y=None)\n--\n\n"
               "y = x @ w.T for 8-bit rows x [rows, n_in] and an 8-bit weight w [n_out, n_in].  bfloat16: sums of the 8-bit matrix\n"
               "instructions, off by at most 7 * 2**-13 of sum |x w|; dtype float32: fp32 sums, at half the rate.\n"
               "With dy's rows and the transposed weight it is the data gradient."),
    MB_METHOD8("mb_linear_fp8_wgrad", wgrad,
               "mb_linear_fp8_wgrad($self, dy, xq, xs, dys=None, T_cap=None, meta=None, dw=None, workspace=None)\n--\n\n"
               "dw = dy.T @ x, float32, for stored 8-bit rows x [rows, n_in]; dy [rows, n_out] bfloat16, or 8-bit rows with dys."),
    MB_METHOD8("mb_geglu_fp8_act", geglu_act,
               "mb_geglu_fp8_act($self, xq, xs, w1vq, w1vs, T_cap=None, meta=None, actq=None, acts=None)\n--\n\n"
               "GeLU(x W1) * x V for 8-bit rows x and the 8-bit weight [2*inter, hidden] (W1 transposed over V transposed), as\n"
               "8-bit rows: (actq [rows, inter], acts)."),
    MB_METHOD8("mb_gelu_gate_fp8_bwd", gate_bwd,
               "mb_gelu_gate_fp8_bwd($self, da, hg, hgs=None, T_cap=None, meta=None, dhgq=None, dhgs=None)\n--\n\n"
               "Backward of GeLU(h) * g from da [rows, inter] bfloat16 and h | g [rows, 2*inter] (bfloat16, or 8-bit rows with\n"
               "hgs), as 8-bit rows dh | dg: (dhgq [rows, 2*inter], dhgs)."),
    {nullptr, nullptr, 0, nullptr}};

void find_all(Calls* c, const std::function<void(void**, const char*)>& address) {
  auto find = [&](auto& to, const char* name) { address(reinterpret_cast<void**>(&to), name); };
  find(c->unpad_index, "mb_unpad_index");
  find(c->unpad, "mb_unpad");
  find(c->pad, "mb_pad");
  find(c->zero_padding, "mb_zero_padding");
  find(c->attn_fwd, "mb_alibi_attn_fwd");
  find(c->attn_fwd_bytes, "mb_alibi_attn_fwd_workspace_bytes");
  find(c->attn_bwd, "mb_alibi_attn_bwd");
  find(c->attn_bwd_bytes, "mb_alibi_attn_bwd_workspace_bytes");
  find(c->layernorm_fwd, "mb_add_layernorm_fwd");
  find(c->layernorm_bwd, "mb_add_layernorm_bwd");
  find(c->layernorm_bwd_bytes, "mb_add_layernorm_bwd_workspace_bytes");
  find(c->geglu_fwd, "mb_geglu_fwd");
  find(c->geglu_bwd, "mb_geglu_bwd");
  find(c->geglu_bwd_bytes, "mb_geglu_bwd_workspace_bytes");
  find(c->linear_fwd, "mb_linear_fwd");
}
void find_all(Fp8Calls* c, const std::function<void(void**, const char*)>& address) {
  auto find = [&](auto& to, const char* name) { address(reinterpret_cast<void**>(&to), name); };
  find(c->quant, "mb_fp8_quant");
  find(c->dequant, "mb_fp8_dequant");
  find(c->quant_weight, "mb_fp8_quant_weight");
  find(c->linear, "mb_linear_fp8_fwd");
  find(c->wgrad, "mb_linear_fp8_wgrad");
  find(c->wgrad_bytes, "mb_linear_fp8_wgrad_workspace_bytes");
  find(c->act, "mb_geglu_fp8_act");
  find(c->gate_bwd, "mb_gelu_gate_fp8_bwd");
}

// Calls(addresses, error, device, raw_stream, stream): `addresses` maps names of the C ABI to function addresses.
template <typename C>
PyObject* calls_new(PyTypeObject* type, PyObject* args, PyObject*) {
  PyObject *addresses, *error, *device, *raw_stream, *stream;
  if (!PyArg_ParseTuple(args, "O!OOOO", &PyDict_Type, &addresses, &error, &device, &raw_stream, &stream)) return nullptr;
  C* c = reinterpret_cast<C*>(type->tp_alloc(type, 0));
  if (!c) return nullptr;
  auto keep = [](PyObject*& to, PyObject* x) {
    Py_INCREF(x);
    to = x;
  };
  keep(c->error, error);
  keep(c->device, device);
  keep(c->raw_stream, raw_stream);
  keep(c->stream, stream);
  bool ok = true;
  auto address = [&](void** to, const char* name) {
    PyObject* x = ok ? PyDict_GetItemString(addresses, name) : nullptr;
    void* p = x ? PyLong_AsVoidPtr(x) : nullptr;
    if (ok && !p) {
      if (!PyErr_Occurred()) PyErr_Format(PyExc_KeyError, "no address of %s", name);
      ok = false;
    }
    *to = p;
  };
  address(reinterpret_cast<void**>(&c->last_error), "mb_last_error");
  find_all(c, address);
  if (!ok) {
    Py_DECREF(c);
    return nullptr;
  }
  return reinterpret_cast<PyObject*>(c);
}

void calls_dealloc(PyObject* self) {
  Host* c = reinterpret_cast<Host*>(self);
  Py_XDECREF(c->error);
  Py_XDECREF(c->device);
  Py_XDECREF(c->raw_stream);
  Py_XDECREF(c->stream);
  PyTypeObject* type = Py_TYPE(self);
  type->tp_free(self);
  Py_DECREF(type);
}

PyType_Slot slots[] = {{Py_tp_new, (void*)calls_new<Calls>},
                       {Py_tp_dealloc, (void*)calls_dealloc},
                       {Py_tp_methods, methods},
                       {0, nullptr}};
PyType_Spec spec = {"_mosaic_marshal.Calls", sizeof(Calls), 0, Py_TPFLAGS_DEFAULT, slots};
PyType_Slot slots8[] = {{Py_tp_new, (void*)calls_new<Fp8Calls>},
                        {Py_tp_dealloc, (void*)calls_dealloc},
                        {Py_tp_methods, methods8},
                        {0, nullptr}};
PyType_Spec spec8 = {"_mosaic_marshal.Fp8Calls", sizeof(Fp8Calls), 0, Py_TPFLAGS_DEFAULT, slots8};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_mosaic_marshal", nullptr, 0, nullptr, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__mosaic_marshal() {
  PyObject* m = PyModule_Create(&module_def);
  if (!m) return nullptr;
  for (auto [name, made] : {std::pair<const char*, PyType_Spec*>{"Calls", &spec}, {"Fp8Calls", &spec8}}) {
    PyObject* type = PyType_FromSpec(made);
    if (!type || PyModule_AddObject(m, name, type) < 0) {
      Py_XDECREF(type);
      Py_DECREF(m);
      return nullptr;
    }
  }
  if (PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
