// The calls of experts.py: checks of the tensors, outputs and scratch memory from torch's allocator, the call into libmix.so.
//
// A decode step makes five of these calls and its kernels take a few microseconds each; through ctypes and torch.empty in
// Python a call took some 20 us (64 tokens on 8 experts, selection and order: 51.7 us a pass).  Here the tensors' fields are read
// and outputs allocated by torch's C++ interface.  The GIL is released round the call into the library: a launch can wait for
// room in a full queue.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <climits>
#include <cstdarg>
#include <initializer_list>
#include <optional>
#include <stdexcept>
#include <string>

#include "mix.h"

namespace {

using at::ScalarType;
using at::Tensor;

struct Refused : std::runtime_error {            // ValueError
  using std::runtime_error::runtime_error;
};
struct Raised {};                                // a Python error that is set already
struct Failed {                                  // MixError
  int code;
  std::string message;
};

__attribute__((format(printf, 2, 3))) void need(bool ok, const char* format, ...) {
  if (ok) return;
  char text[256];
  va_list ap;
  va_start(ap, format);
  vsnprintf(text, sizeof text, format, ap);
  va_end(ap);
  throw Refused(text);
}

int dtype_id(ScalarType t) {
  return t == ScalarType::Float ? MIX_DTYPE_F32 : t == ScalarType::BFloat16 ? MIX_DTYPE_BF16 : t == ScalarType::Half ? MIX_DTYPE_F16 : -1;
}

const Tensor& tensor(PyObject* o, const char* name, int64_t dim, const Tensor* like = nullptr) {
  need(THPVariable_Check(o), "%s must be a CUDA tensor", name);
  const Tensor& t = THPVariable_Unpack(o);
  need(t.is_cuda(), "%s must be a CUDA tensor", name);
  need(t.dim() == dim, "%s must have %d dimensions, not %d", name, (int)dim, (int)t.dim());
  for (const int64_t n : t.sizes()) need(n <= INT_MAX, "%s is too large", name);
  need(!like || t.get_device() == like->get_device(), "%s is on another device", name);
  return t;
}
const Tensor& tensor(PyObject* o, const char* name, ScalarType type, int64_t dim, const Tensor* like = nullptr) {
  const Tensor& t = tensor(o, name, dim, like);
  need(t.scalar_type() == type, "%s has type %s, not %s", name, c10::toString(t.scalar_type()), c10::toString(type));
  return t;
}
// A tensor without gaps, of one type and shape.
template <typename T>
T* dense(const Tensor& t, const char* name, std::initializer_list<int64_t> shape) {
  need(t.sizes() == at::IntArrayRef(shape), "%s has a shape that does not go with the others'", name);
  need(t.is_contiguous(), "%s must be contiguous", name);
  return static_cast<T*>(t.data_ptr());
}
template <typename T>
T* dense(PyObject* o, const char* name, ScalarType type, std::initializer_list<int64_t> shape, const Tensor& like) {
  return dense<T>(tensor(o, name, type, (int64_t)shape.size(), &like), name, shape);
}
// A matrix of floating-point numbers whose rows may lie apart.
struct Rows {
  const Tensor& t;
  void* p;
  int64_t ld, n, m;
  int dtype;
};
Rows rows_of(const Tensor& t, const char* name) {
  const int id = dtype_id(t.scalar_type());
  need(id >= 0, "%s has type %s", name, c10::toString(t.scalar_type()));
  const int64_t n = t.size(0), m = t.size(1);
  need(m <= 1 || t.stride(1) == 1, "%s: the elements of a row must lie next to each other", name);
  return Rows{t, t.data_ptr(), n > 1 ? t.stride(0) : (m > 1 ? m : 1), n, m, id};
}

long long integer(PyObject* o, const char* name, long long lo, long long hi) {
  PyObject* v = PyNumber_Index(o);
  if (!v) throw Raised();
  const long long x = PyLong_AsLongLong(v);
  Py_DECREF(v);
  if (x == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    need(false, "%s is out of range", name);
  }
  need(x >= lo && x <= hi, "%s %lld outside [%lld, %lld]", name, x, lo, hi);
  return x;
}

// One call: its device made current, its stream, and what it allocates, in order.
// A stream that is given is made current as well, so that outputs and scratch memory are the given stream's: what the allocator gave back
// on the stream that was current may still be used by work queued there.  The outputs are then marked as used by that one, on which
// the caller is likely to read and to drop them.
struct Call {
  c10::cuda::OptionalCUDAGuard guard;
  c10::cuda::OptionalCUDAStreamGuard as_current;
  int device;
  cudaStream_t stream;
  std::optional<c10::cuda::CUDAStream> before;   // the current stream, where another one is given
  Tensor made[8], scratch_memory;
  int n_made = 0;

  Call(int dev, PyObject* s) : device(dev) {
    if (c10::cuda::current_device() != dev) guard.set_index(dev);
    const c10::cuda::CUDAStream now = c10::cuda::getCurrentCUDAStream(dev);
    if (s == Py_None) {
      stream = now.stream();
      return;
    }
    PyObject* v = PyObject_GetAttrString(s, "cuda_stream");
    if (!v) {
      PyErr_Clear();
      v = PyNumber_Long(s);
    }
    if (!v) throw Raised();
    stream = static_cast<cudaStream_t>(PyLong_AsVoidPtr(v));
    Py_DECREF(v);
    if (!stream && PyErr_Occurred()) throw Raised();
    if (stream == now.stream()) return;
    before = now;
    as_current.reset_stream(stream ? c10::cuda::getStreamFromExternal(stream, (c10::DeviceIndex)dev)
                                   : c10::cuda::getDefaultCUDAStream((c10::DeviceIndex)dev));
  }
  Tensor allocated(at::IntArrayRef shape, ScalarType type) const {
    return Tensor(at::detail::empty_cuda(shape, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)device), std::nullopt));
  }
  Tensor& empty(at::IntArrayRef shape, ScalarType type) {
    Tensor& t = made[n_made++];
    t = allocated(shape, type);
    return t;
  }
  // The dense outputs of the call, in the order of the returned tuple: given (checked), or new.  New ones are pieces of one
  // allocation, each on 256 bytes: an allocation and its tensor cost 0.8 us, a tensor on a piece 0.3.
  struct Piece {
    int64_t at;
    ScalarType type;
    at::DimVector shape;
    void** p;
    PyObject** out;
  };
  Piece piece[4];
  int n_pieces = 0;
  int64_t bytes = 0;
  template <typename T>
  void want(PyObject* given, const char* name, ScalarType type, std::initializer_list<int64_t> shape, const Tensor& like, T** p, PyObject** out) {
    if (given != Py_None) {
      *p = dense<T>(given, name, type, shape, like);
      Py_INCREF(given);
      *out = given;
      return;
    }
    Piece& w = piece[n_pieces++];
    int64_t n = sizeof(T);
    for (const int64_t d : shape) n *= d;
    w = Piece{bytes, type, at::DimVector(shape), reinterpret_cast<void**>(p), out};
    bytes += (n + 255) / 256 * 256;
  }
  void allocate() {
    if (n_pieces == 0) return;
    const Tensor& all = empty({bytes}, ScalarType::Byte);
    for (int i = 0; i < n_pieces; ++i) {
      Piece& w = piece[i];
      const caffe2::TypeMeta meta = c10::scalarTypeToTypeMeta(w.type);
      Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), meta);
      t.unsafeGetTensorImpl()->set_sizes_contiguous(w.shape);
      t.unsafeGetTensorImpl()->set_storage_offset(w.at / (int64_t)meta.itemsize());
      *w.p = static_cast<char*>(all.data_ptr()) + w.at;
      *w.out = THPVariable_Wrap(std::move(t));
      if (!*w.out) throw Raised();
    }
  }
  Rows result_rows(PyObject* given, const char* name, ScalarType type, int64_t n, int64_t m, const Tensor& like, PyObject** out) {
    if (given != Py_None) {
      const Tensor& t = tensor(given, name, 2, &like);
      need(t.size(0) == n && t.size(1) == m, "%s has a shape that does not go with the others'", name);
      const Rows r = rows_of(t, name);
      Py_INCREF(given);
      *out = given;
      return r;
    }
    Tensor& t = empty({n, m}, type);
    *out = THPVariable_Wrap(t);
    if (!*out) throw Raised();
    return rows_of(t, name);
  }
  void* scratch(long long bytes) {
    if (bytes < 0) throw Failed{(int)bytes, "the sizes are out of range"};
    if (bytes == 0) return nullptr;
    scratch_memory = allocated({(int64_t)bytes}, ScalarType::Byte);
    return scratch_memory.data_ptr();
  }
  template <typename F>
  void run(F f) {
    char text[256] = "";
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(static_cast<void*>(stream), text, (int)sizeof text);
    Py_END_ALLOW_THREADS
    if (before)
      for (int i = 0; i < n_made; ++i)
        if (made[i].numel() > 0) c10::cuda::CUDACachingAllocator::recordStream(made[i].storage().data_ptr(), *before);
    if (rc != MIX_OK) throw Failed{rc, text};
  }
};

struct Results {                                 // references for the tuple that is returned
  PyObject* o[4] = {nullptr, nullptr, nullptr, nullptr};
  ~Results() {
    for (PyObject* x : o) Py_XDECREF(x);
  }
  PyObject* take(int i) {
    PyObject* x = o[i];
    o[i] = nullptr;
    return x;
  }
  PyObject* tuple(int n) {
    PyObject* t = PyTuple_New(n);
    if (!t) throw Raised();
    for (int i = 0; i < n; ++i) PyTuple_SET_ITEM(t, i, take(i));
    return t;
  }
};

// router_topk(logits, k, act, renormalise, n_live | None, idx | None, weights | None, stream | None)
PyObject* router_topk(PyObject* const* a) {
  const Rows x = rows_of(tensor(a[0], "logits", 2), "logits");
  const int64_t k = integer(a[1], "k", 1, x.m);
  const int act = (int)integer(a[2], "act", 0, 2);
  const int renorm = PyObject_IsTrue(a[3]);
  if (renorm < 0) throw Raised();
  const int* live = a[4] == Py_None ? nullptr : dense<int>(a[4], "n_live", ScalarType::Int, {1}, x.t);
  Call c(x.t.get_device(), a[7]);
  Results r;
  int* idx;
  float* w;
  c.want(a[5], "idx", ScalarType::Int, {x.n, k}, x.t, &idx, &r.o[0]);
  c.want(a[6], "weights", ScalarType::Float, {x.n, k}, x.t, &w, &r.o[1]);
  c.allocate();
  c.run([&](void* s, char* e, int n) { return mix_router_topk(x.p, x.dtype, x.ld, (int)x.n, (int)x.m, (int)k, act, renorm, live, idx, w, s, e, n); });
  return r.tuple(2);
}

// router_topk_grad(logits, idx, weights, d_weights, act, renormalise, d_logits | None, stream | None)
PyObject* router_topk_grad(PyObject* const* a) {
  const Rows x = rows_of(tensor(a[0], "logits", 2), "logits");
  const Tensor& it = tensor(a[1], "idx", ScalarType::Int, 2, &x.t);
  const int64_t k = it.size(1);
  const int* idx = dense<int>(it, "idx", {x.n, k});
  const float* w = dense<float>(a[2], "weights", ScalarType::Float, {x.n, k}, x.t);
  const float* dw = dense<float>(a[3], "d_weights", ScalarType::Float, {x.n, k}, x.t);
  const int act = (int)integer(a[4], "act", 0, 2);
  const int renorm = PyObject_IsTrue(a[5]);
  if (renorm < 0) throw Raised();
  Call c(x.t.get_device(), a[7]);
  Results r;
  const Rows d = c.result_rows(a[6], "d_logits", x.t.scalar_type(), x.n, x.m, x.t, &r.o[0]);
  need(d.dtype == x.dtype, "d_logits must have the logits' type");
  c.run([&](void* s, char* e, int n) {
    return mix_router_topk_grad(x.p, x.dtype, x.ld, (int)x.n, (int)x.m, (int)k, act, renorm, idx, w, dw, d.p, d.ld, s, e, n);
  });
  return r.take(0);
}

// expert_order(idx, n_experts, offsets | None, order | None, position | None, stream | None)
PyObject* expert_order(PyObject* const* a) {
  const Tensor& it = tensor(a[0], "idx", ScalarType::Int, 2);
  const int64_t n = it.numel(), E = integer(a[1], "n_experts", 1, INT_MAX - 1);
  const int* idx = dense<int>(it, "idx", {it.size(0), it.size(1)});
  const long long bytes = mix_expert_order_workspace(n, (int)E);
  if (bytes < 0) throw Failed{(int)bytes, "n_experts or the number of entries is out of range"};
  Call c(it.get_device(), a[5]);
  Results r;
  int *offsets, *order, *position;
  c.want(a[2], "offsets", ScalarType::Int, {E + 1}, it, &offsets, &r.o[0]);
  c.want(a[3], "order", ScalarType::Int, {n}, it, &order, &r.o[1]);
  c.want(a[4], "position", ScalarType::Int, {it.size(0), it.size(1)}, it, &position, &r.o[2]);
  c.allocate();
  void* ws = c.scratch(bytes);
  c.run([&](void* s, char* e, int m) { return mix_expert_order(idx, n, (int)E, offsets, order, position, ws, bytes, s, e, m); });
  return r.tuple(3);
}

const int* segments(PyObject* o, const Tensor& like, int* n_seg) {
  *n_seg = 1;
  if (o == Py_None) return nullptr;
  const Tensor& t = tensor(o, "seg", ScalarType::Int, 1, &like);
  need(t.numel() >= 2, "seg must hold the offsets of at least one segment");
  *n_seg = (int)t.numel() - 1;
  return dense<int>(t, "seg", {t.numel()});
}

// router_balance(logits, idx, seg | None, act, stream | None)
PyObject* router_balance(PyObject* const* a) {
  const Rows x = rows_of(tensor(a[0], "logits", 2), "logits");
  const Tensor& it = tensor(a[1], "idx", ScalarType::Int, 2, &x.t);
  const int64_t k = it.size(1);
  const int* idx = dense<int>(it, "idx", {x.n, k});
  int n_seg;
  const int* seg = segments(a[2], x.t, &n_seg);
  const int act = (int)integer(a[3], "act", 0, 2);
  Call c(x.t.get_device(), a[4]);
  Results r;
  float *loss, *mean;
  int *counts, *rows;
  c.want(Py_None, "loss", ScalarType::Float, {n_seg}, x.t, &loss, &r.o[0]);
  c.want(Py_None, "counts", ScalarType::Int, {n_seg, x.m}, x.t, &counts, &r.o[1]);
  c.want(Py_None, "mean_p", ScalarType::Float, {n_seg, x.m}, x.t, &mean, &r.o[2]);
  c.want(Py_None, "rows", ScalarType::Int, {n_seg}, x.t, &rows, &r.o[3]);
  c.allocate();
  const long long bytes = mix_router_balance_workspace((int)x.n, (int)x.m, n_seg);
  void* ws = c.scratch(bytes);
  c.run([&](void* s, char* e, int n) {
    return mix_router_balance(x.p, x.dtype, x.ld, idx, (int)x.n, (int)x.m, (int)k, act, seg, n_seg, loss, counts, mean, rows, ws, bytes, s, e, n);
  });
  return r.tuple(4);
}

// router_balance_grad(logits, idx, counts, rows, d_loss, seg | None, act, d_logits | None, stream | None)
PyObject* router_balance_grad(PyObject* const* a) {
  const Rows x = rows_of(tensor(a[0], "logits", 2), "logits");
  const Tensor& it = tensor(a[1], "idx", ScalarType::Int, 2, &x.t);
  const int64_t k = it.size(1);
  const int* idx = dense<int>(it, "idx", {x.n, k});
  int n_seg;
  const int* seg = segments(a[5], x.t, &n_seg);
  const int* counts = dense<int>(a[2], "counts", ScalarType::Int, {n_seg, x.m}, x.t);
  const int* rows = dense<int>(a[3], "rows", ScalarType::Int, {n_seg}, x.t);
  const float* d_loss = dense<float>(a[4], "d_loss", ScalarType::Float, {n_seg}, x.t);
  const int act = (int)integer(a[6], "act", 0, 2);
  Call c(x.t.get_device(), a[8]);
  Results r;
  const Rows d = c.result_rows(a[7], "d_logits", x.t.scalar_type(), x.n, x.m, x.t, &r.o[0]);
  need(d.dtype == x.dtype, "d_logits must have the logits' type");
  c.run([&](void* s, char* e, int n) {
    return mix_router_balance_grad(x.p, x.dtype, x.ld, idx, (int)x.n, (int)x.m, (int)k, act, seg, n_seg, counts, rows, d_loss, d.p, d.ld, s, e, n);
  });
  return r.take(0);
}

// quantize_rows(x, order | None, k, codes | None, scale | None, stream | None)
PyObject* quantize_rows(PyObject* const* a) {
  const Rows x = rows_of(tensor(a[0], "x", 2), "x");
  int64_t n = x.n;
  const int* order = nullptr;
  if (a[1] != Py_None) {
    const Tensor& t = tensor(a[1], "order", ScalarType::Int, 1, &x.t);
    n = t.numel();
    order = dense<int>(t, "order", {n});
  }
  const int k = (int)integer(a[2], "k", 1, INT_MAX);
  Call c(x.t.get_device(), a[5]);
  Results r;
  int8_t* codes;
  float* scale;
  c.want(a[3], "codes", ScalarType::Char, {n, x.m}, x.t, &codes, &r.o[0]);
  c.want(a[4], "scale", ScalarType::Float, {n}, x.t, &scale, &r.o[1]);
  c.allocate();
  if (order && n == 0) return r.tuple(2);
  c.run([&](void* s, char* e, int len) {
    return mix_quantize_rows(x.p, x.dtype, x.ld, (int)x.n, order, k, (int)n, (int)x.m, reinterpret_cast<signed char*>(codes), scale, s, e, len);
  });
  return r.tuple(2);
}

ScalarType dtype_arg(PyObject* o) {
  need(THPDtype_Check(o), "dtype must be a torch dtype");
  const ScalarType t = reinterpret_cast<THPDtype*>(o)->scalar_type;
  need(dtype_id(t) >= 0, "dtype %s is none of float32, bfloat16 and float16", c10::toString(t));
  return t;
}

// linear_int(codes, scale, W, w_scale, offsets | None, bias | None, out | None, dtype, stream | None); offsets: by experts
PyObject* linear_int(PyObject* const* a) {
  const Tensor& ct = tensor(a[0], "codes", ScalarType::Char, 2);
  const bool grouped = a[4] != Py_None;
  const Tensor& wt = tensor(a[2], "W", ScalarType::Char, grouped ? 3 : 2, &ct);
  const int64_t T = ct.size(0), K = ct.size(1), E = grouped ? wt.size(0) : 1, N = wt.size(grouped ? 1 : 0);
  const signed char* codes = dense<signed char>(ct, "codes", {T, K});
  const float* scale = dense<float>(a[1], "scale", ScalarType::Float, {T}, ct);
  const signed char* W = grouped ? dense<signed char>(wt, "W", {E, N, K}) : dense<signed char>(wt, "W", {N, K});
  const auto channels = [&](PyObject* o, const char* name) -> const float* {
    return grouped ? dense<float>(o, name, ScalarType::Float, {E, N}, ct) : dense<float>(o, name, ScalarType::Float, {N}, ct);
  };
  const float* w_scale = channels(a[3], "w_scale");
  const int* offsets = grouped ? dense<int>(a[4], "offsets", ScalarType::Int, {E + 1}, ct) : nullptr;
  const float* bias = a[5] == Py_None ? nullptr : channels(a[5], "bias");
  const ScalarType type = dtype_arg(a[7]);
  Call c(ct.get_device(), a[8]);
  Results r;
  const Rows out = c.result_rows(a[6], "out", type, T, N, ct, &r.o[0]);
  c.run([&](void* s, char* e, int n) {
    return grouped ? mix_linear_int_grouped(codes, scale, (int)T, (int)K, W, w_scale, (int)E, (int)N, offsets, bias, out.p, out.dtype, out.ld, s, e, n)
                   : mix_linear_int(codes, scale, (int)T, (int)K, W, w_scale, (int)N, bias, out.p, out.dtype, out.ld, s, e, n);
  });
  return r.take(0);
}

// expert_combine(y, weights, position, out | None, stream | None)
PyObject* expert_combine(PyObject* const* a) {
  const Rows y = rows_of(tensor(a[0], "y", 2), "y");
  const Tensor& pt = tensor(a[2], "position", ScalarType::Int, 2, &y.t);
  const int64_t T = pt.size(0), k = pt.size(1);
  const int* position = dense<int>(pt, "position", {T, k});
  const float* w = dense<float>(a[1], "weights", ScalarType::Float, {T, k}, y.t);
  Call c(y.t.get_device(), a[4]);
  Results r;
  const Rows out = c.result_rows(a[3], "out", y.t.scalar_type(), T, y.m, y.t, &r.o[0]);
  need(out.dtype == y.dtype, "out must have y's type");
  c.run([&](void* s, char* e, int n) {
    return mix_expert_combine(y.p, y.dtype, y.ld, (int)y.n, w, position, (int)T, (int)k, (int)y.m, out.p, out.ld, s, e, n);
  });
  return r.take(0);
}

// expert_combine_grad(d_out, y, weights, position, want_y, d_weights | None, d_y | None, stream | None)
PyObject* expert_combine_grad(PyObject* const* a) {
  const int want_y = PyObject_IsTrue(a[4]);
  if (want_y < 0) throw Raised();
  need(want_y || a[6] == Py_None, "d_y is given, but want_y is not set");
  const Rows y = rows_of(tensor(a[1], "y", 2), "y");
  const Tensor& pt = tensor(a[3], "position", ScalarType::Int, 2, &y.t);
  const int64_t T = pt.size(0), k = pt.size(1);
  const int* position = dense<int>(pt, "position", {T, k});
  const float* w = dense<float>(a[2], "weights", ScalarType::Float, {T, k}, y.t);
  const Rows d = rows_of(tensor(a[0], "d_out", 2, &y.t), "d_out");
  need(d.n == T && d.m == y.m && d.dtype == y.dtype, "d_out must be [T, N] in y's type");
  Call c(y.t.get_device(), a[7]);
  Results r;
  float* dw;
  c.want(a[5], "d_weights", ScalarType::Float, {T, k}, y.t, &dw, &r.o[0]);
  c.allocate();
  if (!want_y) {
    c.run([&](void* s, char* e, int n) {
      return mix_expert_combine_grad(y.p, y.dtype, y.ld, (int)y.n, w, position, (int)T, (int)k, (int)y.m, d.p, d.ld, dw, nullptr, y.m, s, e, n);
    });
    return r.take(0);
  }
  const Rows dy = c.result_rows(a[6], "d_y", y.t.scalar_type(), y.n, y.m, y.t, &r.o[1]);
  need(dy.dtype == y.dtype, "d_y must have y's type");
  c.run([&](void* s, char* e, int n) {
    return mix_expert_combine_grad(y.p, y.dtype, y.ld, (int)y.n, w, position, (int)T, (int)k, (int)y.m, d.p, d.ld, dw, dy.p, dy.ld, s, e, n);
  });
  return r.tuple(2);
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N) return PyErr_Format(PyExc_TypeError, "takes %d arguments", N);
  try {
    return F(a);
  } catch (const Raised&) {
    return nullptr;
  } catch (const Refused& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
    return nullptr;
  } catch (const Failed& e) {
    PyObject* module = PyImport_ImportModule("paper_2607_22595_b200.binding");
    PyObject* type = module ? PyObject_GetAttrString(module, "MixError") : nullptr;
    PyObject* args = type ? Py_BuildValue("(is)", e.code, e.message.c_str()) : nullptr;
    if (args) PyErr_SetObject(type, args);
    Py_XDECREF(args);
    Py_XDECREF(type);
    Py_XDECREF(module);
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

#define ENTRY(f, n) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(entry<f, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(router_topk, 8), ENTRY(router_topk_grad, 8), ENTRY(expert_order, 6), ENTRY(router_balance, 5),
                         ENTRY(router_balance_grad, 9), ENTRY(quantize_rows, 6), ENTRY(linear_int, 9), ENTRY(expert_combine, 5), ENTRY(expert_combine_grad, 8),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The layout of torch's C++ objects is compiled in: experts.py compares this with the torch that is running.
PyMODINIT_FUNC PyInit__fastops(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) != 0) Py_CLEAR(m);
  return m;
}
