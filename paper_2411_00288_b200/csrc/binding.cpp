// CPython binding of the library's launching entry points: torch tensors in, status out.
//
// A layer of a few images runs 4 us on the GPU; the Python around its call (a check per tensor, addresses, the stream, a
// foreign call that converts ten arguments by their declared types) took as long again.  Here every argument is converted
// by the type that the C prototype gives it, in one native call:
//   const ssconv_desc_t*   the ctypes structure (any object with a buffer of that size); likewise ssconv_resnorm_t
//   other pointers         None, or a contiguous CUDA tensor
//   size_t                 the bytes of a tensor (0 for None): scratch is passed twice, as address and size
//   the last void*         the stream: None for the current one, or an object with `cuda_stream`
// The GIL is released around the call.  The entry points and their results are those of include/ssconv.h.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <memory>
#include <tuple>
#include <type_traits>
#include <utility>
#include <vector>

#include "ssconv.h"

namespace {

struct PythonError {};  // a Python exception is set

[[noreturn]] void raise(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw PythonError{};
}

int64_t as_int(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PythonError{};
  return v;
}

const at::Tensor& as_tensor(PyObject* o) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "a tensor (or None) is expected");
  return THPVariable_Unpack(o);
}

void* as_address(PyObject* o) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = as_tensor(o);
  if (!t.is_cuda() || !t.is_contiguous()) raise(PyExc_ValueError, "tensors must be contiguous CUDA tensors");
  return t.mutable_data_ptr();  // (as data_ptr() in Python: a lazily copied tensor becomes one of its own)
}

void* as_stream(PyObject* o) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
  PyObject* handle = PyObject_GetAttrString(o, "cuda_stream");
  if (handle == nullptr) throw PythonError{};
  void* s = PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  if (s == nullptr && PyErr_Occurred()) throw PythonError{};
  return s;
}

// One argument of type T from a Python object; `held` keeps a descriptor's buffer.
struct Held {
  Py_buffer buffer{};
  ~Held() { PyBuffer_Release(&buffer); }  // (nothing to do if it was never taken)
};
template <class T>
T convert(PyObject* o, Held& held, bool last) {
  if constexpr (std::is_same_v<T, const ssconv_desc_t*> || std::is_same_v<T, const ssconv_resnorm_t*>) {
    if (PyObject_GetBuffer(o, &held.buffer, PyBUF_SIMPLE) != 0) throw PythonError{};
    if (held.buffer.len != (Py_ssize_t)sizeof(std::remove_pointer_t<T>)) raise(PyExc_TypeError, "a descriptor of this call's kind is expected");
    return static_cast<T>(held.buffer.buf);
  } else if constexpr (std::is_pointer_v<T>) {
    return static_cast<T>(last ? as_stream(o) : as_address(o));
  } else if constexpr (std::is_same_v<T, float>) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError{};
    return (float)v;
  } else if constexpr (std::is_same_v<T, size_t>) {
    return o == Py_None ? 0 : (size_t)as_tensor(o).nbytes();
  } else {
    return (T)as_int(o);
  }
}

template <auto FN>
struct Entry;
template <class... A, int32_t (*FN)(A...)>
struct Entry<FN> {
  template <size_t... I>
  static int32_t run(PyObject* const* args, std::index_sequence<I...>) {
    Held held;
    // (braces: converted from left to right)
    std::tuple<A...> v{convert<A>(args[I], held, I + 1 == sizeof...(A))...};
    int32_t rc;
    Py_BEGIN_ALLOW_THREADS
    rc = FN(std::get<I>(v)...);
    Py_END_ALLOW_THREADS
    return rc;
  }
  static PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != (Py_ssize_t)sizeof...(A)) {
      PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, (Py_ssize_t)sizeof...(A));
      return nullptr;
    }
    int32_t rc;
    try {
      rc = run(args, std::index_sequence_for<A...>{});
    } catch (const PythonError&) {
      return nullptr;
    }
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
  }
};

// output(desc, x): an uninitialised bf16 tensor for the layer's output on x's device, or the library's status.
PyObject* output(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    if (n != 2) raise(PyExc_TypeError, "output(desc, x)");
    Held held;
    const ssconv_desc_t* d = convert<const ssconv_desc_t*>(args[0], held, false);
    const at::Tensor& x = as_tensor(args[1]);
    int32_t ho = 0, wo = 0;
    const int32_t rc = ssconv_out_shape(d, &ho, &wo);
    if (rc != SSCONV_OK) return PyLong_FromLong(rc);
    return THPVariable_Wrap(at::empty({d->N, ho, wo, d->C_out}, at::TensorOptions().dtype(at::kBFloat16).device(x.device())));
  } catch (const PythonError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// blob(n, x): n uninitialised bytes on x's device.
PyObject* blob(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    if (n != 2) raise(PyExc_TypeError, "blob(n, x)");
    return THPVariable_Wrap(
        at::empty({as_int(args[0])}, at::TensorOptions().dtype(at::kByte).device(as_tensor(args[1]).device())));
  } catch (const PythonError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// ---- Calls that also check and allocate their tensors here: as much Python as the call itself takes would double its time.
// (Outputs that are not given are allocated for the current stream.)

bool here(const at::Tensor& t) { return t.is_cuda() && t.is_contiguous() && t.get_device() == c10::cuda::current_device(); }
bool on(int device, const at::Tensor& t) { return t.is_cuda() && t.is_contiguous() && t.get_device() == device; }

// The address of a tensor of `numel` elements of `type` on the current device, or nullptr for None.
void* expect(PyObject* o, const char* name, at::ScalarType type, int64_t numel) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = as_tensor(o);
  if (t.scalar_type() != type) {
    PyErr_Format(PyExc_TypeError, "%s: %s is expected, not %s", name, c10::toString(type), c10::toString(t.scalar_type()));
    throw PythonError{};
  }
  if (t.numel() != numel) {
    PyErr_Format(PyExc_ValueError, "%s: %lld elements are expected, not %lld", name, (long long)numel, (long long)t.numel());
    throw PythonError{};
  }
  if (!here(t)) {
    PyErr_Format(PyExc_ValueError, "%s: tensors must be contiguous and on the current CUDA device", name);
    throw PythonError{};
  }
  return t.mutable_data_ptr();
}

// A new tensor beside `like` if o is None, o itself otherwise (checked by expect()).
at::Tensor given_or_new(PyObject* o, at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) {
  if (o != Py_None) return as_tensor(o);
  return at::detail::empty_cuda(shape, type, like.device(), std::nullopt);
}
// A part of a contiguous tensor's allocation, from one of its elements on.
at::Tensor part_of(const at::Tensor& all, int64_t from, at::IntArrayRef shape) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), all.dtype());
  t.unsafeGetTensorImpl()->set_storage_offset(from);
  t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
  return t;
}
// New fp32 tensors shaped like those of `like` that are not None, one after the other in one allocation (extents: multiples of 8).
template <size_t N>
void allocate_like(PyObject* const* like, at::Tensor (&out)[N], const at::Tensor& beside) {
  int64_t total = 0;
  bool any = false;
  for (size_t i = 0; i < N; ++i) {
    if (like[i] == Py_None) continue;
    any = true;
    total += as_tensor(like[i]).numel();
  }
  if (!any) return;
  const at::Tensor all = at::detail::empty_cuda({total}, at::kFloat, beside.device(), std::nullopt);
  int64_t from = 0;
  for (size_t i = 0; i < N; ++i) {
    if (like[i] == Py_None) continue;
    const at::Tensor& shape = as_tensor(like[i]);
    out[i] = part_of(all, from, shape.sizes());
    from += shape.numel();
  }
}
void* address(const at::Tensor& t) { return t.numel() != 0 ? t.mutable_data_ptr() : nullptr; }

// (status, results...): what a call gives back to its Python function.
template <class... T>
PyObject* results(int32_t rc, const T&... tensors) {
  PyObject* out = PyTuple_New(1 + sizeof...(T));
  if (out == nullptr) throw PythonError{};
  PyTuple_SET_ITEM(out, 0, PyLong_FromLong(rc));
  Py_ssize_t i = 1;
  const auto put = [&](const at::Tensor& t) {
    if (t.defined()) {
      PyTuple_SET_ITEM(out, i++, THPVariable_Wrap(t));
    } else {
      Py_INCREF(Py_None);
      PyTuple_SET_ITEM(out, i++, Py_None);
    }
  };
  (put(tensors), ...);
  return out;
}

template <class F>
int32_t without_gil(F f) {
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return rc;
}

void* current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

double as_double(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PythonError{};
  return v;
}

// The body of such a call: its arguments are counted, its exceptions become Python's.
template <PyObject* (*BODY)(PyObject* const*)>
PyObject* checked(PyObject* const* args, Py_ssize_t n, Py_ssize_t expected) {
  HANDLE_TH_ERRORS
  if (n != expected) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, expected);
    return nullptr;
  }
  try {
    return BODY(args);
  } catch (const PythonError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// Lists (or what else gives tensors one after the other) of contiguous fp32 tensors, or bf16 ones where the call takes them, on the
// current device, as many and of the same extents in each list.  The tensors are held until the call is made: a generator's are
// nobody else's, and another thread may change a list.  (One piece of memory, of the list itself where it has few tensors.)
struct TensorList {
  static constexpr size_t kFew = 32;
  PyObject** items;  // held
  void** p;
  int64_t* n;
  int32_t* type;
  int32_t count = 0;
  at::Tensor first;  // (undefined: an empty list)
  TensorList(PyObject* o, bool takes_bf16, const TensorList* like) {
    const Owned sequence{PySequence_Fast(o, "a list of tensors is expected")};
    if (sequence.o == nullptr) throw PythonError{};
    const Py_ssize_t all = PySequence_Fast_GET_SIZE(sequence.o);
    if (all > INT32_MAX) raise(PyExc_ValueError, "too many tensors");
    if (like != nullptr && all != like->count) raise(PyExc_ValueError, "the lists have different lengths");
    const size_t room = (size_t)all <= kFew ? kFew : (size_t)all;
    if (room > kFew) many.reset(new uint64_t[room * kBytes / 8 + 1]);
    items = reinterpret_cast<PyObject**>(room > kFew ? many.get() : few);
    p = reinterpret_cast<void**>(items + room);
    n = reinterpret_cast<int64_t*>(p + room);
    type = reinterpret_cast<int32_t*>(n + room);
    held.list = this;  // (from here on what is held is released, also if a tensor is refused)
    int device = -1;
    for (Py_ssize_t i = 0; i < all; ++i) {
      PyObject* const item = PySequence_Fast_GET_ITEM(sequence.o, i);
      const at::Tensor& t = as_tensor(item);
      if (i == 0 && t.is_cuda()) device = c10::cuda::current_device();
      if (!on(device, t)) raise(PyExc_ValueError, "tensors must be contiguous and on the current CUDA device");
      const bool bf16 = t.scalar_type() == at::kBFloat16;
      if (!bf16 && t.scalar_type() != at::kFloat) raise(PyExc_TypeError, "float32 or bfloat16 tensors are expected");
      if (bf16 && !takes_bf16) raise(PyExc_TypeError, "float32 tensors are expected");
      if (like != nullptr && t.numel() != like->n[i]) raise(PyExc_ValueError, "tensors of one position have different extents");
      if (i == 0) first = t;
      Py_INCREF(item);
      items[i] = item;
      p[i] = address(t);
      n[i] = t.numel();
      type[i] = bf16 ? SSCONV_BF16 : SSCONV_F32;
      ++count;
    }
  }
  TensorList(const TensorList&) = delete;
  TensorList& operator=(const TensorList&) = delete;
  bool same_types(const TensorList& other) const { return std::equal(type, type + count, other.type, other.type + other.count); }

 private:
  struct Owned {
    PyObject* o;
    ~Owned() { Py_XDECREF(o); }
  };
  struct Release {
    TensorList* list = nullptr;
    ~Release() {
      for (int32_t i = 0; list != nullptr && i < list->count; ++i) Py_DECREF(list->items[i]);
    }
  };
  static constexpr size_t kBytes = sizeof(PyObject*) + sizeof(void*) + sizeof(int64_t) + sizeof(int32_t);  // of a tensor
  uint64_t few[kFew * kBytes / 8];
  std::unique_ptr<uint64_t[]> many;
  Release held;  // (the last member: it goes first)
};

// grad_norm(grads, kind, norm, ws) -> (status, norm)
PyObject* grad_norm(PyObject* const* a) {
  const TensorList g(a[0], true, nullptr);
  const int64_t kind = as_int(a[1]);
  if (kind != (int32_t)kind) raise(PyExc_ValueError, "kind: GRAD_NORM_L2 or GRAD_NORM_INF is expected");
  expect(a[2], "norm", at::kFloat, 1);
  if (!g.first.defined() && (a[2] == Py_None || a[3] == Py_None))
    raise(PyExc_ValueError, "without gradients the norm's tensor and the scratch have to be given");
  at::Tensor norm = given_or_new(a[2], {1}, at::kFloat, g.first), ws;
  if (a[3] != Py_None) {
    ws = as_tensor(a[3]);
    expect(a[3], "ws", ws.scalar_type(), ws.numel());
  } else {
    size_t bytes = 0;
    const int32_t rc = ssconv_grad_norm_ws_bytes(g.count, &bytes);
    if (rc != SSCONV_OK) return results(rc, at::Tensor());
    ws = given_or_new(Py_None, {(int64_t)bytes}, at::kByte, g.first);
  }
  void* stream = current_stream();
  return results(without_gil([&] {
                   return ssconv_grad_norm(g.p, g.n, g.type, g.count, (int32_t)kind, static_cast<float*>(address(norm)), address(ws),
                                           ws.nbytes(), stream);
                 }),
                 norm);
}

// clip_grads(grads, out, norm, max_norm) -> (status,)
PyObject* clip_grads(PyObject* const* a) {
  const TensorList g(a[0], true, nullptr), out(a[1], true, &g);
  if (!g.same_types(out)) raise(PyExc_TypeError, "a gradient and its output have different types");
  const float* norm = static_cast<const float*>(expect(a[2], "norm", at::kFloat, 1));
  const float max_norm = (float)as_double(a[3]);
  void* stream = current_stream();
  return results(without_gil(
      [&] { return ssconv_clip_grads(g.p, out.p, g.n, g.type, g.count, norm, max_norm, stream); }));
}

// adamw_multi(theta, grads, m, v, step, lr, beta1, beta2, eps, weight_decay, norm, max_norm) -> (status,)
PyObject* adamw_multi(PyObject* const* a) {
  const TensorList g(a[1], true, nullptr), theta(a[0], false, &g), m(a[2], false, &g), v(a[3], false, &g);
  const int64_t step = as_int(a[4]);
  if (step < 1 || step > INT32_MAX) raise(PyExc_ValueError, "steps count from 1");
  const double lr = as_double(a[5]), beta1 = as_double(a[6]), beta2 = as_double(a[7]), eps = as_double(a[8]), decay = as_double(a[9]);
  const float* norm = static_cast<const float*>(expect(a[10], "norm", at::kFloat, 1));
  const float max_norm = (float)as_double(a[11]);
  void* stream = current_stream();
  return results(without_gil([&] {
    return ssconv_adamw_multi(theta.p, g.p, m.p, v.p, g.n, g.type, g.count, (int32_t)step, lr, beta1,
                              beta2, eps, decay, norm, max_norm, stream);
  }));
}

int64_t elements(const ssconv_resnorm_t& d) { return d.rows * d.C; }
// (of a descriptor that the library refuses any number will do: nothing is allocated by it)
int64_t gates(const ssconv_resnorm_t& d) {
  return d.rows_per_gate > 0 ? (d.rows / d.rows_per_gate + (d.rows % d.rows_per_gate != 0)) * d.C : d.C;
}

struct ResNormInputs {
  Held held;
  const ssconv_resnorm_t* d;
  void *x, *b;
  float *gate, *post_gamma, *post_beta, *pre_gamma, *pre_beta;
  // desc, x, b, gate, post_gamma, post_beta, pre_gamma, pre_beta
  explicit ResNormInputs(PyObject* const* a) {
    d = convert<const ssconv_resnorm_t*>(a[0], held, false);
    x = expect(a[1], "x", at::kBFloat16, elements(*d));
    b = expect(a[2], "b", at::kBFloat16, elements(*d));
    if (a[1] == Py_None) raise(PyExc_TypeError, "x: a tensor is expected");
    gate = static_cast<float*>(expect(a[3], "gate", at::kFloat, gates(*d)));
    post_gamma = static_cast<float*>(expect(a[4], "post_gamma", at::kFloat, d->C));
    post_beta = static_cast<float*>(expect(a[5], "post_beta", at::kFloat, d->C));
    pre_gamma = static_cast<float*>(expect(a[6], "pre_gamma", at::kFloat, d->C));
    pre_beta = static_cast<float*>(expect(a[7], "pre_beta", at::kFloat, d->C));
  }
};

// residual_norm(desc, x, b, gate, post_gamma, post_beta, pre_gamma, pre_beta, want_stats, h, y, stats) -> (status, h, y, stats)
PyObject* residual_norm(PyObject* const* a) {
  const ResNormInputs in(a);
  const ssconv_resnorm_t& d = *in.d;
  const at::Tensor& x = as_tensor(a[1]);
  expect(a[9], "h", at::kBFloat16, elements(d));
  expect(a[10], "y", at::kBFloat16, elements(d));
  expect(a[11], "stats", at::kFloat, 4 * d.rows);
  const int want_stats = PyObject_IsTrue(a[8]);
  if (want_stats < 0) throw PythonError{};
  at::Tensor h = given_or_new(a[9], x.sizes(), at::kBFloat16, x), y, stats;
  if (a[10] != Py_None || d.pre != SSCONV_NORM_NONE) y = given_or_new(a[10], x.sizes(), at::kBFloat16, x);
  if (a[11] != Py_None || want_stats) stats = given_or_new(a[11], {d.rows, 4}, at::kFloat, x);
  void* stream = current_stream();
  const int32_t rc = without_gil([&] {
    return ssconv_residual_norm(&d, in.x, in.b, in.gate, in.post_gamma, in.post_beta, in.pre_gamma, in.pre_beta, address(h),
                                y.defined() ? address(y) : nullptr, stats.defined() ? static_cast<float*>(address(stats)) : nullptr, stream);
  });
  return results(rc, h, y, stats);
}

// residual_norm_backward(desc, x, b, gate, post_gamma, post_beta, pre_gamma, pre_beta, stats, dh, dy, ws)
//   -> (status, dx, db, dgate, dpost_gamma, dpost_beta, dpre_gamma, dpre_beta)
PyObject* residual_norm_backward(PyObject* const* a) {
  const ResNormInputs in(a);
  const ssconv_resnorm_t& d = *in.d;
  const at::Tensor& x = as_tensor(a[1]);
  const float* stats = static_cast<const float*>(expect(a[8], "stats", at::kFloat, 4 * d.rows));
  const void* dh = expect(a[9], "dh", at::kBFloat16, elements(d));
  const void* dy = expect(a[10], "dy", at::kBFloat16, elements(d));
  at::Tensor dx = given_or_new(Py_None, x.sizes(), at::kBFloat16, x), db = given_or_new(Py_None, x.sizes(), at::kBFloat16, x), sums[5], ws;
  float* out[5];
  allocate_like(a + 3, sums, x);
  for (int i = 0; i < 5; ++i) {
    out[i] = sums[i].defined() ? static_cast<float*>(address(sums[i])) : nullptr;
  }
  if (a[11] != Py_None) {
    ws = as_tensor(a[11]);
    expect(a[11], "ws", ws.scalar_type(), ws.numel());
  } else {
    size_t bytes = 0;
    const int32_t rc = ssconv_residual_norm_ws_bytes(&d, &bytes);
    if (rc != SSCONV_OK) return results(rc, dx, db, sums[0], sums[1], sums[2], sums[3], sums[4]);
    ws = given_or_new(Py_None, {(int64_t)bytes}, at::kByte, x);
  }
  void* stream = current_stream();
  const int32_t rc = without_gil([&] {
    return ssconv_residual_norm_backward(&d, in.x, in.b, stats, dh, dy, in.gate, in.post_gamma, in.post_beta, in.pre_gamma, address(dx), address(db),
                                         out[0], out[1], out[2], out[3], out[4], address(ws), ws.nbytes(), stream);
  });
  return results(rc, dx, db, sums[0], sums[1], sums[2], sums[3], sums[4]);
}

std::vector<int64_t> with_last(const at::Tensor& t, int64_t last) {
  std::vector<int64_t> shape(t.sizes().begin(), t.sizes().end());
  shape.back() = last;
  return shape;
}

// quantize_mxfp4(x, codes, scales) -> (status, codes, scales)
PyObject* quantize_mxfp4(PyObject* const* a) {
  const at::Tensor& x = as_tensor(a[0]);
  if (x.dim() == 0) raise(PyExc_ValueError, "x: rows of channels are expected");
  const int64_t C = x.size(-1), rows = C > 0 ? x.numel() / C : 0;
  void* px = expect(a[0], "x", at::kBFloat16, rows * C);
  if (C > INT32_MAX) raise(PyExc_ValueError, "x: too many channels");
  size_t n_codes = 0, n_scales = 0;
  const int32_t sized = ssconv_sizes_mxfp4(rows, (int32_t)C, &n_codes, &n_scales);
  if (sized != SSCONV_OK) return results(sized, at::Tensor(), at::Tensor());
  expect(a[1], "codes", at::kByte, (int64_t)n_codes);
  expect(a[2], "scales", at::kByte, (int64_t)n_scales);
  const std::vector<int64_t> shape = with_last(x, (C + 31) / 32 * 16);
  at::Tensor codes, scales;
  if (a[1] == Py_None && a[2] == Py_None) {  // both in one allocation: one is of no use without the other
    const at::Tensor all = at::detail::empty_cuda({(int64_t)(n_codes + n_scales)}, at::kByte, x.device(), std::nullopt);
    codes = part_of(all, 0, shape);
    scales = part_of(all, (int64_t)n_codes, {(int64_t)n_scales});
  } else {
    codes = given_or_new(a[1], shape, at::kByte, x);
    scales = given_or_new(a[2], {(int64_t)n_scales}, at::kByte, x);
  }
  void* stream = current_stream();
  const int32_t rc = without_gil([&] { return ssconv_quantize_mxfp4(px, rows, (int32_t)C, address(codes), address(scales), stream); });
  return results(rc, codes, scales);
}

// dequantize_mxfp4(codes, scales, C, x) -> (status, x)
PyObject* dequantize_mxfp4(PyObject* const* a) {
  const at::Tensor& codes = as_tensor(a[0]);
  const int64_t C = as_int(a[2]);
  if (C <= 0 || C > INT32_MAX) raise(PyExc_ValueError, "C: a positive number of channels is expected");
  const int64_t row = (C + 31) / 32 * 16;
  if (codes.dim() == 0 || codes.size(-1) != row) {
    PyErr_Format(PyExc_ValueError, "codes: rows of %lld channels are %lld bytes", (long long)C, (long long)row);
    throw PythonError{};
  }
  const int64_t rows = codes.numel() / row;
  size_t n_codes = 0, n_scales = 0;
  const int32_t sized = ssconv_sizes_mxfp4(rows, (int32_t)C, &n_codes, &n_scales);
  if (sized != SSCONV_OK) return results(sized, at::Tensor());
  void* pc = expect(a[0], "codes", at::kByte, (int64_t)n_codes);
  void* ps = expect(a[1], "scales", at::kByte, (int64_t)n_scales);
  expect(a[3], "x", at::kBFloat16, rows * C);
  const at::Tensor x = given_or_new(a[3], with_last(codes, C), at::kBFloat16, codes);
  void* stream = current_stream();
  return results(without_gil([&] { return ssconv_dequantize_mxfp4(pc, ps, rows, (int32_t)C, address(x), stream); }), x);
}

// forward_dense_mxfp4(desc, x_codes, x_scales, w_codes, w_scales, bias, y, dev_status) -> (status, y)
PyObject* forward_dense_mxfp4(PyObject* const* a) {
  Held held;
  const ssconv_desc_t& d = *convert<const ssconv_desc_t*>(a[0], held, false);
  const int64_t pixels = (int64_t)d.N * d.H * d.W;
  size_t n[4];
  int32_t rc = ssconv_sizes_mxfp4(pixels, d.C_in, &n[0], &n[1]);
  if (rc == SSCONV_OK) rc = ssconv_sizes_mxfp4(d.C_out, d.C_in, &n[2], &n[3]);
  if (rc != SSCONV_OK) return results(rc, at::Tensor());
  static const char* const names[4] = {"x_codes", "x_scales", "w_codes", "w_scales"};
  void* p[4];
  for (int i = 0; i < 4; ++i) p[i] = expect(a[1 + i], names[i], at::kByte, (int64_t)n[i]);
  const float* bias = static_cast<const float*>(expect(a[5], "bias", at::kFloat, d.C_out));
  expect(a[6], "y", at::kBFloat16, pixels * d.C_out);
  int32_t* status = static_cast<int32_t*>(expect(a[7], "dev_status", at::kInt, 1));
  const at::Tensor y = given_or_new(a[6], {d.N, d.H, d.W, d.C_out}, at::kBFloat16, as_tensor(a[1]));
  void* stream = current_stream();
  rc = without_gil([&] { return ssconv_forward_dense_mxfp4(&d, p[0], p[1], p[2], p[3], bias, address(y), status, stream); });
  return results(rc, y);
}

template <PyObject* (*BODY)(PyObject* const*), Py_ssize_t COUNT>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return checked<BODY>(args, n, COUNT);
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))Entry<&name>::call, METH_FASTCALL, nullptr}
#define CALL(name, count) {#name, (PyCFunction)(void (*)(void))call<name, count>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    ENTRY(ssconv_select_mask), ENTRY(ssconv_compress), ENTRY(ssconv_maxpool), ENTRY(ssconv_space_to_depth),
    ENTRY(ssconv_forward), ENTRY(ssconv_forward_res), ENTRY(ssconv_forward_dense), ENTRY(ssconv_forward_dense_res),
    ENTRY(ssconv_forward_dense_strided), ENTRY(ssconv_soft_mask), ENTRY(ssconv_mask_grad), ENTRY(ssconv_adamw),
    ENTRY(ssconv_wgrad), ENTRY(ssconv_dgrad), ENTRY(ssconv_forward_grouped), ENTRY(ssconv_forward_dense_grouped),
    ENTRY(ssconv_depthwise), ENTRY(ssconv_layernorm), ENTRY(ssconv_quantize_e4m3), ENTRY(ssconv_forward_fp8),
    ENTRY(ssconv_forward_dense_fp8),
    CALL(grad_norm, 4), CALL(clip_grads, 4), CALL(adamw_multi, 12), CALL(residual_norm, 12), CALL(residual_norm_backward, 12),
    CALL(quantize_mxfp4, 3), CALL(dequantize_mxfp4, 4), CALL(forward_dense_mxfp4, 8),
    {"output", (PyCFunction)(void (*)(void))output, METH_FASTCALL, nullptr},
    {"blob", (PyCFunction)(void (*)(void))blob, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
