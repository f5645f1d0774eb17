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
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

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

// The calls over many tensors: lists (or tuples) of contiguous fp32 tensors, or bf16 ones where the call takes them, on the
// current device, as many and of the same extents in each list.
struct TensorList {
  std::vector<void*> p;
  std::vector<int64_t> n;
  std::vector<int32_t> type;
  TensorList(PyObject* o, bool takes_bf16, const TensorList* like) {
    PyObject* items = PySequence_Fast(o, "a list of tensors is expected");
    if (items == nullptr) throw PythonError{};
    struct Release {
      PyObject* o;
      ~Release() { Py_DECREF(o); }
    } release{items};
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(items);
    if (like != nullptr && (size_t)count != like->n.size()) raise(PyExc_ValueError, "the lists have different lengths");
    p.reserve(count);
    n.reserve(count);
    type.reserve(count);
    for (Py_ssize_t i = 0; i < count; ++i) {
      const at::Tensor& t = as_tensor(PySequence_Fast_GET_ITEM(items, i));
      if (!t.is_cuda() || !t.is_contiguous() || t.get_device() != c10::cuda::current_device())
        raise(PyExc_ValueError, "tensors must be contiguous and on the current CUDA device");
      const bool bf16 = t.scalar_type() == at::kBFloat16;
      if (!bf16 && t.scalar_type() != at::kFloat) raise(PyExc_TypeError, "float32 or bfloat16 tensors are expected");
      if (bf16 && !takes_bf16) raise(PyExc_TypeError, "float32 tensors are expected");
      if (like != nullptr && t.numel() != like->n[i]) raise(PyExc_ValueError, "tensors of one position have different extents");
      p.push_back(t.numel() != 0 ? t.mutable_data_ptr() : nullptr);
      n.push_back(t.numel());
      type.push_back(bf16 ? SSCONV_BF16 : SSCONV_F32);
    }
    if (count > INT32_MAX) raise(PyExc_ValueError, "too many tensors");
  }
  int32_t size() const { return (int32_t)p.size(); }
};
const float* as_norm(PyObject* o) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = as_tensor(o);
  if (!t.is_cuda() || t.numel() != 1 || t.scalar_type() != at::kFloat || t.get_device() != c10::cuda::current_device())
    raise(PyExc_ValueError, "the norm is one float32 number on the current CUDA device");
  return static_cast<const float*>(t.mutable_data_ptr());
}
double as_double(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PythonError{};
  return v;
}

// grad_norm(grads, kind, norm, ws, stream)
PyObject* grad_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    if (n != 5) raise(PyExc_TypeError, "grad_norm(grads, kind, norm, ws, stream)");
    const TensorList g(args[0], true, nullptr);
    const int32_t kind = (int32_t)as_int(args[1]);
    float* norm = const_cast<float*>(as_norm(args[2]));
    void* ws = as_address(args[3]);
    const size_t ws_bytes = args[3] == Py_None ? 0 : as_tensor(args[3]).nbytes();
    void* stream = as_stream(args[4]);
    int32_t rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ssconv_grad_norm(g.p.data(), g.n.data(), g.type.data(), g.size(), kind, norm, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  } catch (const PythonError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// clip_grads(grads, out, norm, max_norm, stream)
PyObject* clip_grads(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    if (n != 5) raise(PyExc_TypeError, "clip_grads(grads, out, norm, max_norm, stream)");
    const TensorList g(args[0], true, nullptr), out(args[1], true, &g);
    if (g.type != out.type) raise(PyExc_TypeError, "a gradient and its output have different types");
    const float* norm = as_norm(args[2]);
    const float max_norm = (float)as_double(args[3]);
    void* stream = as_stream(args[4]);
    int32_t rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ssconv_clip_grads(g.p.data(), out.p.data(), g.n.data(), g.type.data(), g.size(), norm, max_norm, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  } catch (const PythonError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// adamw_multi(theta, grads, m, v, step, lr, beta1, beta2, eps, weight_decay, norm, max_norm, stream)
PyObject* adamw_multi(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  try {
    if (n != 13) raise(PyExc_TypeError, "adamw_multi(theta, grads, m, v, step, lr, beta1, beta2, eps, weight_decay, norm, max_norm, stream)");
    const TensorList g(args[1], true, nullptr), theta(args[0], false, &g), m(args[2], false, &g), v(args[3], false, &g);
    const int64_t step = as_int(args[4]);
    if (step < 1 || step > INT32_MAX) raise(PyExc_ValueError, "steps count from 1");
    const double lr = as_double(args[5]), beta1 = as_double(args[6]), beta2 = as_double(args[7]), eps = as_double(args[8]),
                 decay = as_double(args[9]);
    const float* norm = as_norm(args[10]);
    const float max_norm = (float)as_double(args[11]);
    void* stream = as_stream(args[12]);
    int32_t rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ssconv_adamw_multi(theta.p.data(), g.p.data(), m.p.data(), v.p.data(), g.n.data(), g.type.data(), g.size(), (int32_t)step, lr, beta1,
                            beta2, eps, decay, norm, max_norm, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  } catch (const PythonError&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))Entry<&name>::call, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    ENTRY(ssconv_select_mask), ENTRY(ssconv_compress), ENTRY(ssconv_maxpool), ENTRY(ssconv_space_to_depth),
    ENTRY(ssconv_forward), ENTRY(ssconv_forward_res), ENTRY(ssconv_forward_dense), ENTRY(ssconv_forward_dense_res),
    ENTRY(ssconv_forward_dense_strided), ENTRY(ssconv_soft_mask), ENTRY(ssconv_mask_grad), ENTRY(ssconv_adamw),
    ENTRY(ssconv_wgrad), ENTRY(ssconv_dgrad), ENTRY(ssconv_forward_grouped), ENTRY(ssconv_forward_dense_grouped),
    ENTRY(ssconv_depthwise), ENTRY(ssconv_layernorm), ENTRY(ssconv_quantize_e4m3), ENTRY(ssconv_forward_fp8),
    ENTRY(ssconv_forward_dense_fp8), ENTRY(ssconv_residual_norm), ENTRY(ssconv_residual_norm_backward),
    ENTRY(ssconv_quantize_mxfp4), ENTRY(ssconv_dequantize_mxfp4), ENTRY(ssconv_forward_dense_mxfp4),
    {"grad_norm", (PyCFunction)(void (*)(void))grad_norm, METH_FASTCALL, nullptr},
    {"clip_grads", (PyCFunction)(void (*)(void))clip_grads, METH_FASTCALL, nullptr},
    {"adamw_multi", (PyCFunction)(void (*)(void))adamw_multi, METH_FASTCALL, nullptr},
    {"output", (PyCFunction)(void (*)(void))output, METH_FASTCALL, nullptr},
    {"blob", (PyCFunction)(void (*)(void))blob, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
