// Argument marshalling of the paged-cache entry points for Python: checks tensors and calls
// libseer's C functions.  In Python each tensor argument cost 0.35 us of a call whose kernels
// take 2 to 5 (page tables: 9.8 us a call there, of which 3.3 in the library).
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <stdexcept>
#include <string>
#include <tuple>
#include <type_traits>

#include "../../include/seer.h"

namespace {

struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};
struct PythonError {};

// The address of a tensor on the current device, of a raw address, or null for None.
void* address(PyObject* o, int device, const c10::ScalarType* type) {
  if (o == Py_None) return nullptr;
  if (THPVariable_Check(o)) {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device)
      throw Refused("a tensor on " + t.device().str() + " is not on the current device cuda:" + std::to_string(device));
    if (type != nullptr && (t.scalar_type() != *type || !t.is_contiguous()))
      throw Refused(std::string("expected a contiguous ") + c10::toString(*type) + " tensor, got " + c10::toString(t.scalar_type()) +
                    (t.is_contiguous() ? "" : ", not contiguous"));
    return const_cast<void*>(t.const_data_ptr());
  }
  if (PyLong_Check(o)) {
    void* p = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) throw PythonError();
    return p;
  }
  throw Refused(std::string("expected a tensor, an address or None, got ") + Py_TYPE(o)->tp_name);
}

constexpr c10::ScalarType kInt32 = c10::ScalarType::Int, kInt64 = c10::ScalarType::Long;

template <typename T>
struct Arg {                                // integers
  static T get(PyObject* o, int) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError();
    if (static_cast<long long>(static_cast<T>(v)) != v || (v < 0 && std::is_unsigned_v<T>)) throw Refused("an integer argument is out of range");
    return static_cast<T>(v);
  }
};
template <>
struct Arg<seer_dtype> {
  static seer_dtype get(PyObject* o, int d) { return static_cast<seer_dtype>(Arg<int>::get(o, d)); }
};
template <>
struct Arg<float> {
  static float get(PyObject* o, int) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError();
    return static_cast<float>(v);
  }
};
template <>
struct Arg<const void*> {
  static const void* get(PyObject* o, int d) { return address(o, d, nullptr); }
};
template <>
struct Arg<void*> {
  static void* get(PyObject* o, int d) { return address(o, d, nullptr); }
};
template <>
struct Arg<const int32_t*> {
  static const int32_t* get(PyObject* o, int d) { return static_cast<const int32_t*>(address(o, d, &kInt32)); }
};
template <>
struct Arg<int32_t*> {
  static int32_t* get(PyObject* o, int d) { return static_cast<int32_t*>(address(o, d, &kInt32)); }
};
template <>
struct Arg<const uint64_t*> {
  static const uint64_t* get(PyObject* o, int d) { return static_cast<const uint64_t*>(address(o, d, &kInt64)); }
};
template <>
struct Arg<uint64_t*> {
  static uint64_t* get(PyObject* o, int d) { return static_cast<uint64_t*>(address(o, d, &kInt64)); }
};
template <>
struct Arg<const seer_pages*> {             // the ctypes struct
  static const seer_pages* get(PyObject* o, int) {
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw PythonError();
    const void* p = b.buf;
    const bool fits = b.len == static_cast<Py_ssize_t>(sizeof(seer_pages));
    PyBuffer_Release(&b);
    if (!fits) throw Refused("pages is not a seer_pages");
    return static_cast<const seer_pages*>(p);
  }
};

// stream: None for PyTorch's current one, a torch.cuda.Stream or a raw handle.
void* stream_of(PyObject* o, int device) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream(device).stream();
  if (PyLong_Check(o)) return address(o, device, nullptr);
  PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
  if (h == nullptr) throw PythonError();
  void* p = PyLong_AsVoidPtr(h);
  Py_DECREF(h);
  if (PyErr_Occurred()) throw PythonError();
  return p;
}

template <auto Fn>
struct Call;
// A C entry point whose last parameter is the stream; its arguments in order, the stream last.
template <typename... P, seer_status (*Fn)(P...)>
struct Call<Fn> {
  static constexpr size_t N = sizeof...(P);
  using Params = std::tuple<P...>;

  template <size_t... I>
  static seer_status run(PyObject* const* a, std::index_sequence<I...>) {
    const int device = c10::cuda::current_device();
    const std::tuple<std::tuple_element_t<I, Params>..., void*> v{Arg<std::tuple_element_t<I, Params>>::get(a[I], device)...,
                                                                 stream_of(a[N - 1], device)};
    return std::apply(Fn, v);
  }
  static PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
      if (n != static_cast<Py_ssize_t>(N)) throw Refused("takes " + std::to_string(N) + " arguments");
      return PyLong_FromLong(run(a, std::make_index_sequence<N - 1>()));
    } catch (const PythonError&) {
    } catch (const Refused& e) {
      PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception& e) {
      PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
  }
};

#define SEER_ENTRY(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&Call<&f>::entry)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {SEER_ENTRY(seer_page_tables), SEER_ENTRY(seer_kv_append), SEER_ENTRY(seer_kv_accept),
                          SEER_ENTRY(seer_attention_causal), SEER_ENTRY(seer_attention_tree), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_seer_binding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__seer_binding() { return PyModule_Create(&kModule); }
