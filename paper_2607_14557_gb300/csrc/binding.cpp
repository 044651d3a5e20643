// Argument marshalling of the paged-cache entry points for Python: checks tensors (device, type,
// contiguity of arrays, and that their memory holds what the call names) and calls libseer's C
// functions.  Addresses given as integers are taken as they are.  In Python each tensor argument cost 0.35 us of a call whose kernels
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

// ------------------------------------------------------------------ what a call's tensors have to hold
// All of these let pass what is not a tensor and sizes that the C entry refuses.
long long integer(PyObject* o) { return Arg<long long>::get(o, 0); }

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

// The element type of a seer_dtype; Undefined for others.
c10::ScalarType element(long long dt) {
  return dt == SEER_F32 ? c10::ScalarType::Float
                        : (dt == SEER_BF16 ? c10::ScalarType::BFloat16 : (dt == SEER_F16 ? c10::ScalarType::Half : c10::ScalarType::Undefined));
}

// n elements from the tensor's first on.
void holds(const char* name, PyObject* o, long long n) {
  const at::Tensor* t = tensor(o);
  if (t != nullptr && t->numel() < n)
    throw Refused(std::string(name) + " holds " + std::to_string(t->numel()) + " elements, the call names " + std::to_string(n));
}

// `rows` rows of `cols` values of type dt, ld apart; the tensor may be a column block of a wider buffer.
void rows_hold(const char* name, PyObject* o, long long dt, long long rows, long long ld, long long cols) {
  const at::Tensor* t = tensor(o);
  const c10::ScalarType type = element(dt);
  if (t == nullptr || type == c10::ScalarType::Undefined) return;
  if (t->scalar_type() != type)
    throw Refused(std::string(name) + " is a " + c10::toString(t->scalar_type()) + " tensor, the call's type is " + c10::toString(type));
  if (rows <= 0 || ld < cols || cols <= 0) return;
  const long long have = static_cast<long long>(t->storage().nbytes() / t->itemsize()) - t->storage_offset();
  if ((rows - 1) * ld + cols > have)
    throw Refused(std::string(name) + ": " + std::to_string(rows) + " rows of " + std::to_string(cols) + " values, " + std::to_string(ld) +
                  " apart, end behind the tensor's memory");
}

// A pool of type dt and a table of B rows: make_pages leaves (dtype code, device, rows of the table) as _held,
// -1 for what it was given as an address.
void pages_hold(PyObject* pages, long long dt, long long B, bool on_device) {
  static PyObject* const kHeld = PyUnicode_InternFromString("_held");
  PyObject* held = PyObject_GetAttr(pages, kHeld);
  if (held == nullptr) {
    PyErr_Clear();
    return;
  }
  int type = -1, device = -1, table_rows = -1;
  const bool known = held != Py_None && PyArg_ParseTuple(held, "iii", &type, &device, &table_rows) != 0;
  Py_DECREF(held);
  if (!known) {
    if (PyErr_Occurred()) throw PythonError();
    return;
  }
  if (on_device) {
    if (device != -1 && device != c10::cuda::current_device()) throw Refused("the page pool or its table is not on the current device");
    return;
  }
  if (type != -1 && type != dt && element(dt) != c10::ScalarType::Undefined)
    throw Refused(std::string("the page pool is of another type than the call's ") + c10::toString(element(dt)));
  if (table_rows != -1 && B > table_rows)
    throw Refused("the page table has " + std::to_string(table_rows) + " rows, the call names " + std::to_string(B) + " requests");
}

seer_pages pages_of(PyObject* o) { return *Arg<const seer_pages*>::get(o, 0); }

// Per entry point, before anything asks for a device; then the index of its `pages`, or -1.
template <auto Fn>
void check(PyObject* const*);
template <auto Fn>
constexpr int kPages = -1;

template <>
void check<&seer_page_tables>(PyObject* const* a) {
  const long long B = integer(a[2]), free = integer(a[6]), pages = integer(a[9]), cap = integer(a[10]);
  holds("cached_len", a[0], B);
  holds("new_len", a[1], B);
  holds("free_pages", a[5], free);
  holds("free_head", a[7], 1);
  if (B <= SEER_MAX_REQUESTS) holds("table", a[8], B * pages);
  holds("parent", a[11], cap);
  holds("cu_new_out", a[12], B + 1);
  holds("kv_len_out", a[13], B);
  holds("slot_out", a[14], cap);
  holds("position_out", a[15], cap);
  holds("mask_out", a[16], cap);
  holds("free_head_out", a[17], 1);
}

template <>
constexpr int kPages<&seer_kv_append> = 11;
template <>
void check<&seer_kv_append>(PyObject* const* a) {
  const long long ld = integer(a[1]), dt = integer(a[2]), heads = integer(a[3]), cap = integer(a[4]), ld_rot = integer(a[10]);
  const seer_pages g = pages_of(a[11]);
  rows_hold("qkv", a[0], dt, cap, ld, (heads + 2ll * g.n_kv_heads) * g.head_dim);
  holds("M_dev", a[5], 1);
  holds("slot", a[6], cap);
  holds("position", a[7], cap);
  rows_hold("rotated", a[9], dt, cap, ld_rot, (heads + g.n_kv_heads) * g.head_dim);
  pages_hold(a[11], dt, 0, false);
}

template <>
constexpr int kPages<&seer_kv_accept> = 6;
template <>
void check<&seer_kv_accept>(PyObject* const* a) {
  const long long B = integer(a[4]), draft = integer(a[5]);
  holds("cached_len", a[1], B);
  if (B <= SEER_MAX_REQUESTS) holds("accepted", a[2], B * draft);
  holds("n_accepted", a[3], B);
  holds("len_out", a[7], B);
  pages_hold(a[6], integer(a[0]), B, false);
}

template <>
void check<&seer_attention_causal>(PyObject* const* a) {
  const long long dt = integer(a[8]), B = integer(a[10]), cap = integer(a[11]), dh = integer(a[14]);
  const long long q = integer(a[12]) * dh, k = integer(a[13]) * dh;
  rows_hold("q", a[0], dt, cap, integer(a[1]), q);
  rows_hold("k", a[2], dt, cap, integer(a[3]), k);
  rows_hold("v", a[4], dt, cap, integer(a[5]), k);
  rows_hold("o", a[6], dt, cap, integer(a[7]), q);
  holds("cu_seqlens", a[9], B + 1);
}

template <>
constexpr int kPages<&seer_attention_tree> = 12;
template <>
void check<&seer_attention_tree>(PyObject* const* a) {
  const long long dt = integer(a[4]), B = integer(a[8]), cap = integer(a[9]), bytes = Arg<size_t>::get(a[14], 0);
  const seer_pages g = pages_of(a[12]);
  const long long cols = integer(a[10]) * g.head_dim;
  rows_hold("q", a[0], dt, cap, integer(a[1]), cols);
  rows_hold("o", a[2], dt, cap, integer(a[3]), cols);
  holds("cu_new", a[5], B + 1);
  holds("kv_len", a[6], B);
  const at::Tensor* ws = tensor(a[13]);
  if (ws != nullptr && (!ws->is_contiguous() || static_cast<long long>(ws->nbytes()) < bytes))
    throw Refused("ws holds " + std::to_string(ws->nbytes()) + " bytes" + (ws->is_contiguous() ? "" : ", not contiguous") + ", the call names " +
                  std::to_string(bytes));
  pages_hold(a[12], dt, B, false);
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
    check<Fn>(a);
    if constexpr (kPages<Fn> >= 0) pages_hold(a[kPages<Fn>], 0, 0, true);
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
