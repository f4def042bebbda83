// What the Python binding of the paged calls does for every argument, without the interpreter: compares a tensor with the layout
// that its struct was made for, and hands integers and addresses to a C entry point.  A call of the paged cache has a dozen tensors; looked
// over attribute by attribute in Python they take 0.6 to 1 us each, and as much again for the conversions of ctypes, longer than most of the
// kernels behind them; here it is 0.1 us.  Nothing is remembered from one call to the next.
// A function that does not find what it expects answers None, and the binding says in its own words what is wrong.
#include <Python.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>
#include <utility>

namespace {

bool same_shape(const at::Tensor& t, PyObject* shape) {   // a tuple of ints, or a torch.Size, which is one
  if (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != t.dim()) return false;
  for (int64_t i = 0; i < t.dim(); ++i)
    if (PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i)) != t.size(i)) return PyErr_Clear(), false;
  return true;
}
bool is_on(const at::Tensor& t, PyObject* dtype, PyObject* device) {
  return THPDtype_Check(dtype) && reinterpret_cast<THPDtype*>(dtype)->scalar_type == t.scalar_type() && t.is_cuda() &&
         PyLong_Check(device) && PyLong_AsLongLong(device) == t.get_device();
}
// A tensor without memory of its own (a wrapper that other code sees as a CUDA tensor) has no address, or throws: no answer.
PyObject* address(const at::Tensor& t) {
  const void* const p = t.data_ptr();
  if (!p && t.numel() > 0) Py_RETURN_NONE;
  return PyLong_FromUnsignedLongLong(reinterpret_cast<uintptr_t>(p));
}
template <class F>
PyObject* or_none(F&& f) {
  try {
    return f();
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// dense(tensor, shape, dtype, device): the address of a contiguous tensor of that shape, type and CUDA device, or None.
PyObject* dense(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 4 || !THPVariable_Check(args[0])) Py_RETURN_NONE;
  return or_none([&]() -> PyObject* {
    const at::Tensor& t = THPVariable_Unpack(args[0]);
    if (!is_on(t, args[2], args[3]) || !t.is_contiguous() || !same_shape(t, args[1])) Py_RETURN_NONE;
    return address(t);
  });
}

// same(tensor, (shape, stride, dtype, device)): the address of a tensor of that layout, or None (also where only strides of extents of
// one differ).
PyObject* same(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 2 || !THPVariable_Check(args[0]) || !PyTuple_Check(args[1]) || PyTuple_GET_SIZE(args[1]) != 4) Py_RETURN_NONE;
  return or_none([&]() -> PyObject* {
    const at::Tensor& t = THPVariable_Unpack(args[0]);
    PyObject *const shape = PyTuple_GET_ITEM(args[1], 0), *const stride = PyTuple_GET_ITEM(args[1], 1);
    if (!is_on(t, PyTuple_GET_ITEM(args[1], 2), PyTuple_GET_ITEM(args[1], 3)) || !same_shape(t, shape)) Py_RETURN_NONE;
    if (!PyTuple_Check(stride) || PyTuple_GET_SIZE(stride) != t.dim()) Py_RETURN_NONE;
    for (int64_t i = 0; i < t.dim(); ++i)
      if (PyLong_AsLongLong(PyTuple_GET_ITEM(stride, i)) != t.stride(i)) {
        PyErr_Clear();
        Py_RETURN_NONE;
      }
    return address(t);
  });
}

// call(address of a function, arguments ...): its int result.  Arguments are integers and addresses (None: null), each of which takes a
// register or eight bytes of the stack whatever its width; none is a floating-point number.  The interpreter runs on meanwhile.
constexpr int kMost = 20;
template <size_t>
using Word = uint64_t;
template <size_t... I>
int call_with(const uint64_t* a, std::index_sequence<I...>) {
  return reinterpret_cast<int (*)(Word<I>...)>(a[0])(a[I + 1]...);
}
template <size_t N>
int caller(const uint64_t* a) { return call_with(a, std::make_index_sequence<N>()); }
typedef int (*Caller)(const uint64_t*);
template <size_t... N>
constexpr std::array<Caller, sizeof...(N)> callers_of(std::index_sequence<N...>) { return {caller<N>...}; }
constexpr auto callers = callers_of(std::make_index_sequence<kMost + 1>());   // by the number of arguments
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n < 1 || n > kMost + 1) return PyErr_Format(PyExc_TypeError, "call takes a function and up to %d arguments", kMost);
  uint64_t a[kMost + 1] = {};
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (args[i] == Py_None) continue;
    a[i] = PyLong_AsUnsignedLongLongMask(args[i]);
    if (a[i] == (uint64_t)-1 && PyErr_Occurred()) return nullptr;
  }
  int result;
  Py_BEGIN_ALLOW_THREADS
  result = callers[n - 1](a);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(result);
}

PyMethodDef methods[] = {{"dense", (PyCFunction)(void (*)(void))dense, METH_FASTCALL, nullptr},
                         {"same", (PyCFunction)(void (*)(void))same, METH_FASTCALL, nullptr},
                         {"call", (PyCFunction)(void (*)(void))call, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
