// Addresses of many tensors for a call that takes them as an array: what the binding would ask each of them for in Python (five calls, 0.2 us a tensor)
// in one loop (0.01 us).  Host code; it knows torch's tensors, which the library does not.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>

namespace {

// addresses(tensors, sizes, dtype, device) -> bytes of n addresses, or None where a tensor is not what the call takes.
//   tensors  a list or tuple of tensors or None; sizes: n numbers of 64 bits, the elements of each
//   dtype    a tensor of the type that all have; device: the index of the one that all are on
// A tensor that is None or whose size is 0 has the address 0.
PyObject* addresses(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  if (n_args != 4 || !PyBytes_Check(args[1]) || !THPVariable_Check(args[2])) {
    PyErr_SetString(PyExc_TypeError, "addresses(tensors, sizes as bytes, a tensor of the type, device index)");
    return nullptr;
  }
  const long device = PyLong_AsLong(args[3]);
  if (device == -1 && PyErr_Occurred()) return nullptr;
  PyObject* const list = PySequence_Fast(args[0], "tensors: a list or tuple");
  if (list == nullptr) return nullptr;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
  PyObject* const out = PyBytes_GET_SIZE(args[1]) == n * 8 ? PyBytes_FromStringAndSize(nullptr, n * 8) : nullptr;
  bool good = out != nullptr;
  if (good) {
    char* const to = PyBytes_AS_STRING(out);
    const char* const sizes = PyBytes_AS_STRING(args[1]);
    try {
      const at::ScalarType dtype = THPVariable_Unpack(args[2]).scalar_type();
      for (Py_ssize_t i = 0; good && i < n; ++i) {
        PyObject* const item = PySequence_Fast_GET_ITEM(list, i);
        int64_t size;
        std::memcpy(&size, sizes + i * 8, 8);
        uint64_t address = 0;
        if (item != Py_None && size != 0) {
          good = THPVariable_Check(item);
          if (!good) break;
          const at::Tensor& t = THPVariable_Unpack(item);
          good = t.numel() == size && t.scalar_type() == dtype && t.is_cuda() && t.get_device() == device && t.is_contiguous();
          if (good) address = reinterpret_cast<uint64_t>(t.data_ptr());
        }
        std::memcpy(to + i * 8, &address, 8);
      }
    } catch (const std::exception&) {   // a tensor without memory of its own
      good = false;
    }
  }
  Py_DECREF(list);
  if (good) return out;
  Py_XDECREF(out);
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"addresses", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(addresses)), METH_FASTCALL,
                          "Addresses of tensors of known sizes, one type and one device, as bytes; None where one is not that."},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
