// The host's share of a call that has many tensors, for the Python binding: results allocated in one go, and the facts of
// a list of tensors read in one go.  In the interpreter the first costs 1.6 us a tensor and the second 0.25 us, which is
// most of a call whose kernels take a few microseconds.  No computation and no CUDA call of its own.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <iterator>

#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

constexpr at::ScalarType kTypes[] = {at::kFloat, at::kBFloat16, at::kHalf, at::kInt, at::kByte};

// Results of a call that are small together are parts of one allocation, each from a multiple of 256 bytes on: an
// allocation takes 0.9 us, a tensor on another's memory 0.3.  (They belong together, and live as long as any of them.)
constexpr int64_t kShared = 4 << 20, kApart = 256;

// empties(like, (type, size, ...), ...) -> a tuple of new tensors on like's device.
PyObject* empties(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  constexpr Py_ssize_t kMost = 16;
  if (n < 1 || n > kMost || !THPVariable_Check(args[0])) {
    PyErr_SetString(PyExc_TypeError, "empties takes a tensor and the results' types and sizes");
    return nullptr;
  }
  const auto device = THPVariable_Unpack(args[0]).device();
  int64_t spec[kMost][4], total = 0;
  int dims[kMost];
  for (Py_ssize_t i = 1; i < n; ++i) {
    const bool ok = PyTuple_Check(args[i]) && PyTuple_GET_SIZE(args[i]) >= 1 && PyTuple_GET_SIZE(args[i]) <= 4;
    dims[i] = ok ? static_cast<int>(PyTuple_GET_SIZE(args[i])) - 1 : -1;
    double size = 1;
    for (int d = 0; d <= dims[i]; ++d) {
      spec[i][d] = PyLong_AsLongLong(PyTuple_GET_ITEM(args[i], d));
      if (PyErr_Occurred()) return nullptr;
      if (spec[i][d] < 0) dims[i] = -1;
      else if (d > 0) size *= static_cast<double>(spec[i][d]);
    }
    if (dims[i] < 0 || spec[i][0] >= static_cast<int64_t>(std::size(kTypes))) {
      PyErr_SetString(PyExc_ValueError, "a result is (type, size, ...), of at most three sizes");
      return nullptr;
    }
    if (size > kShared) total = kShared + 1;
    else if (total <= kShared) total += (static_cast<int64_t>(size) * c10::elementSize(kTypes[spec[i][0]]) + kApart - 1) / kApart * kApart;
  }
  const bool shared = total <= kShared;
  at::Tensor block;
  if (shared) block = at::empty(at::IntArrayRef(&total, 1), at::TensorOptions(at::kByte).device(device));
  PyObject* out = PyTuple_New(n - 1);
  if (!out) return nullptr;
  try {
    int64_t at = 0;
    for (Py_ssize_t i = 1; i < n; ++i) {
      const at::IntArrayRef sizes(spec[i] + 1, dims[i]);
      const at::ScalarType type = kTypes[spec[i][0]];
      at::Tensor t;
      if (shared) {
        t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(block.storage()), block.key_set(), caffe2::TypeMeta::fromScalarType(type));
        t.unsafeGetTensorImpl()->set_storage_offset(at / c10::elementSize(type));
        t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
        at += (t.numel() * static_cast<int64_t>(c10::elementSize(type)) + kApart - 1) / kApart * kApart;
      } else {
        t = at::empty(sizes, at::TensorOptions(type).device(device));
      }
      PyObject* o = THPVariable_Wrap(t);
      if (!o) {
        Py_DECREF(out);
        return nullptr;
      }
      PyTuple_SET_ITEM(out, i - 1, o);
    }
  } catch (...) {
    Py_DECREF(out);
    throw;
  }
  return out;
  END_HANDLE_TH_ERRORS
}

// facts(list) -> (addresses, types, elements, device): the first three as the bytes of uint64, int32 and int64 arrays.
// The device is -1 where a tensor is not on a GPU, -2 where they are on several, -3 where one is not contiguous or of
// another type, -4 where one is no tensor.
PyObject* facts(PyObject*, PyObject* list) {
  HANDLE_TH_ERRORS
  PyObject* seq = PySequence_Fast(list, "a sequence of tensors");
  if (!seq) return nullptr;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
  PyObject* a = PyBytes_FromStringAndSize(nullptr, n * 8);
  PyObject* t = PyBytes_FromStringAndSize(nullptr, n * 4);
  PyObject* e = PyBytes_FromStringAndSize(nullptr, n * 8);
  if (!a || !t || !e) {
    Py_XDECREF(a);
    Py_XDECREF(t);
    Py_XDECREF(e);
    Py_DECREF(seq);
    return nullptr;
  }
  auto* address = reinterpret_cast<uint64_t*>(PyBytes_AS_STRING(a));
  auto* type = reinterpret_cast<int32_t*>(PyBytes_AS_STRING(t));
  auto* elements = reinterpret_cast<int64_t*>(PyBytes_AS_STRING(e));
  int64_t device = -5;
  try {
    for (Py_ssize_t i = 0; i < n; ++i) {
      PyObject* o = PySequence_Fast_GET_ITEM(seq, i);
      if (!THPVariable_Check(o)) {
        device = -4;
        break;
      }
      const at::Tensor& x = THPVariable_Unpack(o);
      int32_t code = 0;
      while (code < 3 && kTypes[code] != x.scalar_type()) ++code;
      const int64_t d = x.is_cuda() ? x.get_device() : -1;
      if (d < 0) device = -1;
      else if (code == 3 || x.layout() != at::kStrided || !x.is_contiguous()) device = -3;
      else if (device != -5 && device != d) device = -2;
      else device = d;
      if (device < 0) break;
      address[i] = reinterpret_cast<uint64_t>(x.data_ptr());
      type[i] = code;
      elements[i] = x.numel();
    }
  } catch (...) {
    Py_DECREF(a);
    Py_DECREF(t);
    Py_DECREF(e);
    Py_DECREF(seq);
    throw;
  }
  Py_DECREF(seq);
  return Py_BuildValue("(NNNL)", a, t, e, static_cast<long long>(device));
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"empties", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(empties)), METH_FASTCALL, nullptr},
    {"facts", facts, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&module); }
