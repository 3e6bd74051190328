// The host's share of small calls, for the Python binding: results allocated in one go, the facts of a list of tensors
// read in one go, and the operators' usual calls from their tensors to the C ABI.  In the interpreter an
// allocation costs 1.6 us, a tensor's field 0.1 us and a call of 18 arguments 1.4 us, together most of a call
// whose kernels take a few microseconds.
//
// The calls below take what is usual: tensors on the current GPU that pass every check, on its current stream, results
// that are new.  For anything else they do nothing and return None; the binding then goes through its own checks, and
// raises what is to be raised.  No computation.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <algorithm>
#include <iterator>
#include <limits>
#include <vector>

#include <ATen/ops/empty.h>
#include <c10/core/Allocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

// The first three as HA_TYPE_*.
constexpr at::ScalarType kTypes[] = {at::kFloat, at::kBFloat16, at::kHalf, at::kInt, at::kByte};
constexpr int kF32 = 0, kI32 = 3, kU8 = 4;

// The C ABI's functions, and for tests, of the thread that asks for it: CPU tensors stand for a GPU's, and their calls are noted
// in `noted` instead of made.  Calls on a GPU's tensors are made all the same.
void *g_route, *g_route_backward, *g_dispatch, *g_combine, *g_combine_backward, *g_verify, *g_norm;
thread_local bool g_pretend = false;
thread_local PyObject* g_noted = nullptr;

// ---------------------------------------------------------------- results
// Results of a call that are small together are parts of one allocation, each from a multiple of 256 bytes on: an
// allocation takes 0.9 us, a tensor on another's memory 0.3.  (They belong together, and live as long as any of them.)
constexpr int64_t kShared = 4 << 20, kApart = 256;

struct Spec {
  int type;
  std::initializer_list<int64_t> sizes;
};
int64_t bytes_of(int type, at::IntArrayRef sizes) {
  double n = static_cast<double>(c10::elementSize(kTypes[type]));
  for (const int64_t s : sizes) n *= static_cast<double>(s);
  return n > kShared ? kShared + 1 : (static_cast<int64_t>(n) + kApart - 1) / kApart * kApart;
}
at::Tensor part_of(const at::Tensor& block, int64_t& at, int type, at::IntArrayRef sizes) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(block.storage()), block.key_set(),
                                                          caffe2::TypeMeta::fromScalarType(kTypes[type]));
  t.unsafeGetTensorImpl()->set_storage_offset(at / static_cast<int64_t>(c10::elementSize(kTypes[type])));
  t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
  at += bytes_of(type, sizes);
  return t;
}
template <typename Specs, typename Get>
std::vector<at::Tensor> make(const Specs& specs, Get get, at::Device device) {
  int64_t total = 0;
  for (const auto& s : specs) {
    const auto [type, sizes] = get(s);
    if (total <= kShared) total += bytes_of(type, sizes);
  }
  std::vector<at::Tensor> out;
  out.reserve(specs.size());
  at::Tensor block;
  if (total <= kShared) block = at::empty(at::IntArrayRef(&total, 1), at::TensorOptions(at::kByte).device(device));
  int64_t at = 0;
  for (const auto& s : specs) {
    const auto [type, sizes] = get(s);
    out.push_back(total <= kShared ? part_of(block, at, type, sizes)
                                   : at::empty(sizes, at::TensorOptions(kTypes[type]).device(device)));
  }
  return out;
}
std::vector<at::Tensor> results(at::Device device, std::initializer_list<Spec> specs) {
  return make(specs, [](const Spec& s) { return std::pair<int, at::IntArrayRef>(s.type, s.sizes); }, device);
}

// A call's workspace.  It is not the results', which would hold it as long as a caller keeps any of them (128 sequences of 5 drafts:
// 0.5 MB behind 7 KB), unless it is small: memory of its own takes 2 us (clipping 300 tensors by 6.7 KB of sums 20.0 us a call, 16.5 so).
constexpr int64_t kSmallWork = 8192;
struct Work {
  int64_t bytes;
  c10::DataPtr own;
  Work(int64_t n, at::Device device) : bytes(n) {
    if (n > kSmallWork) own = c10::GetAllocator(device.type())->allocate(static_cast<size_t>(n));
  }
  int64_t shared() const { return own.get() ? 0 : bytes; }
  void* in(const at::Tensor& shared) const { return own.get() ? own.get() : shared.data_ptr(); }
};

// The first n of them as a tuple.
PyObject* tuple_of(const std::vector<at::Tensor>& t, size_t n) {
  PyObject* out = PyTuple_New(static_cast<Py_ssize_t>(n));
  if (!out) return nullptr;
  for (size_t i = 0; i < n; ++i) {
    PyObject* o = nullptr;
    try {
      o = THPVariable_Wrap(t[i]);
    } catch (...) {
      Py_DECREF(out);
      throw;
    }
    if (!o) {
      Py_DECREF(out);
      return nullptr;
    }
    PyTuple_SET_ITEM(out, static_cast<Py_ssize_t>(i), o);
  }
  return out;
}

// empties(like, (type, size, ...), ...) -> a tuple of new tensors on like's device.
PyObject* empties(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n < 1 || n > 16 || !THPVariable_Check(args[0])) {
    PyErr_SetString(PyExc_TypeError, "empties takes a tensor and the results' types and sizes");
    return nullptr;
  }
  struct Given {
    int64_t v[4];
    size_t dims;
  };
  std::vector<Given> specs;
  for (Py_ssize_t i = 1; i < n; ++i) {
    Given g;
    bool ok = PyTuple_Check(args[i]) && PyTuple_GET_SIZE(args[i]) >= 1 && PyTuple_GET_SIZE(args[i]) <= 4;
    g.dims = ok ? static_cast<size_t>(PyTuple_GET_SIZE(args[i])) - 1 : 0;
    for (size_t d = 0; ok && d <= g.dims; ++d) {
      g.v[d] = PyLong_AsLongLong(PyTuple_GET_ITEM(args[i], static_cast<Py_ssize_t>(d)));
      if (PyErr_Occurred()) return nullptr;
      ok = g.v[d] >= 0;
    }
    if (!ok || g.v[0] >= static_cast<int64_t>(std::size(kTypes))) {
      PyErr_SetString(PyExc_ValueError, "a result is (type, size, ...), of at most three sizes");
      return nullptr;
    }
    specs.push_back(g);
  }
  const auto made = make(specs, [](const Given& g) {
    return std::pair<int, at::IntArrayRef>(static_cast<int>(g.v[0]), at::IntArrayRef(g.v + 1, g.dims));
  }, THPVariable_Unpack(args[0]).device());
  return tuple_of(made, made.size());
  END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------- arguments
int type_of(const at::Tensor& t) {
  for (int i = 0; i < 3; ++i)
    if (kTypes[i] == t.scalar_type()) return i;
  return -1;
}
bool plain(const at::Tensor& t) { return t.layout() == at::kStrided && (t.is_cuda() || (g_pretend && t.is_cpu())); }

// What a call's tensors have to share: the current GPU.
struct Where {
  at::Device device{at::kCPU};
  void* stream = nullptr;
  bool ok = false;
  explicit Where(const at::Tensor& t) {
    if (!plain(t)) return;
    device = t.device();
    if (t.is_cuda()) {
      if (device.index() != c10::cuda::current_device()) return;
      stream = c10::cuda::getCurrentCUDAStream(device.index()).stream();
    }
    ok = true;
  }
  bool here(const at::Tensor& t) const { return plain(t) && t.device() == device; }
};

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

// A matrix of one of the first three types with rows of unit stride that do not overlap.
struct Matrix {
  void* p;
  int64_t rows, cols, ld;
  int type;
};
bool matrix(const at::Tensor* t, const Where& w, Matrix& m) {
  if (!t || !w.here(*t) || t->dim() != 2 || (m.type = type_of(*t)) < 0) return false;
  m.rows = t->size(0);
  m.cols = t->size(1);
  if (m.cols < 1 || (t->stride(1) != 1 && m.cols != 1)) return false;
  m.ld = m.rows <= 1 ? m.cols : t->stride(0);
  m.p = t->data_ptr();
  return m.ld >= m.cols;
}
// A contiguous tensor of a type and sizes.
bool exact(const at::Tensor* t, const Where& w, at::ScalarType type, at::IntArrayRef sizes) {
  return t && w.here(*t) && t->scalar_type() == type && t->sizes() == sizes && t->is_contiguous();
}
// Offsets: their groups.
bool offsets(const at::Tensor* t, const Where& w, int64_t& groups) {
  if (!t || !w.here(*t) || t->scalar_type() != at::kInt || t->dim() != 1 || !t->is_contiguous()) return false;
  groups = t->size(0) - 1;
  return groups >= 1 && groups <= 0x7FFFFFFF;
}
bool places(const at::Tensor* t, const Where& w, int64_t& rows, int64_t& k) {
  if (!t || !w.here(*t) || t->scalar_type() != at::kInt || t->dim() != 2 || !t->is_contiguous()) return false;
  rows = t->size(0);
  k = t->size(1);
  return k >= 1 && k <= 0x7FFFFFFF;
}
template <typename T>
T* data(const at::Tensor* t) { return t ? static_cast<T*>(t->data_ptr()) : nullptr; }

template <typename A>
PyObject* number(A a) {
  if constexpr (std::is_pointer_v<A>) return PyLong_FromVoidPtr(const_cast<void*>(static_cast<const void*>(a)));
  else if constexpr (std::is_floating_point_v<A>) return PyFloat_FromDouble(a);
  else return PyLong_FromLongLong(static_cast<long long>(a));
}
template <typename... A>
int invoke(const Where& w, void* f, A... a) {
  if (w.device.is_cpu()) {
    Py_XDECREF(g_noted);
    g_noted = PyTuple_New(sizeof...(A));
    Py_ssize_t i = 0;
    if (g_noted) (PyTuple_SET_ITEM(g_noted, i++, number(a)), ...);
    return 0;
  }
  return f ? reinterpret_cast<int (*)(A...)>(f)(a...) : -1;
}
#define NONE_UNLESS(x) \
  do {                 \
    if (!(x)) Py_RETURN_NONE; \
  } while (0)

using at::IntArrayRef;
using P = void*;
using I = int64_t;

// ---------------------------------------------------------------- the calls
// route(logits, k, over all, learners)
PyObject* route(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor* z = n == 4 ? tensor(args[0]) : nullptr;
  NONE_UNLESS(z && PyLong_Check(args[1]));
  const Where w(*z);
  Matrix m;
  NONE_UNLESS(w.ok && matrix(z, w, m));
  int over = 0;
  const I k = PyLong_AsLongLongAndOverflow(args[1], &over), T = m.rows, E = m.cols;
  NONE_UNLESS(!over && k >= 1 && k <= 32 && k <= E && E <= 1024);
  const at::Tensor* learners = args[3] == Py_None ? nullptr : tensor(args[3]);
  I P_ = 0;
  NONE_UNLESS(args[3] == Py_None || offsets(learners, w, P_));
  const I G = E * std::max<I>(P_, 1);
  NONE_UNLESS(G <= 1024 && T * k <= I(1) << 27);
  const I bytes = T <= 32 && T * k <= 1024 ? 0 : 4 * 154 * G;           // no less than hier_avg_sort_workspace says
  const Work work(bytes, w.device);
  const auto r = results(w.device, {{kI32, {T, k}}, {kF32, {T, k}}, {kF32, {T}}, {kI32, {G + 1}}, {kI32, {T, k}}, {kI32, {T * k}},
                                    {kU8, {work.shared()}}});
  const int s = invoke<const void*, int, I, int, I, int, int, const int*, int, int*, float*, float*, int*, int*, int*, P, I, P>(
      w, g_route, m.p, m.type, T, static_cast<int>(E), m.ld, static_cast<int>(k), PyObject_IsTrue(args[2]) == 1, data<int>(learners),
      static_cast<int>(P_), data<int>(&r[0]), data<float>(&r[1]), data<float>(&r[2]), data<int>(&r[3]), data<int>(&r[4]),
      data<int>(&r[5]), work.in(r[6]), bytes, w.stream);
  NONE_UNLESS(s == 0);
  return tuple_of(r, 6);
  END_HANDLE_TH_ERRORS
}

// route_backward(dweights, logits, experts, weights, lse, over all)
PyObject* route_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor* z = n == 6 ? tensor(args[1]) : nullptr;
  NONE_UNLESS(z);
  const Where w(*z);
  Matrix m;
  const at::Tensor *dw = tensor(args[0]), *e = tensor(args[2]), *wt = tensor(args[3]);
  const at::Tensor* lse = args[4] == Py_None ? nullptr : tensor(args[4]);
  NONE_UNLESS(w.ok && matrix(z, w, m) && e && e->dim() == 2);
  const I T = m.rows, E = m.cols, k = e->size(1);
  const bool all = PyObject_IsTrue(args[5]) == 1;
  NONE_UNLESS(k >= 1 && k <= 32 && k <= E && E <= 1024 && (lse || (args[4] == Py_None && !all)));
  NONE_UNLESS(exact(e, w, at::kInt, {T, k}) && exact(wt, w, at::kFloat, {T, k}) && exact(dw, w, at::kFloat, {T, k}) &&
              (!lse || exact(lse, w, at::kFloat, {T})));
  const auto r = results(w.device, {{m.type, {T, E}}});
  const int s = invoke<const float*, const void*, int, I, int, I, int, int, const int*, const float*, const float*, P, I, P>(
      w, g_route_backward, data<float>(dw), m.p, m.type, T, static_cast<int>(E), m.ld, static_cast<int>(k), all, data<int>(e),
      data<float>(wt), data<float>(lse), r[0].data_ptr(), E, w.stream);
  NONE_UNLESS(s == 0);
  return THPVariable_Wrap(r[0]);
  END_HANDLE_TH_ERRORS
}

// dispatch(x, place, offsets)
PyObject* dispatch(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor* x = n == 3 ? tensor(args[0]) : nullptr;
  NONE_UNLESS(x);
  const Where w(*x);
  Matrix m;
  const at::Tensor *place = tensor(args[1]), *off = tensor(args[2]);
  I T, k, G;
  NONE_UNLESS(w.ok && matrix(x, w, m) && places(place, w, T, k) && offsets(off, w, G) && m.rows == T && m.cols <= 0x7FFFFFFF);
  const auto r = results(w.device, {{m.type, {T * k, m.cols}}});
  const int s = invoke<const void*, int, I, int, I, const int*, int, const int*, int, P, I, P>(
      w, g_dispatch, m.p, m.type, T, static_cast<int>(m.cols), m.ld, data<int>(place), static_cast<int>(k), data<int>(off),
      static_cast<int>(G), r[0].data_ptr(), m.cols, w.stream);
  NONE_UNLESS(s == 0);
  return THPVariable_Wrap(r[0]);
  END_HANDLE_TH_ERRORS
}

// combine(y, place, weights, out type)
PyObject* combine(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor* y = n == 4 ? tensor(args[0]) : nullptr;
  NONE_UNLESS(y);
  const Where w(*y);
  Matrix m;
  const at::Tensor *place = tensor(args[1]), *wt = args[2] == Py_None ? nullptr : tensor(args[2]);
  I T, k;
  NONE_UNLESS(w.ok && matrix(y, w, m) && places(place, w, T, k) && m.rows == T * k && m.cols <= 0x7FFFFFFF);
  NONE_UNLESS(args[2] == Py_None || exact(wt, w, at::kFloat, {T, k}));
  int type = m.type;
  if (args[3] != Py_None) {
    NONE_UNLESS(THPDtype_Check(args[3]));
    const at::ScalarType t = reinterpret_cast<THPDtype*>(args[3])->scalar_type;
    NONE_UNLESS(t == kTypes[type] || t == at::kFloat);
    if (t == at::kFloat) type = kF32;
  }
  const auto r = results(w.device, {{type, {T, m.cols}}});
  const int s = invoke<const void*, int, I, int, I, const int*, int, const float*, P, I, int, P>(
      w, g_combine, m.p, m.type, T, static_cast<int>(m.cols), m.ld, data<int>(place), static_cast<int>(k), data<float>(wt),
      r[0].data_ptr(), m.cols, type, w.stream);
  NONE_UNLESS(s == 0);
  return THPVariable_Wrap(r[0]);
  END_HANDLE_TH_ERRORS
}

// combine_backward(dout, y, place, weights, offsets)
PyObject* combine_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor* y = n == 5 ? tensor(args[1]) : nullptr;
  NONE_UNLESS(y);
  const Where w(*y);
  Matrix m, d;
  const at::Tensor *place = tensor(args[2]), *wt = tensor(args[3]), *off = tensor(args[4]);
  I T, k, G;
  NONE_UNLESS(w.ok && matrix(y, w, m) && matrix(tensor(args[0]), w, d) && places(place, w, T, k) && offsets(off, w, G));
  NONE_UNLESS(m.rows == T * k && d.rows == T && d.cols == m.cols && m.cols <= 0x7FFFFFFF && (d.type == m.type || d.type == kF32) &&
              exact(wt, w, at::kFloat, {T, k}));
  const auto r = results(w.device, {{m.type, {T * k, m.cols}}, {kF32, {T, k}}});
  const int s = invoke<const void*, int, I, const void*, int, I, int, I, const int*, int, const float*, const int*, int, P, I, float*, P>(
      w, g_combine_backward, d.p, d.type, d.ld, m.p, m.type, T, static_cast<int>(m.cols), m.ld, data<int>(place),
      static_cast<int>(k), data<float>(wt), data<int>(off), static_cast<int>(G), r[0].data_ptr(), m.cols, data<float>(&r[1]),
      w.stream);
  NONE_UNLESS(s == 0);
  return tuple_of(r, 2);
  END_HANDLE_TH_ERRORS
}

// verify(logits, drafts, uniform, noise, draft_probs, temperature, allowed)
PyObject* verify(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor* z = n == 7 ? tensor(args[0]) : nullptr;
  NONE_UNLESS(z && PyFloat_Check(args[5]));
  const Where w(*z);
  NONE_UNLESS(w.ok && z->dim() == 3 && type_of(*z) >= 0);
  const I B = z->size(0), R = z->size(1), V = z->size(2), K = R - 1;
  NONE_UNLESS(R >= 1 && R <= 1 << 20 && B <= 1 << 20 && V >= 1 && (z->stride(2) == 1 || V == 1));
  const at::Tensor *x = tensor(args[1]), *u = tensor(args[2]), *e = tensor(args[3]);
  const at::Tensor *q = args[4] == Py_None ? nullptr : tensor(args[4]), *ok = args[6] == Py_None ? nullptr : tensor(args[6]);
  NONE_UNLESS(exact(x, w, at::kInt, {B, K}) || exact(x, w, at::kLong, {B, K}));
  NONE_UNLESS(exact(u, w, at::kFloat, {B, K}) && e && w.here(*e) && e->scalar_type() == at::kFloat && e->sizes() == IntArrayRef({B, V}) &&
              (e->stride(1) == 1 || V == 1));
  NONE_UNLESS(args[4] == Py_None || (q && w.here(*q) && type_of(*q) >= 0 && q->sizes() == IntArrayRef({B, K, V}) && (q->stride(2) == 1 || V == 1)));
  const double temperature = PyFloat_AS_DOUBLE(args[5]);
  NONE_UNLESS(temperature >= 0x1p-126 && temperature <= 1e27);
  I ok_seq = 0, ok_row = 0;
  if (args[6] != Py_None) {
    NONE_UNLESS(ok && w.here(*ok) && (ok->scalar_type() == at::kBool || ok->scalar_type() == at::kByte));
    if (ok->dim() == 3) {
      NONE_UNLESS(ok->sizes() == z->sizes());
      ok_seq = ok->stride(0);
      ok_row = ok->stride(1);
    } else {
      NONE_UNLESS(ok->dim() == 1 && ok->size(0) == V);
    }
    NONE_UNLESS(ok->stride(-1) == 1 || V == 1);
  }
  const I bytes = B * (272 * R + 2052);                                 // as hier_avg_verify_workspace says
  const Work work(bytes, w.device);
  const auto r = results(w.device, {{kI32, {B, R}}, {kI32, {B}}, {kF32, {B, R}}, {kU8, {work.shared()}}});
  const int s = invoke<const void*, int, I, int, I, I, I, const void*, int, const float*, const float*, I, const void*, int, I, I,
                       const uint8_t*, I, I, double, int*, int*, float*, P, I, P>(
      w, g_verify, z->data_ptr(), type_of(*z), B, static_cast<int>(K), V, z->stride(0), z->stride(1), x->data_ptr(),
      x->scalar_type() == at::kInt ? 4 : 8, data<float>(u), data<float>(e), e->stride(0), q ? q->data_ptr() : nullptr,
      q ? type_of(*q) : 0, q ? q->stride(0) : 0, q ? q->stride(1) : 0, data<uint8_t>(ok), ok_seq, ok_row, temperature,
      data<int>(&r[0]), data<int>(&r[1]), data<float>(&r[2]), work.in(r[3]), bytes, w.stream);
  NONE_UNLESS(s == 0);
  return tuple_of(r, 3);
  END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------- lists of gradients
constexpr int64_t kPretended = 1 << 20;  // the device of CPU tensors that stand for a GPU's
struct Facts {
  std::vector<void*> address;
  std::vector<int> type;
  std::vector<int64_t> elements;
  int64_t device = -5;      // -1: a tensor is not on a GPU; -2: they are on several; -3: one is not contiguous or of another type;
                            // -4: one is no tensor
};
Facts read(PyObject* seq) {
  Facts f;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
  f.address.resize(n);
  f.type.resize(n);
  f.elements.resize(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor* t = tensor(PySequence_Fast_GET_ITEM(seq, i));
    if (!t) f.device = -4;
    else if (!t->is_cuda() && !(g_pretend && t->is_cpu())) f.device = -1;
    else if (type_of(*t) < 0 || t->layout() != at::kStrided || !t->is_contiguous()) f.device = -3;
    else if (const int64_t d = t->is_cuda() ? t->get_device() : kPretended; f.device != -5 && f.device != d) f.device = -2;
    else f.device = d;
    if (f.device < 0) return f;
    f.address[i] = t->data_ptr();
    f.type[i] = type_of(*t);
    f.elements[i] = t->numel();
  }
  return f;
}
struct Sequence {
  PyObject* o;
  explicit Sequence(PyObject* list) : o(PySequence_Fast(list, "a sequence of tensors")) {}
  ~Sequence() { Py_XDECREF(o); }
};

// facts(list) -> (addresses, types, elements, device), the first three as the bytes of uint64, int32 and int64 arrays.
PyObject* facts(PyObject*, PyObject* list) {
  HANDLE_TH_ERRORS
  const Sequence seq(list);
  if (!seq.o) return nullptr;
  const Facts f = read(seq.o);
  auto bytes = [](const auto& v) {
    return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(v.data()), static_cast<Py_ssize_t>(v.size() * sizeof(v[0])));
  };
  return Py_BuildValue("(NNNL)", bytes(f.address), bytes(f.type), bytes(f.elements), static_cast<long long>(f.device));
  END_HANDLE_TH_ERRORS
}

// norm(grads, max_norm, learners, clip) -> (norm, scale or None)
PyObject* norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  NONE_UNLESS(n == 4 && (PyList_Check(args[0]) || PyTuple_Check(args[0])));
  const Sequence seq(args[0]);
  NONE_UNLESS(seq.o && PySequence_Fast_GET_SIZE(seq.o) >= 1);
  const Facts f = read(seq.o);
  NONE_UNLESS(f.device >= 0);
  const Where w(*tensor(PySequence_Fast_GET_ITEM(seq.o, 0)));
  NONE_UNLESS(w.ok);
  I P_ = 1;
  if (args[2] != Py_None) {
    int over = 0;
    NONE_UNLESS(PyLong_Check(args[2]));
    P_ = PyLong_AsLongLongAndOverflow(args[2], &over);
    NONE_UNLESS(!over && P_ >= 1 && P_ <= 0x7FFFFFFF);
    for (size_t i = 0; i < f.address.size(); ++i) {
      const at::Tensor* t = tensor(PySequence_Fast_GET_ITEM(seq.o, static_cast<Py_ssize_t>(i)));
      NONE_UNLESS(t->dim() >= 1 && t->size(0) == P_);
    }
  }
  const bool scaled = args[1] != Py_None, clip = PyObject_IsTrue(args[3]) == 1;
  NONE_UNLESS(!scaled || PyFloat_Check(args[1]));
  const double most = scaled ? PyFloat_AS_DOUBLE(args[1]) : 0.0;
  NONE_UNLESS(most >= 0.0 && most <= std::numeric_limits<double>::max());
  const int count = static_cast<int>(f.address.size());
  I total = 0, pieces = 0;                                              // no less than hier_avg_grad_norm_workspace says
  for (int i = 0; i < count; ++i) {
    total += f.elements[i] * (f.type[i] == kF32 ? 4 : 2);
    pieces += f.elements[i] > 0 ? P_ : 0;
  }
  const I bytes = 8 * (total / (total < 8192 * pieces ? 2048 : 32768) + pieces + 1);
  const Work work(bytes, w.device);
  const auto r = results(w.device, {{kF32, {P_}}, {kF32, {P_}}, {kU8, {work.shared()}}});
  const int s = invoke<int, void* const*, const int*, const I*, int, double, int, float*, float*, P, I, P>(
      w, g_norm, count, f.address.data(), f.type.data(), f.elements.data(), static_cast<int>(P_), most, clip, data<float>(&r[0]),
      scaled ? data<float>(&r[1]) : nullptr, work.in(r[2]), bytes, w.stream);
  NONE_UNLESS(s == 0);
  PyObject* out = tuple_of(r, 2);
  if (out && !scaled) {
    Py_INCREF(Py_None);
    Py_DECREF(PyTuple_GET_ITEM(out, 1));
    PyTuple_SET_ITEM(out, 1, Py_None);
  }
  return out;
  END_HANDLE_TH_ERRORS
}

// bind(addresses of the C ABI's functions): route, route_backward, dispatch, combine, combine_backward, verify_drafts, grad_norm
PyObject* bind(PyObject*, PyObject* args) {
  void** const to[] = {&g_route, &g_route_backward, &g_dispatch, &g_combine, &g_combine_backward, &g_verify, &g_norm};
  if (!PyTuple_Check(args) || PyTuple_GET_SIZE(args) != static_cast<Py_ssize_t>(std::size(to))) {
    PyErr_SetString(PyExc_TypeError, "bind takes the functions' addresses");
    return nullptr;
  }
  for (size_t i = 0; i < std::size(to); ++i) {
    *to[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args, static_cast<Py_ssize_t>(i)));
    if (PyErr_Occurred()) return nullptr;
  }
  Py_RETURN_NONE;
}

// pretend(on) -> the arguments of the last call that was noted (for tests without a GPU)
PyObject* pretend(PyObject*, PyObject* on) {
  g_pretend = PyObject_IsTrue(on) == 1;
  PyObject* last = g_noted;
  g_noted = nullptr;
  if (last) return last;
  Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(empties), FAST(route), FAST(route_backward), FAST(dispatch), FAST(combine), FAST(combine_backward),
                         FAST(verify), FAST(norm), {"facts", facts, METH_O, nullptr}, {"bind", bind, METH_VARARGS, nullptr},
                         {"pretend", pretend, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&module); }
