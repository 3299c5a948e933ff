// Native half of the Python binding (diffopt.py, tree.py): argument checks,
// address extraction and the C ABI call of one entry point in one function
// call, and the host part of a tree operation over a list of leaves.
//
// In Python an entry point spent about 0.6 us on the checks of each operand
// and 3 us in ctypes (the 5-step leaf-direct driver on a 6-leaf tree: 12 us a
// call, its kernel 3.7 us); leaf_pointers replaces a Python loop, a tensor
// built from a list of ints and a copy into pinned memory.
//
// Every function here handles the ordinary case (plain tensors and parameters
// that pass every check) and returns None for anything else; the Python
// caller then takes its own path, which accepts or refuses the arguments with
// its own messages.  No check is remembered from one call to the next.
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/torch.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>
#include <utility>
#include <vector>

#include "diffopt.h"

namespace {

// An argument that the ordinary path does not take.
struct Other {};

// The tensor an object is, if it is exactly a torch.Tensor or a Parameter.
const at::Tensor& tensor_of(PyObject* o) {
  if (!THPVariable_CheckExact(o)) throw Other{};
  return THPVariable_Unpack(o);
}

constexpr int64_t kAnyCount = -1;  // an operand of any number of elements

// Address of a contiguous device tensor of this type with n elements; None is
// the null pointer, an int an address.
void* address(PyObject* o, at::ScalarType type, int64_t n) {
  if (o == Py_None) return nullptr;
  if (PyLong_CheckExact(o)) {
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) {
      PyErr_Clear();
      throw Other{};
    }
    return p;
  }
  const at::Tensor& t = tensor_of(o);
  if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous() || (n != kAnyCount && t.numel() != n)) throw Other{};
  return t.data_ptr();
}

constexpr Py_ssize_t kMaxList = 256;  // entries of one operand list on the ordinary path

// One C argument made from one Python argument.
struct Slot {
  void* p = nullptr;
  int64_t i = 0;
  double d = 0.0;
  void* list[kMaxList];
};

template <class T>
struct Arg;

template <class T, at::ScalarType TYPE>
struct PointerArg {
  static T get(Slot& s) { return static_cast<T>(s.p); }
  static void set(Slot& s, PyObject* o, int64_t n) { s.p = address(o, TYPE, n); }
};
template <>
struct Arg<const float*> : PointerArg<const float*, at::kFloat> {};
template <>
struct Arg<float*> : PointerArg<float*, at::kFloat> {};
template <>
struct Arg<const uint64_t*> : PointerArg<const uint64_t*, at::kLong> {};

// A host array of addresses, from a list or tuple.
template <class T, at::ScalarType TYPE>
struct ListArg {
  static T get(Slot& s) { return reinterpret_cast<T>(s.list); }
  static void set(Slot& s, PyObject* o, int64_t n) {
    if (!PyList_CheckExact(o) && !PyTuple_CheckExact(o)) throw Other{};
    const Py_ssize_t k = PySequence_Fast_GET_SIZE(o);
    if (k > kMaxList) throw Other{};
    PyObject** items = PySequence_Fast_ITEMS(o);
    for (Py_ssize_t j = 0; j < k; ++j) s.list[j] = address(items[j], TYPE, n);
  }
};
template <>
struct Arg<const float* const*> : ListArg<const float* const*, at::kFloat> {};
template <>
struct Arg<float* const*> : ListArg<float* const*, at::kFloat> {};
template <>
struct Arg<const uint64_t* const*> : ListArg<const uint64_t* const*, at::kLong> {};

// Opaque addresses: a segment table's handle, a stream.
template <class T>
struct HandleArg {
  static T get(Slot& s) { return static_cast<T>(s.p); }
  static void set(Slot& s, PyObject* o, int64_t) {
    if (o != Py_None && !PyLong_CheckExact(o)) throw Other{};
    s.p = address(o, at::kLong, kAnyCount);
  }
};
template <>
struct Arg<const diffopt_segtable*> : HandleArg<const diffopt_segtable*> {};
template <>
struct Arg<void*> : HandleArg<void*> {};

template <class T>
struct IntArg {
  static T get(Slot& s) { return static_cast<T>(s.i); }
  static void set(Slot& s, PyObject* o, int64_t) {
    if (!PyLong_Check(o)) throw Other{};
    s.i = std::is_unsigned_v<T> ? static_cast<int64_t>(PyLong_AsUnsignedLongLong(o)) : PyLong_AsLongLong(o);
    if ((s.i == -1 && PyErr_Occurred()) || (sizeof(T) == 4 && s.i != static_cast<int32_t>(s.i))) {
      PyErr_Clear();
      throw Other{};
    }
  }
};
template <>
struct Arg<int64_t> : IntArg<int64_t> {};
template <>
struct Arg<uint64_t> : IntArg<uint64_t> {};
template <>
struct Arg<int32_t> : IntArg<int32_t> {};

template <>
struct Arg<double> {
  static double get(Slot& s) { return s.d; }
  static void set(Slot& s, PyObject* o, int64_t) {
    if (PyFloat_CheckExact(o)) {
      s.d = PyFloat_AS_DOUBLE(o);
    } else if (PyLong_Check(o)) {
      s.d = PyLong_AsDouble(o);
      if (s.d == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Other{};
      }
    } else {
      throw Other{};
    }
  }
};

template <class... A, size_t... I>
int invoke(int (*fn)(A...), Slot* s, PyObject* const* args, int64_t n, std::index_sequence<I...>) {
  (Arg<A>::set(s[I], args[I], n), ...);
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(Arg<A>::get(s[I])...);
  Py_END_ALLOW_THREADS
  return rc;
}

template <class... A>
PyObject* call(int (*fn)(A...), PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != static_cast<Py_ssize_t>(sizeof...(A)) + 1) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    Slot count;
    if (args[0] != Py_None) Arg<int64_t>::set(count, args[0], 0);
    if (count.i < 0) throw Other{};  // no tensor has that many elements
    const int64_t n = args[0] == Py_None ? kAnyCount : count.i;
    Slot slots[sizeof...(A)];
    return PyLong_FromLong(invoke(fn, slots, args + 1, n, std::index_sequence_for<A...>{}));
  } catch (...) {  // an argument of another kind, or a tensor without storage
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (n, then the C arguments) -> return code, or None: n is the element count
// that every tensor operand must have (None: any).
template <auto FN>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return call(FN, args, nargs);
}

// The interpreter lock given up for a scope.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

// leaf_pointers(groups, device index) -> list with, per group of leaves, a
// device int64 tensor of their addresses (None for None): slices of one device
// tensor, filled by one asynchronous copy from pinned host memory on the
// current stream.  The addresses are listed under the interpreter lock, the
// allocations and the copy, which can wait for the runtime, run without it.
PyObject* leaf_pointers(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 2 || (!PyList_CheckExact(args[0]) && !PyTuple_CheckExact(args[0]))) Py_RETURN_NONE;
  PyObject* out = nullptr;
  try {
    const long device = PyLong_AsLong(args[1]);
    if (device == -1 && PyErr_Occurred()) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    const Py_ssize_t k = PySequence_Fast_GET_SIZE(args[0]);
    PyObject** groups = PySequence_Fast_ITEMS(args[0]);
    std::vector<int64_t> addresses, lengths(static_cast<size_t>(k), -1);  // -1: None
    for (Py_ssize_t g = 0; g < k; ++g) {
      if (groups[g] == Py_None) continue;
      if (!PyList_CheckExact(groups[g]) && !PyTuple_CheckExact(groups[g])) throw Other{};
      const Py_ssize_t len = PySequence_Fast_GET_SIZE(groups[g]);
      PyObject** leaves = PySequence_Fast_ITEMS(groups[g]);
      for (Py_ssize_t j = 0; j < len; ++j) {
        const at::Tensor& t = tensor_of(leaves[j]);
        if (!t.is_contiguous()) throw Other{};
        addresses.push_back(reinterpret_cast<int64_t>(t.data_ptr()));
      }
      lengths[static_cast<size_t>(g)] = len;
    }
    at::Tensor dev;
    {
      const Unlocked unlocked;
      const auto opts = at::TensorOptions().dtype(at::kLong);
      const at::Tensor host = at::empty({static_cast<int64_t>(addresses.size())}, opts.pinned_memory(true));
      std::copy(addresses.begin(), addresses.end(), host.data_ptr<int64_t>());
      dev = host.to(opts.device(at::kCUDA, static_cast<at::DeviceIndex>(device)), /*non_blocking=*/true);
    }
    out = PyList_New(k);
    if (!out) return nullptr;
    int64_t at = 0;
    for (Py_ssize_t g = 0; g < k; ++g) {
      const int64_t len = lengths[static_cast<size_t>(g)];
      if (len < 0) {
        Py_INCREF(Py_None);
        PyList_SET_ITEM(out, g, Py_None);
        continue;
      }
      PyObject* t = THPVariable_Wrap(dev.narrow(0, at, len));
      if (!t) {
        Py_DECREF(out);
        return nullptr;
      }
      PyList_SET_ITEM(out, g, t);
      at += len;
    }
    return out;
  } catch (...) {
    Py_XDECREF(out);
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// leaf_shapes(leaves) -> tuple of the leaves' shapes (tuples of ints) if they
// are plain tensors of one dtype on one device, else None.
PyObject* leaf_shapes(PyObject*, PyObject* leaves) {
  if (!PyList_CheckExact(leaves) || PyList_GET_SIZE(leaves) == 0) Py_RETURN_NONE;
  const Py_ssize_t k = PyList_GET_SIZE(leaves);
  PyObject* out = PyTuple_New(k);
  if (!out) return nullptr;
  try {
    const at::Tensor& first = tensor_of(PyList_GET_ITEM(leaves, 0));
    for (Py_ssize_t j = 0; j < k; ++j) {
      const at::Tensor& t = tensor_of(PyList_GET_ITEM(leaves, j));
      if (t.scalar_type() != first.scalar_type() || t.device() != first.device()) throw Other{};
      const auto sizes = t.sizes();
      PyObject* shape = PyTuple_New(static_cast<Py_ssize_t>(sizes.size()));
      if (!shape) {
        Py_DECREF(out);
        return nullptr;
      }
      PyTuple_SET_ITEM(out, j, shape);
      for (size_t d = 0; d < sizes.size(); ++d) {
        PyObject* v = PyLong_FromLongLong(sizes[d]);
        if (!v) {
          Py_DECREF(out);
          return nullptr;
        }
        PyTuple_SET_ITEM(shape, static_cast<Py_ssize_t>(d), v);
      }
    }
    return out;
  } catch (...) {
    Py_DECREF(out);
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// ---- language-model operators (operators.py) --------------------------------
// Whole calls: the operands' types, shapes and strides are checked, the
// workspace is allocated where none is given, and the entry point is called.

const at::Tensor* optional_tensor(PyObject* o) { return o == Py_None ? nullptr : &tensor_of(o); }

int32_t element_type(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return DIFFOPT_F32;
  if (t.scalar_type() == at::kBFloat16) return DIFFOPT_BF16;
  throw Other{};
}

// What the operands of a call have in common, and the call's arguments.
struct Call {
  PyObject* const* args;
  Py_ssize_t at = 0;
  const at::Tensor* like = nullptr;  // its element type and device

  PyObject* next() { return args[at++]; }

  void check(const at::Tensor& t, at::ScalarType type, at::IntArrayRef shape) const {
    if (!t.is_cuda() || t.scalar_type() != type || t.device() != like->device() || t.sizes() != shape) throw Other{};
  }
  // The operands live on the device that the call launches on.
  void current() const {
    if (like->device() != c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice()) throw Other{};
  }
  // A result's elements must not overlap (diffopt.operators._apart).
  static void apart(const at::Tensor& t) {
    if (t.is_contiguous()) return;
    int64_t strides[4], sizes[4];
    const int n = static_cast<int>(t.dim());
    for (int i = 0; i < n; ++i) {
      int j = i;
      for (; j > 0 && strides[j - 1] > t.stride(i); --j) {
        strides[j] = strides[j - 1];
        sizes[j] = sizes[j - 1];
      }
      strides[j] = t.stride(i);
      sizes[j] = t.size(i);
    }
    int64_t end = 1;
    for (int i = 0; i < n; ++i) {
      if (sizes[i] <= 1) continue;
      if (strides[i] < end) throw Other{};
      end += strides[i] * (sizes[i] - 1);
    }
  }
  // [B, T, heads, width]
  diffopt_heads heads(PyObject* o, at::IntArrayRef shape, bool result) const {
    const at::Tensor& t = tensor_of(o);
    check(t, like->scalar_type(), shape);
    if (shape[3] > 1 && t.stride(3) != 1 && t.numel() > 0) throw Other{};
    if (result) apart(t);
    return diffopt_heads{t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
  }
  // [B, heads, width], as one token
  diffopt_heads token(PyObject* o, at::IntArrayRef shape, bool result) const {
    const at::Tensor& t = tensor_of(o);
    check(t, like->scalar_type(), shape);
    if (shape[2] > 1 && t.stride(2) != 1 && t.numel() > 0) throw Other{};
    if (result) apart(t);
    return diffopt_heads{t.data_ptr(), t.stride(0), 0, t.stride(1)};
  }
  // [B, T, width]
  diffopt_heads seq(PyObject* o, at::IntArrayRef shape, bool result) const {
    const at::Tensor& t = tensor_of(o);
    check(t, like->scalar_type(), shape);
    if (shape[2] > 1 && t.stride(2) != 1 && t.numel() > 0) throw Other{};
    if (result) apart(t);
    return diffopt_heads{t.data_ptr(), t.stride(0), t.stride(1), 0};
  }
  // [B, width], as one token
  diffopt_heads row(PyObject* o, at::IntArrayRef shape, bool result) const {
    const at::Tensor& t = tensor_of(o);
    check(t, like->scalar_type(), shape);
    if (shape[1] > 1 && t.stride(1) != 1 && t.numel() > 0) throw Other{};
    if (result) apart(t);
    return diffopt_heads{t.data_ptr(), t.stride(0), 0, 0};
  }
  void* flat(PyObject* o, at::ScalarType type, at::IntArrayRef shape, bool optional = false) const {
    if (optional && o == Py_None) return nullptr;
    const at::Tensor& t = tensor_of(o);
    check(t, type, shape);
    if (!t.is_contiguous()) throw Other{};
    return t.data_ptr();
  }
  float* floats(PyObject* o, at::IntArrayRef shape, bool optional = false) const {
    return static_cast<float*>(flat(o, at::kFloat, shape, optional));
  }
  double number(PyObject* o) const {
    Slot s;
    Arg<double>::set(s, o, 0);
    return s.d;
  }
  int64_t integer(PyObject* o) const {
    Slot s;
    Arg<int64_t>::set(s, o, 0);
    return s.i;
  }
  void* stream(PyObject* o) const {
    Slot s;
    Arg<void*>::set(s, o, 0);
    return s.p;
  }
};

// A call's scratch memory: the caller's, or allocated on the current stream.
struct Scratch {
  at::Tensor own;
  void* p = nullptr;
  int64_t bytes = 0;
  Scratch(PyObject* given, int64_t need, const at::Tensor& like) {
    if (need < 0) throw Other{};
    if (given != Py_None) {
      const at::Tensor& t = tensor_of(given);
      if (t.scalar_type() != at::kByte || t.device() != like.device() || !t.is_contiguous() || t.numel() < need) throw Other{};
      p = t.data_ptr();
      bytes = t.numel();
    } else if (need > 0) {
      own = at::empty({need}, like.options().dtype(at::kByte));
      p = own.data_ptr();
      bytes = need;
    }
  }
};

template <class F>
PyObject* operator_call(PyObject* const* args, Py_ssize_t nargs, Py_ssize_t want, Py_ssize_t like, F f) {
  if (nargs != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    Call c{args};
    c.like = &tensor_of(args[like]);
    if (!c.like->is_cuda()) throw Other{};
    return PyLong_FromLong(f(c, element_type(*c.like)));
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

template <class F>
int unlocked(F f) {
  const Unlocked scope;
  return f();
}

// (q, k, v, log_decay, out, state, state_out, lengths, scale, workspace, stream)
PyObject* linattn_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 11, 0, [](Call& c, int32_t type) {
    const at::Tensor &q = *c.like, &k = tensor_of(c.args[1]), &v = tensor_of(c.args[2]);
    if (q.dim() != 4 || k.dim() != 4 || v.dim() != 4) throw Other{};
    const int64_t B = q.size(0), T = q.size(1), H = q.size(2), Dk = q.size(3), Hk = k.size(2), Dv = v.size(3);
    const diffopt_heads Q = c.heads(c.next(), {B, T, H, Dk}, false), K = c.heads(c.next(), {B, T, Hk, Dk}, false),
                        V = c.heads(c.next(), {B, T, Hk, Dv}, false);
    const float* lg = c.floats(c.next(), {Hk});
    const diffopt_heads O = c.heads(c.next(), {B, T, H, Dv}, true);
    const float* s0 = c.floats(c.next(), {B, Hk, Dk, Dv}, true);
    float* s1 = c.floats(c.next(), {B, Hk, Dk, Dv}, true);
    const int32_t* n = static_cast<int32_t*>(c.flat(c.next(), at::kInt, {B}, true));
    const double scale = c.number(c.next());
    const Scratch w(c.next(), diffopt_linattn_workspace(B, T, H, Hk, Dk, Dv, type, 0), q);
    void* stream = c.stream(c.next());
    return unlocked([&] { return diffopt_linattn_fwd(&Q, &K, &V, lg, n, s0, B, T, H, Hk, Dk, Dv, type, scale, &O, s1, w.p, w.bytes, stream); });
  });
}

// (dout, q, k, v, log_decay, dq, dk, dv, state, dstate_out, dstate, lengths, scale, workspace, stream)
PyObject* linattn_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 15, 1, [](Call& c, int32_t type) {
    const at::Tensor &q = *c.like, &k = tensor_of(c.args[2]), &v = tensor_of(c.args[3]);
    if (q.dim() != 4 || k.dim() != 4 || v.dim() != 4) throw Other{};
    const int64_t B = q.size(0), T = q.size(1), H = q.size(2), Dk = q.size(3), Hk = k.size(2), Dv = v.size(3);
    const diffopt_heads DO = c.heads(c.next(), {B, T, H, Dv}, false), Q = c.heads(c.next(), {B, T, H, Dk}, false),
                        K = c.heads(c.next(), {B, T, Hk, Dk}, false), V = c.heads(c.next(), {B, T, Hk, Dv}, false);
    const float* lg = c.floats(c.next(), {Hk});
    diffopt_heads out[3];
    const diffopt_heads* d[3];
    for (int i = 0; i < 3; ++i) {
      PyObject* o = c.next();
      d[i] = o == Py_None ? nullptr : &out[i];
      if (d[i]) out[i] = c.heads(o, {B, T, i ? Hk : H, i < 2 ? Dk : Dv}, true);
    }
    const float *s0 = c.floats(c.next(), {B, Hk, Dk, Dv}, true), *ds1 = c.floats(c.next(), {B, Hk, Dk, Dv}, true);
    float* ds0 = c.floats(c.next(), {B, Hk, Dk, Dv}, true);
    const int32_t* n = static_cast<int32_t*>(c.flat(c.next(), at::kInt, {B}, true));
    const double scale = c.number(c.next());
    const Scratch w(c.next(), diffopt_linattn_workspace(B, T, H, Hk, Dk, Dv, type, 1), q);
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_linattn_bwd(&DO, ds1, &Q, &K, &V, lg, n, s0, B, T, H, Hk, Dk, Dv, type, scale, d[0], d[1], d[2], ds0, w.p, w.bytes,
                                 stream);
    });
  });
}

// (q, k, v, log_decay, state, out, scale, stream)
PyObject* linattn_step(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 8, 0, [](Call& c, int32_t type) {
    const at::Tensor &q = *c.like, &k = tensor_of(c.args[1]), &v = tensor_of(c.args[2]);
    if (q.dim() != 3 || k.dim() != 3 || v.dim() != 3) throw Other{};
    const int64_t B = q.size(0), H = q.size(1), Dk = q.size(2), Hk = k.size(1), Dv = v.size(2);
    const diffopt_heads Q = c.token(c.next(), {B, H, Dk}, false), K = c.token(c.next(), {B, Hk, Dk}, false),
                        V = c.token(c.next(), {B, Hk, Dv}, false);
    const float* lg = c.floats(c.next(), {Hk});
    float* state = c.floats(c.next(), {B, Hk, Dk, Dv});
    const diffopt_heads O = c.token(c.next(), {B, H, Dv}, true);
    const double scale = c.number(c.next());
    void* stream = c.stream(c.next());
    return unlocked([&] { return diffopt_linattn_step(&Q, &K, &V, lg, B, H, Hk, Dk, Dv, type, scale, state, &O, stream); });
  });
}

// What the three directions of qknorm_rope share.
struct QkNorm {
  int64_t B, T, H, Hk, D, rows = 0, half = 0;
  const float *wq, *wk, *cos = nullptr, *sin = nullptr;
  const void* positions = nullptr;
  int32_t position_bytes = 0;

  QkNorm(const at::Tensor& q, PyObject* k) {
    if (q.dim() != 4) throw Other{};
    B = q.size(0);
    T = q.size(1);
    H = q.size(2);
    D = q.size(3);
    Hk = 0;
    if (const at::Tensor* t = optional_tensor(k)) {
      if (t->dim() != 4) throw Other{};
      Hk = t->size(2);
    }
  }
  // q_weight, k_weight, cos, sin
  void tables(Call& c) {
    wq = c.floats(c.next(), {D}, true);
    wk = c.floats(c.next(), {D}, true);
    PyObject *co = c.next(), *si = c.next();
    if (const at::Tensor* t = optional_tensor(co)) {
      if (t->dim() != 2) throw Other{};
      rows = t->size(0);
      half = t->size(1);
      cos = c.floats(co, {rows, half});
      sin = c.floats(si, {rows, half});
    }
  }
  void places(Call& c, PyObject* o) {
    if (const at::Tensor* t = optional_tensor(o)) {
      if (t->scalar_type() != at::kInt && t->scalar_type() != at::kLong) throw Other{};
      positions = c.flat(o, t->scalar_type(), {B, T});
      position_bytes = static_cast<int32_t>(t->element_size());
    }
  }
  // An operand of q and k; k's is not looked at without k heads.
  struct Pair {
    diffopt_heads q{}, k{};
    bool no_q = false, no_k = false;
    const diffopt_heads* pq() const { return no_q ? nullptr : &q; }
    const diffopt_heads* pk() const { return no_k ? nullptr : &k; }
  };
  Pair pair(Call& c, bool result, bool optional = false) const {
    Pair p;
    PyObject *q = c.next(), *k = c.next();
    p.no_q = optional && q == Py_None;
    p.no_k = Hk == 0 || (optional && k == Py_None);
    if (!p.no_q) p.q = c.heads(q, {B, T, H, D}, result);
    if (!p.no_k) p.k = c.heads(k, {B, T, Hk, D}, result);
    return p;
  }
  int64_t scratch(const float* a, const float* b) const { return a || b ? diffopt_qknorm_rope_workspace(B, T, H, Hk, D) : 0; }
};

// (q, k, q_weight, k_weight, cos, sin, q_out, k_out, positions, first, eps, interleaved, stream)
PyObject* qknorm_rope_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 13, 0, [](Call& c, int32_t type) {
    QkNorm n(*c.like, c.args[1]);
    const QkNorm::Pair x = n.pair(c, false);
    n.tables(c);
    const QkNorm::Pair y = n.pair(c, true);
    n.places(c, c.next());
    const int64_t first = c.integer(c.next());
    const double eps = c.number(c.next());
    const int32_t inter = c.next() == Py_True;
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_qknorm_rope_fwd(x.pq(), x.pk(), n.wq, n.wk, n.cos, n.sin, n.rows, n.positions, n.position_bytes, first, n.B, n.T, n.H,
                                     n.Hk, n.D, 2 * n.half, inter, type, eps, y.pq(), y.pk(), stream);
    });
  });
}

// (dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, dq, dk, dq_weight, dk_weight, positions, first, eps, interleaved, workspace, stream)
PyObject* qknorm_rope_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 18, 2, [](Call& c, int32_t type) {
    QkNorm n(*c.like, c.args[3]);
    const QkNorm::Pair dy = n.pair(c, false), x = n.pair(c, false);
    n.tables(c);
    const QkNorm::Pair dx = n.pair(c, true);
    float *dwq = c.floats(c.next(), {n.D}, true), *dwk = c.floats(c.next(), {n.D}, true);
    n.places(c, c.next());
    const int64_t first = c.integer(c.next());
    const double eps = c.number(c.next());
    const int32_t inter = c.next() == Py_True;
    const Scratch w(c.next(), n.scratch(dwq, dwk), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_qknorm_rope_bwd(dy.pq(), dy.pk(), x.pq(), x.pk(), n.wq, n.wk, n.cos, n.sin, n.rows, n.positions, n.position_bytes, first,
                                     n.B, n.T, n.H, n.Hk, n.D, 2 * n.half, inter, type, eps, dx.pq(), dx.pk(), dwq, dwk, w.p, w.bytes, stream);
    });
  });
}

// (ddq, ddk, ddq_weight, ddk_weight, dq_out, dk_out, q, k, q_weight, k_weight, cos, sin, out_dq_out, out_dk_out, out_q, out_k,
//  out_q_weight, out_k_weight, positions, first, eps, interleaved, workspace, stream)
PyObject* qknorm_rope_bwd_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 24, 6, [](Call& c, int32_t type) {
    QkNorm n(*c.like, c.args[7]);
    const QkNorm::Pair a = n.pair(c, false, true);
    const float *bq = c.floats(c.next(), {n.D}, true), *bk = c.floats(c.next(), {n.D}, true);
    const QkNorm::Pair dy = n.pair(c, false), x = n.pair(c, false);
    n.tables(c);
    const QkNorm::Pair oy = n.pair(c, true), ox = n.pair(c, true);
    float *owq = c.floats(c.next(), {n.D}, true), *owk = c.floats(c.next(), {n.D}, true);
    n.places(c, c.next());
    const int64_t first = c.integer(c.next());
    const double eps = c.number(c.next());
    const int32_t inter = c.next() == Py_True;
    const Scratch w(c.next(), n.scratch(owq, owk), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_qknorm_rope_bwd_bwd(a.pq(), a.pk(), bq, bk, dy.pq(), dy.pk(), x.pq(), x.pk(), n.wq, n.wk, n.cos, n.sin, n.rows,
                                         n.positions, n.position_bytes, first, n.B, n.T, n.H, n.Hk, n.D, 2 * n.half, inter, type, eps,
                                         oy.pq(), oy.pk(), ox.pq(), ox.pk(), owq, owk, w.p, w.bytes, stream);
    });
  });
}

// What the four calls of distill share: logits, ids, teacher, then the rest.
struct Distill {
  int64_t N, V, K, stride;
  const void *logits, *ids;
  const float* teacher;
  int32_t id_bytes;

  explicit Distill(Call& c) {
    PyObject *x = c.next(), *i = c.next(), *t = c.next();
    const at::Tensor &l = tensor_of(x), &e = tensor_of(i);
    if (l.dim() != 2 || e.dim() != 2 || (e.scalar_type() != at::kInt && e.scalar_type() != at::kLong)) throw Other{};
    N = l.size(0);
    V = l.size(1);
    K = e.size(1);
    logits = rows(c, x, false, &stride);
    ids = c.flat(i, e.scalar_type(), {N, K});
    id_bytes = static_cast<int32_t>(e.element_size());
    teacher = c.floats(t, {N, K});
  }
  void* rows(Call& c, PyObject* o, bool result, int64_t* step) const {
    const at::Tensor& t = tensor_of(o);
    c.check(t, c.like->scalar_type(), {N, V});
    if (V > 1 && t.stride(1) != 1 && t.numel() > 0) throw Other{};
    if (result) Call::apart(t);
    *step = t.stride(0);
    return t.data_ptr();
  }
};

// (logits, ids, teacher, loss, stats, temperature, workspace, stream)
PyObject* distill_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 8, 0, [](Call& c, int32_t type) {
    const Distill d(c);
    float *loss = c.floats(c.next(), {d.N}), *stats = c.floats(c.next(), {d.N, 2});
    const double T = c.number(c.next());
    const Scratch w(c.next(), diffopt_distill_workspace(d.N, d.V, type, d.K), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_distill_fwd(d.logits, d.stride, d.N, d.V, type, d.ids, d.id_bytes, d.teacher, d.K, T, loss, stats, w.p, w.bytes, stream);
    });
  });
}

// (dloss, logits, ids, teacher, stats, dlogits, dteacher, temperature, stream)
PyObject* distill_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 9, 1, [](Call& c, int32_t type) {
    PyObject* og = c.next();
    const Distill d(c);
    const float *g = c.floats(og, {d.N}), *stats = c.floats(c.next(), {d.N, 2});
    int64_t dstride;
    void* dx = d.rows(c, c.next(), true, &dstride);
    float* dt = c.floats(c.next(), {d.N, d.K}, true);
    const double T = c.number(c.next());
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_distill_bwd(g, d.logits, d.stride, d.N, d.V, type, d.ids, d.id_bytes, d.teacher, d.K, T, stats, dx, dstride, dt, stream);
    });
  });
}

// (dloss, logits, ids, teacher, loss, stats, dlogits, dteacher, temperature, workspace, stream)
PyObject* distill_fwd_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 11, 1, [](Call& c, int32_t type) {
    PyObject* og = c.next();
    const Distill d(c);
    const float* g = c.floats(og, {d.N});
    float *loss = c.floats(c.next(), {d.N}), *stats = c.floats(c.next(), {d.N, 2});
    int64_t dstride;
    void* dx = d.rows(c, c.next(), true, &dstride);
    float* dt = c.floats(c.next(), {d.N, d.K}, true);
    const double T = c.number(c.next());
    const Scratch w(c.next(), diffopt_distill_workspace(d.N, d.V, type, d.K), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_distill_fwd_bwd(g, d.logits, d.stride, d.N, d.V, type, d.ids, d.id_bytes, d.teacher, d.K, T, loss, stats, dx, dstride, dt,
                                     w.p, w.bytes, stream);
    });
  });
}

// (ddlogits, ddteacher, dloss, logits, ids, teacher, stats, out_dloss, out_logits, out_teacher, temperature, workspace, stream)
PyObject* distill_bwd_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 13, 3, [](Call& c, int32_t type) {
    PyObject *oa = c.next(), *oc = c.next(), *og = c.next();
    const Distill d(c);
    int64_t astride = 0, ostride;
    const void* a = oa == Py_None ? nullptr : d.rows(c, oa, false, &astride);
    const float *ct = c.floats(oc, {d.N, d.K}, true), *g = c.floats(og, {d.N}), *stats = c.floats(c.next(), {d.N, 2});
    float* out_g = c.floats(c.next(), {d.N}, true);
    void* out_x = d.rows(c, c.next(), true, &ostride);
    float* out_t = c.floats(c.next(), {d.N, d.K}, true);
    const double T = c.number(c.next());
    const Scratch w(c.next(), diffopt_distill_workspace(d.N, d.V, type, d.K), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_distill_bwd_bwd(a, astride, ct, g, d.logits, d.stride, d.N, d.V, type, d.ids, d.id_bytes, d.teacher, d.K, T, stats, out_g,
                                     out_x, ostride, out_t, w.p, w.bytes, stream);
    });
  });
}

// ---- global norm and clipping (diffopt.py) ----------------------------------

// (grad, max_norm, out, stats, eps, workspace, stream)
PyObject* clip_norm_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 7, 3, [](Call& c, int32_t) {
    c.current();
    const at::Tensor& g = tensor_of(c.args[0]);
    const float* grad = c.floats(c.next(), g.sizes());
    const double max_norm = c.number(c.next());
    PyObject* o = c.next();
    const at::Tensor* out = optional_tensor(o);
    if (out && out->numel() != g.numel()) throw Other{};
    float *po = out ? c.floats(o, out->sizes()) : nullptr, *stats = c.floats(c.next(), {2});
    const double eps = c.number(c.next());
    const int64_t n = g.numel();
    const Scratch w(c.next(), diffopt_clip_norm_workspace(n), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] { return diffopt_clip_norm_fwd(grad, n, max_norm, eps, po, stats, w.p, w.bytes, stream); });
  });
}

// A tensor of n fp32 elements of any shape, or None.
float* counted(Call& c, PyObject* o, int64_t n) {
  const at::Tensor* t = optional_tensor(o);
  if (!t) return nullptr;
  if (t->numel() != n) throw Other{};
  return c.floats(o, t->sizes());
}

// (dout, dnorm, grad, stats, dgrad, eps, workspace, stream)
PyObject* clip_norm_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 8, 3, [](Call& c, int32_t) {
    c.current();
    const int64_t n = tensor_of(c.args[2]).numel();
    const float *dout = counted(c, c.next(), n), *dnorm = counted(c, c.next(), 1), *grad = counted(c, c.next(), n), *stats = c.floats(c.next(), {2});
    float* dgrad = counted(c, c.next(), n);
    const double eps = c.number(c.next());
    const Scratch w(c.next(), diffopt_clip_norm_workspace(n), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] { return diffopt_clip_norm_bwd(dout, dnorm, grad, stats, n, eps, dgrad, w.p, w.bytes, stream); });
  });
}

const uint64_t* leaf_array(Call& c, PyObject* o, int64_t k) {
  return o == Py_None ? nullptr : static_cast<const uint64_t*>(c.flat(o, at::kLong, {k}));
}

// (leaves, table, grad, max_norm, out, stats, eps, workspace, stream)
PyObject* clip_norm_fwd_tree(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 9, 5, [](Call& c, int32_t) {
    c.current();
    const int64_t k = c.integer(c.next());
    const diffopt_segtable* table = static_cast<const diffopt_segtable*>(c.stream(c.next()));
    const uint64_t* grad = leaf_array(c, c.next(), k);
    const double max_norm = c.number(c.next());
    const uint64_t* out = leaf_array(c, c.next(), k);
    float* stats = c.floats(c.next(), {2});
    const double eps = c.number(c.next());
    const Scratch w(c.next(), diffopt_clip_norm_workspace_tree(table), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] { return diffopt_clip_norm_fwd_tree(table, grad, max_norm, eps, out, stats, w.p, w.bytes, stream); });
  });
}

// (leaves, table, dout, dnorm, grad, stats, dgrad, eps, workspace, stream)
PyObject* clip_norm_bwd_tree(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 10, 5, [](Call& c, int32_t) {
    c.current();
    const int64_t k = c.integer(c.next());
    const diffopt_segtable* table = static_cast<const diffopt_segtable*>(c.stream(c.next()));
    const uint64_t* dout = leaf_array(c, c.next(), k);
    const float* dnorm = counted(c, c.next(), 1);
    const uint64_t* grad = leaf_array(c, c.next(), k);
    const float* stats = c.floats(c.next(), {2});
    const uint64_t* dgrad = leaf_array(c, c.next(), k);
    const double eps = c.number(c.next());
    const Scratch w(c.next(), diffopt_clip_norm_workspace_tree(table), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] { return diffopt_clip_norm_bwd_tree(table, dout, dnorm, grad, stats, eps, dgrad, w.p, w.bytes, stream); });
  });
}

// ---- language-model operators, continued ------------------------------------

// What the calls of logprob share.
struct Logprob {
  int64_t N, V, stride, K = 0;
  const void *logits, *ids = nullptr;
  int32_t id_bytes = 0, top_bytes = 0;

  Logprob(Call& c, PyObject* x, PyObject* i) {
    if (c.like->dim() != 2) throw Other{};
    c.current();
    N = c.like->size(0);
    V = c.like->size(1);
    logits = rows(c, x, false, &stride);
    ids = tokens(c, i, {N}, &id_bytes);
  }
  void* rows(Call& c, PyObject* o, bool result, int64_t* step) const {
    const at::Tensor& t = tensor_of(o);
    c.check(t, c.like->scalar_type(), {N, V});
    if (V > 1 && t.stride(1) != 1 && t.numel() > 0) throw Other{};
    if (result) Call::apart(t);
    *step = t.stride(0);
    return t.data_ptr();
  }
  static void* tokens(Call& c, PyObject* o, at::IntArrayRef shape, int32_t* bytes) {
    const at::Tensor* t = optional_tensor(o);
    if (!t) return nullptr;
    if (t->scalar_type() != at::kInt && t->scalar_type() != at::kLong) throw Other{};
    *bytes = static_cast<int32_t>(t->element_size());
    return c.flat(o, t->scalar_type(), shape);
  }
  // a row's alternatives: values and ids, or neither
  struct Top {
    float* values = nullptr;
    void* ids = nullptr;
  };
  Top top(Call& c, PyObject* values, PyObject* i) {
    Top t;
    if (const at::Tensor* v = optional_tensor(values)) {
      if (v->dim() != 2 || i == Py_None) throw Other{};
      K = v->size(1);
      t.values = c.floats(values, {N, K});
      t.ids = tokens(c, i, {N, K}, &top_bytes);
    }
    return t;
  }
};

// (logits, ids, logprob, stats, entropy, top_logprob, top_ids, temperature, workspace, stream)
PyObject* logprob_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 10, 0, [](Call& c, int32_t type) {
    PyObject *x = c.next(), *i = c.next();
    Logprob d(c, x, i);
    float *lp = c.floats(c.next(), {d.N}, true), *stats = c.floats(c.next(), {d.N, 2}), *ent = c.floats(c.next(), {d.N}, true);
    PyObject *tv = c.next(), *ti = c.next();
    if (tv == Py_None && ti != Py_None) throw Other{};
    const Logprob::Top t = d.top(c, tv, ti);
    const double T = c.number(c.next());
    const Scratch w(c.next(), diffopt_logprob_workspace(d.N, d.V, type, d.K), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_logprob_fwd(d.logits, d.stride, d.N, d.V, type, d.ids, d.id_bytes, T, lp, ent, stats, t.values, t.ids, d.top_bytes, d.K, w.p,
                                 w.bytes, stream);
    });
  });
}

// (logits, ids, stats, dlogits, dlogprob, dentropy, entropy, dtop_logprob, top_ids, temperature, stream)
PyObject* logprob_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 11, 0, [](Call& c, int32_t type) {
    PyObject *x = c.next(), *i = c.next();
    Logprob d(c, x, i);
    const float* stats = c.floats(c.next(), {d.N, 2});
    int64_t dstride;
    void* dx = d.rows(c, c.next(), true, &dstride);
    const float *g = c.floats(c.next(), {d.N}, true), *h = c.floats(c.next(), {d.N}, true), *ent = c.floats(c.next(), {d.N}, true);
    PyObject *tv = c.next(), *ti = c.next();
    const Logprob::Top t = d.top(c, tv, ti);
    const double T = c.number(c.next());
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_logprob_bwd(g, h, ent, t.values, t.ids, d.top_bytes, d.K, d.logits, d.stride, d.N, d.V, type, d.ids, d.id_bytes, T, stats, dx,
                                 dstride, stream);
    });
  });
}

// (dlogprob, logits, ids, logprob, stats, dlogits, dentropy, entropy, temperature, workspace, stream)
PyObject* logprob_fwd_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 11, 1, [](Call& c, int32_t type) {
    PyObject *og = c.next(), *x = c.next(), *i = c.next();
    Logprob d(c, x, i);
    const float* g = c.floats(og, {d.N});
    float *lp = c.floats(c.next(), {d.N}), *stats = c.floats(c.next(), {d.N, 2});
    int64_t dstride;
    void* dx = d.rows(c, c.next(), true, &dstride);
    const float* h = c.floats(c.next(), {d.N}, true);
    float* ent = c.floats(c.next(), {d.N}, true);
    const double T = c.number(c.next());
    const Scratch w(c.next(), diffopt_logprob_workspace(d.N, d.V, type, 0), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_logprob_fwd_bwd(g, h, d.logits, d.stride, d.N, d.V, type, d.ids, d.id_bytes, T, lp, ent, stats, dx, dstride, w.p, w.bytes,
                                     stream);
    });
  });
}

// (ddlogits, logits, ids, stats, out_logits, dlogprob, dentropy, entropy, dtop_logprob, top_ids, out_dlogprob, out_dentropy,
//  out_dtop_logprob, temperature, workspace, stream)
PyObject* logprob_bwd_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 16, 1, [](Call& c, int32_t type) {
    PyObject *oa = c.next(), *x = c.next(), *i = c.next();
    Logprob d(c, x, i);
    int64_t astride, ostride;
    const void* a = d.rows(c, oa, false, &astride);
    const float* stats = c.floats(c.next(), {d.N, 2});
    void* out = d.rows(c, c.next(), true, &ostride);
    const float *g = c.floats(c.next(), {d.N}, true), *h = c.floats(c.next(), {d.N}, true), *ent = c.floats(c.next(), {d.N}, true);
    PyObject *tv = c.next(), *ti = c.next();
    const Logprob::Top t = d.top(c, tv, ti);
    float *out_g = c.floats(c.next(), {d.N}, true), *out_h = c.floats(c.next(), {d.N}, true);
    PyObject* ot = c.next();
    if (ot != Py_None && tv == Py_None) throw Other{};
    float* out_t = c.floats(ot, {d.N, d.K}, true);
    const double T = c.number(c.next());
    const Scratch w(c.next(), diffopt_logprob_workspace(d.N, d.V, type, 0), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_logprob_bwd_bwd(a, astride, g, h, ent, t.values, t.ids, d.top_bytes, d.K, d.logits, d.stride, d.N, d.V, type, d.ids, d.id_bytes, T,
                                     stats, out_g, out_h, out_t, out, ostride, w.p, w.bytes, stream);
    });
  });
}

// What the calls of gscan share: the sizes, and the operands' shape.
struct Gscan {
  int64_t B, T, C;
  explicit Gscan(const Call& c) {
    if (c.like->dim() != 3) throw Other{};
    c.current();
    B = c.like->size(0);
    T = c.like->size(1);
    C = c.like->size(2);
  }
  diffopt_heads seq(Call& c, bool result = false) const { return c.seq(c.next(), {B, T, C}, result); }
  float* state(Call& c) const { return c.floats(c.next(), {B, C}, true); }
  const int32_t* lengths(Call& c) const { return static_cast<int32_t*>(c.flat(c.next(), at::kInt, {B}, true)); }
};

// (log_gate, x, h, state, state_out, lengths, workspace, stream)
PyObject* gscan_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 8, 1, [](Call& c, int32_t type) {
    const Gscan g(c);
    const diffopt_heads lg = g.seq(c), x = g.seq(c), h = g.seq(c, true);
    const float* s0 = g.state(c);
    float* s1 = g.state(c);
    const int32_t* n = g.lengths(c);
    const Scratch w(c.next(), diffopt_gscan_workspace(g.B, g.T, g.C, type, 0), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] { return diffopt_gscan_fwd(&lg, &x, n, s0, g.B, g.T, g.C, type, &h, s1, w.p, w.bytes, stream); });
  });
}

// (dh, log_gate, x, dlog_gate, dx, state, dstate_out, dstate, lengths, workspace, stream)
PyObject* gscan_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 11, 2, [](Call& c, int32_t type) {
    const Gscan g(c);
    const diffopt_heads dh = g.seq(c), lg = g.seq(c), x = g.seq(c);
    diffopt_heads out[2];
    const diffopt_heads* d[2];
    for (int i = 0; i < 2; ++i) {
      PyObject* o = c.next();
      d[i] = o == Py_None ? nullptr : &out[i];
      if (d[i]) out[i] = c.seq(o, {g.B, g.T, g.C}, true);
    }
    const float *s0 = g.state(c), *ds1 = g.state(c);
    float* ds0 = g.state(c);
    const int32_t* n = g.lengths(c);
    const Scratch w(c.next(), diffopt_gscan_workspace(g.B, g.T, g.C, type, 1), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_gscan_bwd(&dh, ds1, &lg, &x, n, s0, g.B, g.T, g.C, type, d[0], d[1], ds0, w.p, w.bytes, stream);
    });
  });
}

// (ddlog_gate, ddx, dh, log_gate, x, out_dh, out_log_gate, out_x, state, dstate_out, ddstate, out_dstate_out, out_state, lengths,
//  workspace, stream)
PyObject* gscan_bwd_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 16, 4, [](Call& c, int32_t type) {
    const Gscan g(c);
    const diffopt_heads r = g.seq(c), p = g.seq(c), dh = g.seq(c), lg = g.seq(c), x = g.seq(c);
    const diffopt_heads oh = g.seq(c, true), og = g.seq(c, true), ox = g.seq(c, true);
    const float *s0 = g.state(c), *ds1 = g.state(c), *dds0 = g.state(c);
    float *o1 = g.state(c), *o0 = g.state(c);
    const int32_t* n = g.lengths(c);
    const Scratch w(c.next(), diffopt_gscan_workspace(g.B, g.T, g.C, type, 2), *c.like);
    void* stream = c.stream(c.next());
    return unlocked([&] {
      return diffopt_gscan_bwd_bwd(&r, &p, dds0, &dh, ds1, &lg, &x, n, s0, g.B, g.T, g.C, type, &oh, o1, &og, &ox, o0, w.p, w.bytes, stream);
    });
  });
}

// (log_gate, x, state, out, stream)
PyObject* gscan_step(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return operator_call(args, nargs, 5, 1, [](Call& c, int32_t type) {
    if (c.like->dim() != 2) throw Other{};
    c.current();
    const int64_t B = c.like->size(0), C = c.like->size(1);
    const diffopt_heads lg = c.row(c.next(), {B, C}, false), x = c.row(c.next(), {B, C}, false);
    float* state = c.floats(c.next(), {B, C});
    const diffopt_heads out = c.row(c.next(), {B, C}, true);
    void* stream = c.stream(c.next());
    return unlocked([&] { return diffopt_gscan_step(&lg, &x, B, C, type, state, &out, stream); });
  });
}

#define ENTRY(name) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<&diffopt_##name>)), METH_FASTCALL, nullptr}

#define OPERATOR(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&name)), METH_FASTCALL, nullptr}

PyMethodDef methods[] = {
    ENTRY(adam_fwd),
    ENTRY(adam_bwd),
    ENTRY(adam_unrolled_fwd),
    ENTRY(adam_unrolled_bwd),
    ENTRY(adam_fwd_tree),
    ENTRY(adam_bwd_tree),
    ENTRY(adam_unrolled_fwd_tree),
    ENTRY(adam_unrolled_bwd_tree),
    ENTRY(sgd_fwd),
    ENTRY(sgd_bwd),
    ENTRY(rmsprop_fwd),
    ENTRY(rmsprop_bwd),
    ENTRY(sgd_fwd_tree),
    ENTRY(sgd_bwd_tree),
    ENTRY(rmsprop_fwd_tree),
    ENTRY(rmsprop_bwd_tree),
    ENTRY(es_perturb),
    ENTRY(es_estimate),
    ENTRY(es_perturb_gaussian),
    ENTRY(es_estimate_gaussian),
    ENTRY(es_weights),
    OPERATOR(linattn_fwd),
    OPERATOR(linattn_bwd),
    OPERATOR(linattn_step),
    OPERATOR(qknorm_rope_fwd),
    OPERATOR(qknorm_rope_bwd),
    OPERATOR(qknorm_rope_bwd_bwd),
    OPERATOR(distill_fwd),
    OPERATOR(distill_bwd),
    OPERATOR(distill_fwd_bwd),
    OPERATOR(distill_bwd_bwd),
    OPERATOR(clip_norm_fwd),
    OPERATOR(clip_norm_bwd),
    OPERATOR(clip_norm_fwd_tree),
    OPERATOR(clip_norm_bwd_tree),
    OPERATOR(logprob_fwd),
    OPERATOR(logprob_bwd),
    OPERATOR(logprob_fwd_bwd),
    OPERATOR(logprob_bwd_bwd),
    OPERATOR(gscan_fwd),
    OPERATOR(gscan_bwd),
    OPERATOR(gscan_bwd_bwd),
    OPERATOR(gscan_step),
    {"leaf_pointers", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&leaf_pointers)), METH_FASTCALL, nullptr},
    {"leaf_shapes", &leaf_shapes, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
