// Python module _native: argument checks, allocation of results and the calls of the operators whose kernels are shorter than
// what ctypes and Python checks take (an AdamW step over 386 tensors 139 us, of which the library 10; a single token's
// quantisation 22 us, its kernel 6). It calls the C interface of include/defl.h and computes nothing; binding.py documents the arguments.
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAStream.h>
#include <c10/core/ScalarTypeToTypeMeta.h>
#include <map>
#include <mutex>
#include "../../include/defl.h"

namespace {

using at::ScalarType;
using at::Tensor;

defl_ctx* handle(PyObject* o) { return reinterpret_cast<defl_ctx*>(PyLong_AsVoidPtr(o)); }
bool is_none(PyObject* o) { return o == Py_None; }
const Tensor& tensor(PyObject* o, const char* what) {
  TORCH_CHECK_TYPE(THPVariable_Check(o), what, " must be a tensor");
  return THPVariable_Unpack(o);
}
void on_device(const Tensor& t, int device, const char* what) {
  TORCH_CHECK_VALUE(t.is_cuda() && t.get_device() == device, what, " must be on cuda:", device);
}
// a contiguous tensor of `count` elements of one type
void* scalar(PyObject* o, int device, ScalarType type, int64_t count, const char* what) {
  const Tensor& t = tensor(o, what);
  on_device(t, device, what);
  TORCH_CHECK_VALUE(t.scalar_type() == type && t.numel() == count && t.is_contiguous(), what, " must be a contiguous ", type, " tensor of ", count, " on cuda:", device);
  return t.data_ptr();
}
int code_of(ScalarType t) { return t == at::kFloat ? DEFL_F32 : t == at::kBFloat16 ? DEFL_BF16 : t == at::kHalf ? DEFL_F16 : -1; }
Tensor make(at::IntArrayRef shape, ScalarType type, int device) {
  return at::detail::empty_cuda(shape, type, c10::Device(c10::kCUDA, (c10::DeviceIndex)device), std::nullopt);
}
void use_stream(defl_ctx* c, int device) { defl_set_stream(c, c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream()); }

// Python's lock is given up where the library allocates and launches: a launch waits while its stream's queue is full, and what the stream waits for
// may be another thread of the program. Nothing of Python's is touched meanwhile. Setting the stream and the call belong together, so calls
// on one context take turns.
std::mutex& lock_of(defl_ctx* c) {
  static std::mutex all;
  static auto* each = new std::map<defl_ctx*, std::mutex>;   // (never taken apart: a later context at an old address has the old one's)
  static thread_local defl_ctx* last = nullptr;
  static thread_local std::mutex* lock = nullptr;
  if (!lock || last != c) {
    const std::lock_guard<std::mutex> one(all);
    lock = &(*each)[c];
    last = c;
  }
  return *lock;
}
struct Unlocked {
  PyThreadState* const state;
  std::unique_lock<std::mutex> turn;
  explicit Unlocked(defl_ctx* c) : state(PyEval_SaveThread()), turn(lock_of(c)) {}
  ~Unlocked() { turn.unlock(); PyEval_RestoreThread(state); }
};

// A tuple: another thread may change a list while this one is without Python's lock.
struct Sequence {
  PyObject* items;
  explicit Sequence(PyObject* o) : items(PySequence_Tuple(o)) { if (!items) throw python_error(); }
  ~Sequence() { Py_DECREF(items); }
  Py_ssize_t size() const { return PyTuple_GET_SIZE(items); }
  PyObject* operator[](Py_ssize_t i) const { return PyTuple_GET_ITEM(items, i); }
};
// address and type of gradient i after its checks; false for None
bool gradient(PyObject* o, Py_ssize_t i, int device, const void** x, int64_t* n, int* type) {
  if (is_none(o)) return false;
  TORCH_CHECK_TYPE(THPVariable_Check(o), "gradient ", i, " must be a tensor");
  const Tensor& t = THPVariable_Unpack(o);
  TORCH_CHECK_VALUE(t.device() == c10::Device(c10::kCUDA, (c10::DeviceIndex)device) && t.is_contiguous(), "gradient ", i, " must be a contiguous tensor on cuda:", device);
  *type = code_of(t.scalar_type());
  TORCH_CHECK_TYPE(*type == DEFL_F32 || *type == DEFL_BF16, "gradient ", i, " must be float32 or bfloat16");
  *x = t.const_data_ptr();
  *n = t.numel();
  return true;
}

[[noreturn]] __attribute__((noinline, cold)) void moved(const char* what, Py_ssize_t i) {
  TORCH_CHECK_VALUE(false, what, " ", i, " has other memory than when its AdamWGroup was made");
}

// Where the tensors were that an AdamWGroup's table points to beside the parameters, looked at again in every call: each tensor's storage, its place in
// it unless it is all of it (a view of that has the same memory), and each storage's address. (386 parameters have 772 moments, or 1544 tensors with
// scales. What a look costs is the lines of memory it touches, so those of Python's objects and most of those of the tensors are left out.)
struct Held {
  struct Item { const c10::TensorImpl* tensor; const c10::StorageImpl* storage; int64_t offset; };      // offset -1: all of its storage
  struct Place { const char* what; Py_ssize_t i; };
  std::vector<Item> items;
  std::vector<Place> places;                                 // of the items
  std::vector<std::pair<const c10::StorageImpl*, const void*>> memory;
  std::vector<size_t> first;                                 // the first item of each storage
  std::vector<Tensor> tensors;                               // keep what the pointers point to
  std::vector<c10::Storage> storages;

  void add(const Tensor& t, const void* p, const char* what, Py_ssize_t i, std::map<const c10::StorageImpl*, size_t>& known) {
    if (t.data_ptr() != p) moved(what, i);
    const c10::StorageImpl* s = t.storage().unsafeGetStorageImpl();
    if (known.emplace(s, memory.size()).second) {
      memory.emplace_back(s, s->data());
      first.push_back(items.size());
      storages.push_back(t.storage());
    }
    const bool all = t.storage_offset() == 0 && (size_t)t.numel() * t.element_size() == s->nbytes();
    items.push_back({t.unsafeGetTensorImpl(), s, all ? -1 : t.storage_offset()});
    places.push_back({what, i});
    tensors.push_back(t);
  }
  void check() const {
    for (size_t k = 0; k < items.size(); ++k) {
      const Item& x = items[k];
      if (x.tensor->unsafe_storage().unsafeGetStorageImpl() != x.storage || (x.offset >= 0 && x.tensor->storage_offset() != x.offset))
        moved(places[k].what, places[k].i);
    }
    for (size_t k = 0; k < memory.size(); ++k)
      if (memory[k].first->data() != memory[k].second) moved(places[first[k]].what, places[first[k]].i);
  }
};

// adamw_hold(table address, count, others) -> what adamw_step looks at. others: for each parameter that is not empty its moments, their scales in 8 bits, its
// copy if it has one
PyObject* adamw_hold(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK(nargs == 3, "adamw_hold takes 3 arguments");
  const defl_adamw_tensor* table = reinterpret_cast<const defl_adamw_tensor*>(PyLong_AsVoidPtr(a[0]));
  const Py_ssize_t count = PyLong_AsSsize_t(a[1]);
  if (PyErr_Occurred()) throw python_error();
  const Sequence others(a[2]);
  auto held = std::make_unique<Held>();
  std::map<const c10::StorageImpl*, size_t> known;
  Py_ssize_t at = 0;
  auto next = [&](const void* p, const char* what, Py_ssize_t i) {
    TORCH_CHECK_VALUE(at < others.size(), "tensors of the AdamWGroup are missing");
    held->add(tensor(others[at++], what), p, what, i, known);
  };
  for (Py_ssize_t i = 0; i < count; ++i) {
    const defl_adamw_tensor& t = table[i];
    if (t.n == 0) continue;
    next(t.m, "first moment", i);
    next(t.v, "second moment", i);
    if (t.state_bits == 8) {
      next(t.m_scale, "first moment's scales", i);
      next(t.v_scale, "second moment's scales", i);
    }
    if (t.copy) next(t.copy, "copy", i);
  }
  PyObject* made = PyCapsule_New(held.get(), "Held", [](PyObject* o) { delete static_cast<Held*>(PyCapsule_GetPointer(o, "Held")); });
  if (!made) throw python_error();
  held.release();
  return made;
  END_HANDLE_TH_ERRORS
}

// adamw_step(handle, device, table address, params, grads, lr, step, beta1, beta2, eps, weight_decay, grad_scale, stochastic, seed[, adamw_hold's]) -> code
PyObject* adamw_step(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK(nargs == 14 || nargs == 15, "adamw_step takes 14 or 15 arguments");
  defl_ctx* c = handle(a[0]);
  const int device = (int)PyLong_AsLong(a[1]);
  const defl_adamw_tensor* held = reinterpret_cast<const defl_adamw_tensor*>(PyLong_AsVoidPtr(a[2]));
  const Sequence params(a[3]), grads(a[4]);
  const Py_ssize_t count = params.size();
  TORCH_CHECK_VALUE(grads.size() == count, grads.size(), " gradients for ", count, " parameters");
  defl_adamw_opts o = {};
  if (THPVariable_Check(a[5])) o.lr_dev = (const float*)scalar(a[5], device, at::kFloat, 1, "lr"); else o.lr = PyFloat_AsDouble(a[5]);
  if (THPVariable_Check(a[6])) o.step_dev = (const int64_t*)scalar(a[6], device, at::kLong, 1, "step"); else o.step = PyLong_AsLongLong(a[6]);
  o.beta1 = PyFloat_AsDouble(a[7]); o.beta2 = PyFloat_AsDouble(a[8]); o.eps = PyFloat_AsDouble(a[9]); o.weight_decay = PyFloat_AsDouble(a[10]);
  if (!is_none(a[11])) o.grad_scale = (const float*)scalar(a[11], device, at::kFloat, 2, "grad_scale") + 1;
  o.stochastic = PyObject_IsTrue(a[12]);
  o.seed = PyLong_AsUnsignedLongLongMask(a[13]);
  if (PyErr_Occurred()) throw python_error();
  // (a copy for this call, with its gradients: the group's table is shared by all)
  std::vector<defl_adamw_tensor> table;
  table.reserve((size_t)count);
  if (nargs == 15) {
    const Held* rest = static_cast<const Held*>(PyCapsule_GetPointer(a[14], "Held"));
    if (!rest) throw python_error();
    rest->check();
  }
  for (Py_ssize_t i = 0; i < count; ++i) {
    table.push_back(held[i]);
    defl_adamw_tensor& t = table.back();
    const Tensor& p = tensor(params[i], "a parameter");
    if (p.const_data_ptr() != t.p || p.numel() != t.n) moved("parameter", i);
    int64_t n = 0;
    t.g = nullptr;
    if (!gradient(grads[i], i, device, &t.g, &n, &t.g_dtype)) continue;
    TORCH_CHECK_VALUE(n == t.n, "gradient ", i, " has ", n, " elements, its parameter ", t.n);
  }
  int rc;
  {
    const Unlocked unlocked(c);
    use_stream(c, device);
    rc = defl_adamw_step(c, table.data(), (int)count, &o);
  }
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// grad_norm(handle, device, grads, max_norm, out or None, step or None) -> out, or the error code
PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK(nargs == 6, "grad_norm takes 6 arguments");
  defl_ctx* c = handle(a[0]);
  const int device = (int)PyLong_AsLong(a[1]);
  const Sequence grads(a[2]);
  const float max_norm = (float)PyFloat_AsDouble(a[3]);
  int64_t* step = is_none(a[5]) ? nullptr : (int64_t*)scalar(a[5], device, at::kLong, 1, "step");
  if (PyErr_Occurred()) throw python_error();
  std::vector<defl_norm_tensor> table((size_t)grads.size());
  int count = 0;
  for (Py_ssize_t i = 0; i < grads.size(); ++i) {
    defl_norm_tensor& t = table[count];
    if (gradient(grads[i], i, device, &t.x, &t.n, &t.dtype)) ++count;
  }
  Tensor out;
  if (!is_none(a[4])) { scalar(a[4], device, at::kFloat, 2, "out"); out = THPVariable_Unpack(a[4]); }
  int rc;
  {
    const Unlocked unlocked(c);
    if (!out.defined()) out = make({2}, at::kFloat, device);
    const Tensor work = make({(int64_t)defl_grad_norm_work_bytes(count)}, at::kByte, device);
    use_stream(c, device);
    rc = defl_grad_norm(c, table.data(), count, max_norm, out.data_ptr<float>(), step, work.data_ptr());
  }
  return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

struct Shape { int64_t codes[3], scales[4]; };
Shape shape_of(int64_t b, int64_t rows, int64_t cols, int fmt) {
  const int64_t width = (cols + 31) / 32 * 32, per = fmt == DEFL_MXFP4 ? 128 : 64;
  return {{b, rows, width / 2}, {b, (rows + 127) / 128, (width + per - 1) / per, 512}};
}
int side(int64_t x) { return (int)(x > DEFL_MX4_MAX_SIDE ? DEFL_MX4_MAX_SIDE + 1 : x); }

int format_of(PyObject* o) {
  const int f = !PyUnicode_Check(o) ? -1 : PyUnicode_CompareWithASCIIString(o, "mxfp4") == 0 ? DEFL_MXFP4 : PyUnicode_CompareWithASCIIString(o, "nvfp4") == 0 ? DEFL_NVFP4 : -1;
  TORCH_CHECK_VALUE(f >= 0, "the format is mxfp4 or nvfp4");
  return f;
}

// A part of a buffer of bytes as a contiguous tensor.
Tensor part(const Tensor& buffer, int64_t offset, at::IntArrayRef shape, ScalarType type) {
  auto impl = c10::make_intrusive<at::TensorImpl>(c10::Storage(buffer.storage()), c10::DispatchKeySet(c10::DispatchKey::CUDA), c10::scalarTypeToTypeMeta(type));
  impl->set_storage_offset(offset / (int64_t)c10::elementSize(type));
  impl->set_sizes_contiguous(shape);
  return Tensor(std::move(impl));
}

// The tensors of a new Mx4, in one allocation.
struct Made {
  Tensor codes, scales, scale;
  defl_mx4 ref;
  Made(int64_t b, int64_t rows, int64_t cols, int fmt, int device) {
    const Shape s = shape_of(b, rows, cols, fmt);
    const int64_t at_scales = (b * rows * s.codes[2] + 511) / 512 * 512, at_scale = at_scales + b * s.scales[1] * s.scales[2] * 512;
    const Tensor all = make({at_scale + 4 * b}, at::kByte, device);
    codes = part(all, 0, s.codes, at::kByte);
    scales = part(all, at_scales, s.scales, at::kByte);
    if (fmt == DEFL_NVFP4) scale = part(all, at_scale, {b}, at::kFloat);
    ref = {codes.data_ptr(), scales.data_ptr(), scale.defined() ? scale.data_ptr<float>() : nullptr};
  }
  // as an instance of binding.Mx4, a named tuple
  PyObject* object(PyObject* type, PyObject* fmt, int64_t rows, int64_t cols) const {
    PyObject* s = scale.defined() ? THPVariable_Wrap(scale) : Py_NewRef(Py_None);
    PyObject* fields = Py_BuildValue("((NNNOLL))", THPVariable_Wrap(codes), THPVariable_Wrap(scales), s, fmt, (long long)rows, (long long)cols);
    if (!fields) throw python_error();
    PyObject* made = PyTuple_Type.tp_new(reinterpret_cast<PyTypeObject*>(type), fields, nullptr);
    Py_DECREF(fields);
    if (!made) throw python_error();
    return made;
  }
};

// mx4_quantize(handle, device, X, format, which: 1 blocks along cols, 2 along rows, 3 both, Mx4) -> an Mx4 or a pair, or the error code
PyObject* mx4_quantize(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK(nargs == 6, "mx4_quantize takes 6 arguments");
  TORCH_CHECK(PyType_Check(a[5]) && PyType_IsSubtype(reinterpret_cast<PyTypeObject*>(a[5]), &PyTuple_Type), "the last argument is a named tuple");
  defl_ctx* c = handle(a[0]);
  const int device = (int)PyLong_AsLong(a[1]), fmt = format_of(a[3]), which = (int)PyLong_AsLong(a[4]);
  if (PyErr_Occurred()) throw python_error();
  const Tensor& X = tensor(a[2], "X");
  TORCH_CHECK_VALUE(X.dim() == 3 && X.is_cuda() && X.get_device() == device && (X.scalar_type() == at::kBFloat16 || X.scalar_type() == at::kFloat),
                    "X must be a bfloat16 or float32 tensor [b, rows, cols] on cuda:", device);
  const int64_t b = X.size(0), m = X.size(1), n = X.size(2);
  int64_t rows = m, cols = n, sr = X.stride(1), sc = X.stride(2);
  if (b <= 0 || rows <= 0 || cols <= 0) return PyLong_FromLong(DEFL_ERR_ARG);
  if (b > 65535 || rows > DEFL_MX4_MAX_SIDE || cols > DEFL_MX4_MAX_SIDE) return PyLong_FromLong(DEFL_ERR_RANK);
  // the same matrices, seen from the other side
  const bool turned = cols > 1 && sc != 1;
  if (turned) {
    TORCH_CHECK_VALUE(rows == 1 || sr == 1, "one of X's last two dimensions must be contiguous");
    std::swap(rows, cols);
    sr = sc;
  }
  if (rows == 1) sr = cols;
  TORCH_CHECK_VALUE(sr >= cols, "X's rows overlap");
  std::optional<Made> by_rows, by_cols;
  int rc;
  {
    const Unlocked unlocked(c);
    if (which & 1) by_rows.emplace(b, m, n, fmt, device);
    if (which & 2) by_cols.emplace(b, n, m, fmt, device);
    const defl_mx4 *r = by_rows ? &by_rows->ref : nullptr, *t = by_cols ? &by_cols->ref : nullptr;
    if (turned) std::swap(r, t);
    Tensor work;
    if (fmt == DEFL_NVFP4 && rows * cols > DEFL_MX4_SCAN_MOST) work = make({(int64_t)defl_mx4_work_bytes((int)b)}, at::kByte, device);
    use_stream(c, device);
    rc = defl_mx4_quantize(c, X.data_ptr(), code_of(X.scalar_type()), (int)b, (int)rows, (int)cols, sr, X.stride(0), fmt, r, t,
                           work.defined() ? work.data_ptr() : nullptr);
  }
  if (rc) return PyLong_FromLong(rc);
  if (which == 3) {
    PyObject* first = by_rows->object(a[5], a[3], m, n);
    PyObject* second = by_cols->object(a[5], a[3], n, m);
    return Py_BuildValue("(NN)", first, second);
  }
  return which & 1 ? by_rows->object(a[5], a[3], m, n) : by_cols->object(a[5], a[3], n, m);
  END_HANDLE_TH_ERRORS
}

// an Mx4's tensors (codes, scales, scale) after their checks
defl_mx4 reference(PyObject* const* a, int fmt, int64_t rows, int64_t cols, int device, int64_t* batch, const char* what) {
  const Tensor &codes = tensor(a[0], what), &scales = tensor(a[1], what);
  TORCH_CHECK_VALUE(codes.dim() == 3 && scales.dim() == 4 && rows > 0 && cols > 0, what, " is not an Mx4 of its rows and columns");
  const Shape s = shape_of(codes.size(0), rows, cols, fmt);
  auto fine = [&](const Tensor& t, at::IntArrayRef shape) {
    return t.is_cuda() && t.get_device() == device && t.scalar_type() == at::kByte && t.sizes() == shape && t.is_contiguous();
  };
  TORCH_CHECK_VALUE(fine(codes, s.codes) && fine(scales, s.scales), what, " must hold contiguous uint8 tensors of shapes ", at::IntArrayRef(s.codes), " and ",
                    at::IntArrayRef(s.scales), " on cuda:", device);
  *batch = codes.size(0);
  defl_mx4 r = {codes.data_ptr(), scales.data_ptr(), nullptr};
  if (fmt == DEFL_NVFP4) {
    TORCH_CHECK_VALUE(!is_none(a[2]), what, " needs its matrices' scales");
    r.scale = (float*)scalar(a[2], device, at::kFloat, *batch, what);
  }
  return r;
}

// mx4_dequantize(handle, device, codes, scales, scale, format, rows, cols, type code) -> tensor, or the error code
PyObject* mx4_dequantize(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK(nargs == 9, "mx4_dequantize takes 9 arguments");
  defl_ctx* c = handle(a[0]);
  const int device = (int)PyLong_AsLong(a[1]), fmt = format_of(a[5]), type = (int)PyLong_AsLong(a[8]);
  const int64_t rows = PyLong_AsLongLong(a[6]), cols = PyLong_AsLongLong(a[7]);
  int64_t b = 0;
  if (PyErr_Occurred()) throw python_error();
  const defl_mx4 q = reference(a + 2, fmt, rows, cols, device, &b, "q");
  if (b > INT_MAX || (type != DEFL_BF16 && type != DEFL_F32)) return PyLong_FromLong(DEFL_ERR_ARG);
  Tensor out;
  int rc;
  {
    const Unlocked unlocked(c);
    out = make({b, rows, cols}, type == DEFL_BF16 ? at::kBFloat16 : at::kFloat, device);
    use_stream(c, device);
    rc = defl_mx4_dequantize(c, &q, (int)b, side(rows), side(cols), fmt, out.data_ptr(), type);
  }
  return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// mx4_gemm(handle, device, A: codes, scales, scale, B: the same, format, M, N, K, out or None, type code, alpha) -> out, or the error code
PyObject* mx4_gemm(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK(nargs == 15, "mx4_gemm takes 15 arguments");
  defl_ctx* c = handle(a[0]);
  const int device = (int)PyLong_AsLong(a[1]), fmt = format_of(a[8]);
  int type = (int)PyLong_AsLong(a[13]);
  const int64_t M = PyLong_AsLongLong(a[9]), N = PyLong_AsLongLong(a[10]), K = PyLong_AsLongLong(a[11]);
  const double alpha = PyFloat_AsDouble(a[14]);
  if (PyErr_Occurred()) throw python_error();
  int64_t b = 0, bb = 0;
  const defl_mx4 A = reference(a + 2, fmt, M, K, device, &b, "A"), B = reference(a + 5, fmt, N, K, device, &bb, "B");
  TORCH_CHECK_VALUE(bb == 1 || bb == b, "A and B must agree in format, columns and batch");
  Tensor out;
  int64_t ld = N;
  if (is_none(a[12])) {
    if (type != DEFL_BF16 && type != DEFL_F32) return PyLong_FromLong(DEFL_ERR_ARG);
  } else {
    out = tensor(a[12], "out");
    const int64_t want[3] = {b, M, N};
    TORCH_CHECK_VALUE(out.is_cuda() && out.get_device() == device && out.sizes() == at::IntArrayRef(want) && (N == 1 || out.stride(2) == 1),
                      "out must be [b, M, N] on cuda:", device, " with contiguous rows");
    type = code_of(out.scalar_type());
    if (M > 1) ld = out.stride(1);
  }
  if (b > 65535) return PyLong_FromLong(DEFL_ERR_RANK);
  int rc;
  {
    const Unlocked unlocked(c);
    if (!out.defined()) out = make({b, M, N}, type == DEFL_BF16 ? at::kBFloat16 : at::kFloat, device);
    Tensor work;
    const size_t room = defl_mx4_gemm_work_bytes(c, (int)b, side(M), side(N), side(K), type);
    if (room) work = make({(int64_t)room}, at::kByte, device);
    use_stream(c, device);
    rc = defl_mx4_gemm(c, &A, &B, (int)b, side(M), side(N), side(K), bb == 1, fmt, (float)alpha, out.data_ptr(), ld, out.stride(0), type,
                       room ? work.data_ptr() : nullptr);
  }
  return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"adamw_hold", (PyCFunction)(void (*)(void))adamw_hold, METH_FASTCALL, nullptr},
                         {"adamw_step", (PyCFunction)(void (*)(void))adamw_step, METH_FASTCALL, nullptr},
                         {"grad_norm", (PyCFunction)(void (*)(void))grad_norm, METH_FASTCALL, nullptr},
                         {"mx4_quantize", (PyCFunction)(void (*)(void))mx4_quantize, METH_FASTCALL, nullptr},
                         {"mx4_dequantize", (PyCFunction)(void (*)(void))mx4_dequantize, METH_FASTCALL, nullptr},
                         {"mx4_gemm", (PyCFunction)(void (*)(void))mx4_gemm, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }
