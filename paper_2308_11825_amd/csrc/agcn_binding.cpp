// The Python functions of the routed layer's operators (layer norm, groups, products of
// 8-bit integers): checks of their tensors, allocation of their results on the current
// stream, and the C call. Compiled, because a call on a few rows takes as long as this
// takes: layer_norm of one row with residual and statistics 5.8 us a call, 11.5 us as Python code
// with ctypes, of which the launch is 3.2.
//
// The functions take positional arguments only; paper_2308_11825_amd/__init__.py documents
// them and passes the library's addresses to init().
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <stdexcept>
#include <string>
#include <tuple>

#include "../../include/agcn.h"

namespace {

using at::ScalarType;
using at::Tensor;

struct Library {
  decltype(&agcn_layer_norm) layer_norm;
  decltype(&agcn_layer_norm_workspace_size) layer_norm_workspace_size;
  decltype(&agcn_layer_norm_backward) layer_norm_backward;
  decltype(&agcn_sort_groups_workspace_size) sort_groups_workspace_size;
  decltype(&agcn_sort_groups) sort_groups;
  decltype(&agcn_dispatch) dispatch;
  decltype(&agcn_combine) combine;
  decltype(&agcn_combine_backward) combine_backward;
  decltype(&agcn_quantize_rows_int) quantize_rows_int;
  decltype(&agcn_int_linear) int_linear;
  decltype(&agcn_grouped_int_linear) grouped_int_linear;
  decltype(&agcn_last_error) last_error;
} lib;
PyObject *agcn_error = nullptr, *memory_error = nullptr;  // the package's, and torch's where its allocator fails

// A Python exception to raise.
struct Refused {
  PyObject* type;
  std::string what;
};
[[noreturn]] void type_error(const std::string& what) { throw Refused{PyExc_TypeError, what}; }
[[noreturn]] void value_error(const std::string& what) { throw Refused{PyExc_ValueError, what}; }
struct Failed {
  int status;
};
// A call of the library, with other Python threads free to run.
template <class F, class... A>
void call(F f, A... args) {
  PyThreadState* state = PyEval_SaveThread();
  const int status = f(args...);
  PyEval_RestoreThread(state);
  if (status != AGCN_OK) throw Failed{status};
}

std::string text(at::IntArrayRef shape) {
  std::string s = "(";
  for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
  return s + (shape.size() == 1 ? ",)" : ")");
}

const Tensor& tensor(const std::string& name, PyObject* o, at::Device device) {
  if (!THPVariable_Check(o) || THPVariable_Unpack(o).device() != device)
    type_error(name + " must be a tensor on " + device.str());
  const Tensor& t = THPVariable_Unpack(o);
  // The memory of such a view is not its values.
  if (t.is_conj()) type_error(name + " must not be a lazily conjugated view: resolve_conj() writes it out");
  if (t.is_neg()) type_error(name + " must not be a lazily negated view: resolve_neg() writes it out");
  return t;
}
// The tensor that sets a call's sizes and type; matrix() checks the rest of it.
const Tensor& first(const std::string& name, PyObject* o, int64_t dims, bool weight = false) {
  if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda()) type_error(name + " must be a CUDA tensor");
  const Tensor& t = THPVariable_Unpack(o);
  if (t.dim() != dims) value_error(name + " must have " + std::to_string(dims) + " dimensions");
  for (int64_t i = weight ? 0 : dims - 1; i < dims; ++i)
    if (t.size(i) > INT_MAX)
      value_error(name + " must have at most 2^31 - 1 " + (weight ? "rows, columns and groups" : "columns"));
  return t;
}
void same(const std::string& name, const Tensor& t, at::IntArrayRef shape, ScalarType dtype) {
  if (t.scalar_type() != dtype) type_error(name + " must have dtype " + c10::toString(dtype));
  if (t.sizes() != shape) value_error(name + " must have shape " + text(shape));
}
// A matrix (or stacked ones) with unit column stride, and its row stride.
struct Matrix {
  const Tensor* t;
  int64_t ld;
  void* data() const { return t->data_ptr(); }
};
Matrix matrix(const std::string& name, PyObject* o, at::Device device, at::IntArrayRef shape, ScalarType dtype) {
  const Tensor& t = tensor(name, o, device);
  same(name, t, shape, dtype);
  const int64_t rows = shape[shape.size() - 2], columns = shape.back();
  if (columns > 1 && t.numel() > 0 && t.stride(-1) != 1)
    value_error(name + " must have unit column stride, as its contiguous() has");
  if (rows > 1 && t.numel() > 0 && t.stride(-2) < columns)
    value_error(name + " must have rows that do not overlap, as its contiguous() has");
  // Any value >= a row is valid for 0 or 1 rows.
  return {&t, rows > 1 && t.numel() > 0 ? t.stride(-2) : std::max(columns, t.stride(-2))};
}
const Tensor& vector(const std::string& name, PyObject* o, at::Device device, at::IntArrayRef shape, ScalarType dtype) {
  const Tensor& t = tensor(name, o, device);
  same(name, t, shape, dtype);
  if (shape.back() > 1 && t.stride(-1) != 1) value_error(name + " must be contiguous");
  return t;
}
bool given(PyObject* o) { return o != Py_None; }

int32_t type_code(const std::string& name, ScalarType t) {
  if (t == ScalarType::Float) return AGCN_FLOAT;
  if (t == ScalarType::BFloat16) return AGCN_BFLOAT;
  if (t == ScalarType::Half) return AGCN_HALF;
  type_error(name + " must have dtype float32, bfloat16 or float16");
}
// The code of a norm's parameter, f values of the rows' type or float32.
int32_t parameter(const std::string& name, PyObject* o, at::Device device, int64_t f, ScalarType rows) {
  const Tensor& t = tensor(name, o, device);
  if (t.scalar_type() != rows && t.scalar_type() != ScalarType::Float)
    type_error(name + " must be float32 or of X's type");
  vector(name, o, device, {f}, t.scalar_type());
  return type_code(name, t.scalar_type());
}

Tensor fresh(const Tensor& like, at::IntArrayRef shape, ScalarType dtype) {
  at::AutoDispatchBelowAutograd below;
  return at::empty(shape, like.options().dtype(dtype).requires_grad(false));
}
// Rows of one byte a value that start on 16 bytes, and on 128 (the lines of memory) where that
// adds an eighth at most.
Tensor fresh_rows(const Tensor& like, int64_t rows, int64_t k, ScalarType dtype) {
  int64_t ld = (k + 127) / 128 * 128;
  if (ld > k + k / 8) ld = (k + 15) / 16 * 16;
  at::AutoDispatchBelowAutograd below;
  return at::empty_strided({rows, k}, {ld, 1}, like.options().dtype(dtype).requires_grad(false));
}
// The caller's result, checked, or a new one.
struct Result {
  Tensor t;
  int64_t ld;
};
Result result(const std::string& name, PyObject* o, const Tensor& like, at::IntArrayRef shape, ScalarType dtype) {
  if (!given(o)) return {fresh(like, shape, dtype), shape.back()};
  const Matrix m = matrix(name, o, like.device(), shape, dtype);
  return {*m.t, m.ld};
}
std::pair<PyObject*, PyObject*> pair(PyObject* o) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 2) type_error("out must be a pair of tensors");
  return {PyTuple_GET_ITEM(o, 0), PyTuple_GET_ITEM(o, 1)};
}

// The device of the call made current, and its current stream.
class On {
 public:
  explicit On(const Tensor& t) : before_(c10::hip::current_device()), index_(t.device().index()) {
    if (before_ != index_) c10::hip::set_device(index_);
    stream = static_cast<void*>(c10::hip::getCurrentHIPStream(index_).stream());
  }
  ~On() {
    if (before_ != index_) c10::hip::set_device(before_);
  }
  void* stream;

 private:
  c10::DeviceIndex before_, index_;
};

PyObject* wrap(const Tensor& t) { return THPVariable_Wrap(t); }
template <class... T>
PyObject* tuple(const T&... t) {
  PyObject* items[] = {t.defined() ? wrap(t) : (Py_INCREF(Py_None), Py_None)...};
  PyObject* p = PyTuple_New(sizeof...(t));
  for (size_t i = 0; i < sizeof...(t); ++i) {
    if (items[i] == nullptr || p == nullptr) {
      for (size_t j = i; j < sizeof...(t); ++j) Py_XDECREF(items[j]);
      Py_XDECREF(p);
      return nullptr;
    }
    PyTuple_SET_ITEM(p, i, items[i]);
  }
  return p;
}

PyObject* layer_norm(PyObject* const* a) {
  PyObject *weight = a[1], *bias = a[2], *residual = a[3], *hidden = a[6];
  const Tensor& x = first("X", a[0], 2);
  const at::Device device = x.device();
  const auto shape = x.sizes();
  const ScalarType dtype = x.scalar_type();
  const int64_t n = shape[0], f = shape[1];
  const int32_t code = type_code("X", dtype);
  const Matrix mx = matrix("X", a[0], device, shape, dtype);
  const int32_t p_code = parameter("weight", weight, device, f, dtype);
  const Tensor& g = THPVariable_Unpack(weight);
  const void* b = given(bias) ? vector("bias", bias, device, {f}, g.scalar_type()).data_ptr() : nullptr;
  const double eps = PyFloat_AsDouble(a[4]);
  if (eps == -1.0 && PyErr_Occurred()) return nullptr;
  const int stats = PyObject_IsTrue(a[5]);
  if (stats < 0) return nullptr;
  if (stats && f == 0) value_error("rows of no columns have no statistics");
  On on(x);
  Matrix r{nullptr, 0};
  Result h{Tensor(), 0};
  if (given(residual)) {
    r = matrix("residual", residual, device, shape, dtype);
    h = result("hidden", hidden, x, shape, dtype);
  } else if (given(hidden)) {
    value_error("hidden needs a residual: without one h is X");
  }
  const Result y = result("out", a[7], x, shape, dtype);
  const Tensor s = stats ? fresh(x, {n, 2}, ScalarType::Float) : Tensor();
  call(lib.layer_norm, n, (int32_t)f, code, mx.data(), mx.ld, r.t ? r.data() : nullptr, r.ld,
                       h.t.defined() ? h.t.data_ptr() : nullptr, h.ld, g.data_ptr(), b, p_code, (float)eps,
                       y.t.data_ptr(), y.ld, stats ? s.data_ptr<float>() : nullptr, 2, on.stream);
  if (h.t.defined()) return stats ? tuple(y.t, h.t, s) : tuple(y.t, h.t);
  return stats ? tuple(y.t, s) : wrap(y.t);
}

PyObject* layer_norm_backward(PyObject* const* a) {
  const Tensor& dy = first("grad", a[0], 2);
  const at::Device device = dy.device();
  const auto shape = dy.sizes();
  const ScalarType dtype = dy.scalar_type();
  const int64_t n = shape[0], f = shape[1];
  const int32_t code = type_code("grad", dtype);
  const Matrix my = matrix("grad", a[0], device, shape, dtype), h = matrix("H", a[1], device, shape, dtype);
  const Matrix stats = matrix("stats", a[2], device, {n, 2}, ScalarType::Float);
  const int32_t p_code = parameter("weight", a[3], device, f, dtype);
  const Tensor& g = THPVariable_Unpack(a[3]);
  const int bias = PyObject_IsTrue(a[4]);
  if (bias < 0) return nullptr;
  Matrix d{nullptr, 0};
  if (given(a[5])) d = matrix("grad_hidden", a[5], device, shape, dtype);
  On on(dy);
  const Result dx = result("out", a[6], dy, shape, dtype);
  const Tensor dg = fresh(dy, {f}, g.scalar_type()), db = bias ? fresh(dy, {f}, g.scalar_type()) : Tensor();
  size_t bytes = 0;
  call(lib.layer_norm_workspace_size, n, (int32_t)f, code, &bytes);
  const Tensor ws = bytes ? fresh(dy, {(int64_t)bytes / 4}, ScalarType::Float) : Tensor();
  call(lib.layer_norm_backward, n, (int32_t)f, code, my.data(), my.ld, h.data(), h.ld, d.t ? d.data() : nullptr, d.ld,
                                stats.t->data_ptr<float>(), stats.ld, g.data_ptr(), p_code, dx.t.data_ptr(), dx.ld,
                                dg.data_ptr(), bias ? db.data_ptr() : nullptr, bytes ? ws.data_ptr() : nullptr,
                                on.stream);
  return tuple(dx.t, dg, db);
}

PyObject* sort_groups(PyObject* const* a) {
  const Tensor& ids = first("ids", a[0], 2);
  const at::Device device = ids.device();
  const ScalarType dtype = ids.scalar_type();
  if (dtype != ScalarType::Int && dtype != ScalarType::Long) type_error("ids must have dtype int32 or int64");
  const int64_t n = ids.size(0), k = ids.size(1), groups = PyLong_AsLongLong(a[1]);
  if (groups == -1 && PyErr_Occurred()) return nullptr;
  if (groups < 0 || groups > INT_MAX) value_error("groups must be from 0 to 2^31 - 1");
  const Matrix m = matrix("ids", a[0], device, {n, k}, dtype);
  size_t bytes = 0;
  call(lib.sort_groups_workspace_size, n, (int32_t)k, (int32_t)groups, &bytes);
  On on(ids);
  Tensor offsets;
  Result place;
  if (given(a[2])) {
    const auto out = pair(a[2]);
    offsets = vector("out[0]", out.first, device, {groups + 1}, ScalarType::Int);
    place = result("out[1]", out.second, ids, {n, k}, ScalarType::Int);
  } else {
    offsets = fresh(ids, {groups + 1}, ScalarType::Int);
    place = {fresh(ids, {n, k}, ScalarType::Int), k};
  }
  const Tensor ws = bytes ? fresh(ids, {(int64_t)bytes / 4}, ScalarType::Int) : Tensor();
  call(lib.sort_groups, n, (int32_t)k, (int32_t)groups, m.data(), dtype == ScalarType::Int ? 4 : 8, m.ld,
                        offsets.data_ptr<int32_t>(), place.t.data_ptr<int32_t>(), place.ld,
                        bytes ? ws.data_ptr() : nullptr, on.stream);
  return tuple(offsets, place.t);
}

PyObject* dispatch(PyObject* const* a) {
  const Tensor& x = first("X", a[0], 2);
  const at::Device device = x.device();
  const ScalarType dtype = x.scalar_type();
  const int64_t n = x.size(0), f = x.size(1), size = x.element_size();
  const Tensor& places = tensor("place", a[1], device);
  if (places.dim() != 2) value_error("place must have 2 dimensions");
  const int64_t k = places.size(1);
  if (k > INT_MAX) value_error("place must have at most 2^31 - 1 columns");
  const Matrix mx = matrix("X", a[0], device, x.sizes(), dtype);
  const Matrix p = matrix("place", a[1], device, {n, k}, ScalarType::Int);
  On on(x);
  Result y;
  if (!given(a[2]) && size == 1) {
    y.t = fresh_rows(x, n * k, f, dtype);
    y.ld = y.t.stride(0);
  } else {
    y = result("out", a[2], x, {n * k, f}, dtype);
  }
  call(lib.dispatch, n, (int32_t)k, f * size, mx.data(), mx.ld * size, p.t->data_ptr<int32_t>(), p.ld, y.t.data_ptr(),
                     y.ld * size, on.stream);
  return wrap(y.t);
}

// The places of `rows` rows.
Matrix places(PyObject* o, at::Device device, int64_t rows) {
  const Tensor& t = tensor("place", o, device);
  if (t.dim() != 2) value_error("place must have 2 dimensions");
  if (t.size(0) * t.size(1) != rows) value_error("place must name as many rows as there are");
  return matrix("place", o, device, t.sizes(), ScalarType::Int);
}

PyObject* combine(PyObject* const* a) {
  const Tensor& r = first("R", a[0], 2);
  const at::Device device = r.device();
  const ScalarType dtype = r.scalar_type();
  const int32_t code = type_code("R", dtype);
  const int64_t rows = r.size(0), f = r.size(1);
  const Matrix p = places(a[1], device, rows), mr = matrix("R", a[0], device, r.sizes(), dtype);
  const int64_t n = p.t->size(0), k = p.t->size(1);
  Matrix w{nullptr, k};
  if (given(a[2])) w = matrix("weights", a[2], device, {n, k}, ScalarType::Float);
  On on(r);
  const Result y = result("out", a[3], r, {n, f}, dtype);
  call(lib.combine, n, (int32_t)k, (int32_t)f, code, mr.data(), mr.ld, p.t->data_ptr<int32_t>(), p.ld,
                    w.t ? w.t->data_ptr<float>() : nullptr, w.ld, y.t.data_ptr(), y.ld, on.stream);
  return wrap(y.t);
}

PyObject* combine_backward(PyObject* const* a) {
  const Tensor& r = first("R", a[1], 2);
  const at::Device device = r.device();
  const ScalarType dtype = r.scalar_type();
  const int32_t code = type_code("R", dtype);
  const int64_t rows = r.size(0), f = r.size(1);
  const Matrix p = places(a[2], device, rows), mr = matrix("R", a[1], device, r.sizes(), dtype);
  const int64_t n = p.t->size(0), k = p.t->size(1);
  const Matrix g = matrix("grad", a[0], device, {n, f}, dtype);
  const Matrix w = matrix("weights", a[3], device, {n, k}, ScalarType::Float);
  On on(r);
  const Result dr = result("out", a[4], r, r.sizes(), dtype);
  const Tensor dw = fresh(r, {n, k}, ScalarType::Float);
  call(lib.combine_backward, n, (int32_t)k, (int32_t)f, code, g.data(), g.ld, mr.data(), mr.ld,
                             p.t->data_ptr<int32_t>(), p.ld, w.t->data_ptr<float>(), w.ld, dr.t.data_ptr(), dr.ld,
                             dw.data_ptr<float>(), k, on.stream);
  return tuple(dr.t, dw);
}

PyObject* quantize_int(PyObject* const* a) {
  const Tensor& x = first("X", a[0], 2);
  const at::Device device = x.device();
  const ScalarType dtype = x.scalar_type();
  const int64_t n = x.size(0), f = x.size(1);
  const int32_t code = type_code("X", dtype);
  const Matrix m = matrix("X", a[0], device, x.sizes(), dtype);
  On on(x);
  Result q;
  Tensor s;
  if (given(a[1])) {
    const auto out = pair(a[1]);
    q = result("out[0]", out.first, x, {n, f}, ScalarType::Char);
    s = vector("out[1]", out.second, device, {n}, ScalarType::Float);
  } else {
    q.t = fresh_rows(x, n, f, ScalarType::Char);
    q.ld = q.t.stride(0);
    s = fresh(x, {n}, ScalarType::Float);
  }
  call(lib.quantize_rows_int, n, (int32_t)f, code, m.data(), m.ld, q.t.data_ptr(), q.ld, s.data_ptr<float>(),
                              on.stream);
  return tuple(q.t, s);
}

// Q, S, WQ, WS, offsets or None, dtype or None, epilogue, out or None.
PyObject* int_product(PyObject* const* a) {
  const bool grouped = given(a[4]);
  const Tensor& q = first("Q", a[0], 2);
  const Tensor& wq = first("WQ", a[2], grouped ? 3 : 2, true);
  const at::Device device = q.device();
  const int64_t n = q.size(0), fin = q.size(1), fout = wq.size(-2), groups = grouped ? wq.size(0) : 1;
  const Matrix mq = matrix("Q", a[0], device, q.sizes(), ScalarType::Char);
  const Tensor& s = vector("S", a[1], device, {n}, ScalarType::Float);
  const int64_t w_shape[] = {groups, fout, fin};
  const at::IntArrayRef all(w_shape, 3);
  const Matrix mw = matrix("WQ", a[2], device, grouped ? all : all.slice(1), ScalarType::Char);
  const Tensor& ws = vector("WS", a[3], device, grouped ? all.slice(0, 2) : all.slice(1, 1), ScalarType::Float);
  const long epilogue = PyLong_AsLong(a[6]);
  if (epilogue == -1 && PyErr_Occurred()) return nullptr;
  ScalarType dtype = ScalarType::Float;
  if (given(a[5])) {
    if (!THPDtype_Check(a[5])) type_error("dtype must be a torch.dtype");
    dtype = reinterpret_cast<THPDtype*>(a[5])->scalar_type;
  } else if (given(a[7])) {
    dtype = tensor("out", a[7], device).scalar_type();
  }
  const int32_t code = type_code("the result", dtype);
  const int32_t* offsets =
      grouped ? vector("offsets", a[4], device, {groups + 1}, ScalarType::Int).data_ptr<int32_t>() : nullptr;
  On on(q);
  const Result y = result("out", a[7], q, {n, fout}, dtype);
  if (grouped)
    call(lib.grouped_int_linear, n, (int32_t)fin, (int32_t)fout, (int32_t)groups, mq.data(), mq.ld,
                                 s.data_ptr<float>(), mw.data(), mw.ld, wq.stride(0), ws.data_ptr<float>(),
                                 ws.stride(0), offsets, code, y.t.data_ptr(), y.ld, on.stream, (int32_t)epilogue);
  else
    call(lib.int_linear, n, (int32_t)fin, (int32_t)fout, mq.data(), mq.ld, s.data_ptr<float>(), mw.data(), mw.ld,
                         ws.data_ptr<float>(), code, y.t.data_ptr(), y.ld, on.stream, (int32_t)epilogue);
  return wrap(y.t);
}

// No C++ exception leaves for Python's C code.
template <PyObject* (*F)(PyObject* const*), int ARGS>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (count != ARGS) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Refused& r) {
    PyErr_SetString(r.type, r.what.c_str());
  } catch (const Failed& r) {
    if (PyObject* e = PyObject_CallFunction(agcn_error, "is", r.status, lib.last_error())) {
      PyErr_SetObject(agcn_error, e);
      Py_DECREF(e);
    }
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(memory_error, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

void keep(PyObject*& to, PyObject* o) {
  Py_INCREF(o);
  Py_XDECREF(to);
  to = o;
}
// init(AgcnError, torch.OutOfMemoryError, addresses): the addresses of Library's functions in its order.
PyObject* init(PyObject*, PyObject* args) {
  PyObject *error, *memory, *list;
  if (!PyArg_ParseTuple(args, "OOO!", &error, &memory, &PyList_Type, &list)) return nullptr;
  constexpr Py_ssize_t kCount = sizeof(Library) / sizeof(void*);
  if (PyList_GET_SIZE(list) != kCount) {
    PyErr_SetString(PyExc_ValueError, "wrong number of addresses");
    return nullptr;
  }
  void* to[kCount];
  for (Py_ssize_t i = 0; i < kCount; ++i) {
    to[i] = PyLong_AsVoidPtr(PyList_GET_ITEM(list, i));
    if (to[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is 0");
      return nullptr;
    }
  }
  memcpy(static_cast<void*>(&lib), to, sizeof(lib));
  keep(agcn_error, error);
  keep(memory_error, memory);
  Py_RETURN_NONE;
}

#define ENTRY(name, args) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<name, args>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"init", &init, METH_VARARGS, nullptr},
                         ENTRY(layer_norm, 8),
                         ENTRY(layer_norm_backward, 7),
                         ENTRY(sort_groups, 3),
                         ENTRY(dispatch, 3),
                         ENTRY(combine, 4),
                         ENTRY(combine_backward, 5),
                         ENTRY(quantize_int, 2),
                         ENTRY(int_product, 8),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
