// Python module _ops: torch tensors to the calls of prsgd_ops.h.  It checks types, devices and strides, allocates what is not given, and
// passes addresses and the current stream on; nothing is computed here.  The same marshalling in Python took 10 us for a call on
// one row, three times the kernel and twice the launch.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <string>

#include "prsgd_ops.h"

namespace {

using at::Tensor;

struct Refused : std::exception {                          // becomes a ValueError
  std::string text;
  explicit Refused(std::string t) : text(std::move(t)) {}
  const char* what() const noexcept override { return text.c_str(); }
};
struct Raised {};                                          // the Python error is set

PyObject* g_check = nullptr;                               // raises the package's error for a status

void require(bool ok, const char* text) {
  if (!ok) throw Refused(text);
}
void finish(int status) {
  if (status == PRSGD_OK) return;
  PyObject* r = PyObject_CallFunction(g_check, "i", status);
  Py_XDECREF(r);
  throw Raised{};
}

const Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) throw Refused(std::string(what) + " must be a tensor");
  return THPVariable_Unpack(o);
}
// A tensor that a call computes with or writes: no call records anything for autograd
const Tensor& operand(PyObject* o, const char* what) {
  const Tensor& t = tensor(o, what);
  if (t.requires_grad() && c10::GradMode::is_enabled())
    throw Refused(std::string(what) + " requires grad, and the operators record nothing: call them under torch.no_grad() or in a torch.autograd.Function");
  return t;
}
// ... and one that it has written: autograd's check of what it saved has to see that
void written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return v;
}
int32_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  require(v >= INT32_MIN && v <= INT32_MAX, "number out of range");
  return (int32_t)v;
}
int32_t size32(int64_t n) {
  require(n <= INT32_MAX, "size out of range");
  return (int32_t)n;
}
int32_t operand_type(const Tensor& t, const char* text) {
  require(t.is_cuda() && (t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16), text);
  return t.scalar_type() == at::kFloat ? PRSGD_F32 : PRSGD_BF16;
}

// The caching allocator without the dispatcher in front of it, which took as long again for each of a call's tensors
Tensor device_empty(at::IntArrayRef sizes, at::ScalarType type, const Tensor& like) {
  return Tensor(at::detail::empty_cuda(sizes, type, like.device(), std::nullopt));
}

// The tensors' device made current for the call, and its current stream.
struct OnDevice {
  c10::DeviceIndex before;
  c10::DeviceIndex here;
  explicit OnDevice(const Tensor& t) : before(-1), here(t.device().index()) { before = c10::hip::ExchangeDevice(here); }
  ~OnDevice() { c10::hip::MaybeExchangeDevice(before); }
  void* stream() const { return c10::hip::getCurrentHIPStream(here).stream(); }
};

// ---- rows ------------------------------------------------------------------------------------

struct Rows { void* at; int64_t distance; };
Rows rows_of(const Tensor& t, const Tensor& like, at::ScalarType type, const char* name) {
  const bool same = &t == &like || (t.device() == like.device() && t.sizes() == like.sizes());
  if (!t.is_cuda() || t.scalar_type() != type || !same) throw Refused(std::string(name) + " must have the device and shape of the rows, and its type");
  if (t.size(1) > 1 && t.stride(1) != 1) throw Refused(std::string("rows of ") + name + " must be contiguous");
  const int64_t distance = t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1));
  return {t.data_ptr(), distance};
}
struct NormCall {
  prsgd_norm_config cfg;
  const float* w;
  int64_t w_row;
};
NormCall norm_call(const Tensor& x, const Tensor& w, float eps) {
  NormCall c{};
  require(x.dim() == 2, "rows must be a [rows][width] tensor");
  c.cfg.dtype = operand_type(x, "rows must be a device tensor of float32 or bfloat16");
  require(w.scalar_type() == at::kFloat && w.device() == x.device() && (w.dim() == 1 || w.dim() == 2) && w.size(-1) == x.size(1) &&
              (w.size(-1) <= 1 || w.stride(-1) == 1),
          "weights must be float32 on the rows' device, [width] or [workers][width], their rows contiguous");
  const int64_t workers = w.dim() == 2 ? w.size(0) : 1;
  require(workers > 0 && x.size(0) % workers == 0, "every worker must have the same number of rows");
  c.cfg.workers = size32(workers);
  c.cfg.rows_per_worker = x.size(0) / workers;
  c.cfg.width = size32(x.size(1));
  c.cfg.eps = eps;
  c.w = static_cast<const float*>(w.data_ptr());
  c.w_row = w.dim() == 2 && workers > 1 ? w.stride(0) : 0;
  return c;
}
Tensor row_vector(PyObject* o, const Tensor& x, const char* name) {
  if (o == Py_None) return device_empty({x.size(0)}, at::kFloat, x);
  const Tensor& t = operand(o, name);
  if (t.scalar_type() != at::kFloat || t.device() != x.device() || t.dim() != 1 || t.size(0) != x.size(0) || !t.is_contiguous())
    throw Refused(std::string(name) + " must be contiguous float32, one value a row");
  return t;
}
Tensor given_or_empty(PyObject* o, const Tensor& like, at::ScalarType type, const char* name) {
  return o == Py_None ? device_empty(like.sizes(), type, like) : operand(o, name);
}
Tensor workspace(PyObject* o, size_t bytes, const Tensor& like) {
  if (o == Py_None) return device_empty({(int64_t)bytes}, at::kByte, like);
  const Tensor& t = operand(o, "workspace");
  if (t.device() != like.device() || t.nbytes() < bytes || !t.is_contiguous()) throw Refused("the workspace must have " + std::to_string(bytes) + " bytes on the tensors' device");
  return t;
}

// x, w, residual, eps, out, sum_out, stat, in 8 bits -> out, s (or None), stat
PyObject* rms_norm(PyObject* const* a) {
  const Tensor& x = operand(a[0], "x");
  const NormCall c = norm_call(x, operand(a[1], "w"), (float)number(a[3]));
  const bool fp8 = a[7] == Py_True;
  const at::ScalarType type = x.scalar_type(), out_type = fp8 ? at::kFloat8_e4m3fn : type;
  OnDevice on(x);
  const Rows xr = rows_of(x, x, type, "x");
  Rows rr{nullptr, 0}, sr{nullptr, 0};
  Tensor sum = x;
  if (a[2] != Py_None) rr = rows_of(operand(a[2], "residual"), x, type, "residual");
  if (a[2] != Py_None || a[5] != Py_None) {
    sum = given_or_empty(a[5], x, type, "sum_out");
    sr = rows_of(sum, x, type, "sum_out");
  }
  Tensor out = given_or_empty(a[4], x, out_type, "out"), stat = row_vector(a[6], x, fp8 ? "scales" : "rstd");
  const Rows yr = rows_of(out, x, out_type, "out");
  float* st = static_cast<float*>(stat.data_ptr());
  finish(fp8 ? prsgd_rms_norm_fp8(&c.cfg, xr.at, xr.distance, rr.at, rr.distance, c.w, c.w_row, sr.at, sr.distance,
                                  static_cast<uint8_t*>(yr.at), yr.distance, st, on.stream())
             : prsgd_rms_norm(&c.cfg, xr.at, xr.distance, rr.at, rr.distance, c.w, c.w_row, sr.at, sr.distance, yr.at, yr.distance, st,
                              on.stream()));
  written(out);
  written(stat);
  if (sr.at != nullptr) written(sum);
  // rows that were their own sum are gone once the result has their place
  const bool gone = a[2] == Py_None && a[5] == Py_None && x.numel() > 0 && yr.at == xr.at;
  if (gone) Py_INCREF(Py_None);
  return Py_BuildValue("(NNN)", THPVariable_Wrap(out), gone ? Py_None : THPVariable_Wrap(sum), THPVariable_Wrap(stat));
}

size_t back_bytes(const NormCall& c) {
  const size_t n = prsgd_rms_norm_backward_workspace_bytes(&c.cfg);
  if (n == 0) finish(PRSGD_EINVAL);
  return n;
}
// x, w -> bytes
PyObject* rms_norm_backward_bytes(PyObject* const* a) {
  return PyLong_FromSize_t(back_bytes(norm_call(tensor(a[0], "x"), tensor(a[1], "w"), 0.0f)));
}
// dy, s, rstd, w, dsum, dx, dw, workspace -> dx, dw
PyObject* rms_norm_backward(PyObject* const* a) {
  const Tensor& dy = operand(a[0], "dy");
  const Tensor& w = operand(a[3], "w");
  const NormCall c = norm_call(dy, w, 0.0f);
  const at::ScalarType type = dy.scalar_type();
  OnDevice on(dy);
  const Rows dyr = rows_of(dy, dy, type, "dy"), sr = rows_of(operand(a[1], "s"), dy, type, "s");
  Rows dsr{nullptr, 0};
  if (a[4] != Py_None) dsr = rows_of(operand(a[4], "dsum"), dy, type, "dsum");
  require(a[2] != Py_None, "rstd must be a tensor");
  const Tensor rstd = row_vector(a[2], dy, "rstd");
  Tensor dx = given_or_empty(a[5], dy, type, "dx"), dw = given_or_empty(a[6], w, at::kFloat, "dw");
  require(dw.scalar_type() == at::kFloat && dw.device() == dy.device() && dw.sizes() == w.sizes() && (dw.size(-1) <= 1 || dw.stride(-1) == 1),
          "dw must be float32 of w's shape on the rows' device, its rows contiguous");
  const Tensor ws = workspace(a[7], back_bytes(c), dy);
  const Rows dxr = rows_of(dx, dy, type, "dx");
  const int64_t dw_row = dw.dim() == 2 && dw.size(0) > 1 ? dw.stride(0) : 0;
  finish(prsgd_rms_norm_backward(&c.cfg, dyr.at, dyr.distance, dsr.at, dsr.distance, sr.at, sr.distance, static_cast<const float*>(rstd.data_ptr()),
                                 c.w, c.w_row, dxr.at, dxr.distance, static_cast<float*>(dw.data_ptr()), dw_row, ws.data_ptr(), on.stream()));
  for (const Tensor& t : {dx, dw, ws}) written(t);
  return Py_BuildValue("(NN)", THPVariable_Wrap(dx), THPVariable_Wrap(dw));
}

// ---- matrices --------------------------------------------------------------------------------

struct Matrices { void* at; int64_t matrix, row; };
Matrices matrices_of(const Tensor& t, const Tensor& like, at::ScalarType type, const char* name) {
  const bool same = &t == &like || (t.device() == like.device() && t.sizes() == like.sizes());
  if (!t.is_cuda() || t.scalar_type() != type || !same) throw Refused(std::string(name) + " must have the device and shape of the matrices, and its type");
  if (t.size(-1) > 1 && t.stride(-1) != 1) throw Refused(std::string("rows of ") + name + " must be contiguous");
  return {t.data_ptr(), t.dim() == 3 ? t.stride(0) : 0, t.stride(-2)};
}
prsgd_orth_config orth_config(at::IntArrayRef shape, int32_t dtype, PyObject* coefficients, PyObject* steps, PyObject* eps) {
  prsgd_orth_config c{};
  require(shape.size() == 2 || shape.size() == 3, "matrices must be [count][rows][cols] or [rows][cols]");
  PyObject* three = PySequence_Fast(coefficients, "coefficients must be three numbers");
  if (three == nullptr) throw Raised{};
  const bool fits = PySequence_Fast_GET_SIZE(three) == 3;
  double v[3] = {0.0, 0.0, 0.0};
  for (int i = 0; fits && i < 3; ++i) v[i] = PyFloat_AsDouble(PySequence_Fast_GET_ITEM(three, i));
  Py_DECREF(three);
  if (PyErr_Occurred()) throw Raised{};
  require(fits, "coefficients must be three numbers");
  c.dtype = dtype;
  c.count = shape.size() == 3 ? size32(shape[0]) : 1;
  c.rows = size32(shape[shape.size() - 2]);
  c.cols = size32(shape[shape.size() - 1]);
  c.a = (float)v[0];
  c.b = (float)v[1];
  c.c = (float)v[2];
  c.steps = integer(steps);
  c.eps = (float)number(eps);
  return c;
}
size_t orth_bytes(const prsgd_orth_config& c) {
  const size_t n = prsgd_orthogonalize_workspace_bytes(&c);
  if (n == 0 && c.count != 0) finish(PRSGD_EINVAL);
  return n;
}
// count (or None), rows, cols, in bfloat16, coefficients, steps, eps -> bytes
PyObject* orthogonalize_bytes(PyObject* const* a) {
  const int64_t shape[3] = {a[0] == Py_None ? 1 : integer(a[0]), integer(a[1]), integer(a[2])};
  return PyLong_FromSize_t(orth_bytes(orth_config(at::IntArrayRef(shape, 3), a[3] == Py_True ? PRSGD_BF16 : PRSGD_F32, a[4], a[5], a[6])));
}
// g, out, coefficients, steps, eps, workspace -> out
PyObject* orthogonalize(PyObject* const* a) {
  const Tensor& g = operand(a[0], "g");
  const int32_t dtype = operand_type(g, "matrices must be a device tensor of float32 or bfloat16");
  const prsgd_orth_config c = orth_config(g.sizes(), dtype, a[2], a[3], a[4]);
  OnDevice on(g);
  const Matrices src = matrices_of(g, g, g.scalar_type(), "g");
  const Tensor ws = workspace(a[5], orth_bytes(c), g);
  Tensor out = given_or_empty(a[1], g, g.scalar_type(), "out");
  const Matrices dst = matrices_of(out, g, g.scalar_type(), "out");
  finish(prsgd_orthogonalize(&c, src.at, src.matrix, src.row, dst.at, dst.matrix, dst.row, ws.data_ptr(), on.stream()));
  written(out);
  written(ws);
  return THPVariable_Wrap(out);
}
// x, g, m, lr, momentum, nesterov, weight decay, scale, coefficients, steps, eps, workspace
PyObject* muon_step(PyObject* const* a) {
  const Tensor& x = operand(a[0], "x");
  const int32_t dtype = operand_type(x, "matrices must be a device tensor of float32 or bfloat16");
  const prsgd_orth_config c = orth_config(x.sizes(), dtype, a[8], a[9], a[10]);
  OnDevice on(x);
  const Tensor& m = operand(a[2], "m");
  const Matrices xs = matrices_of(x, x, x.scalar_type(), "x"), gs = matrices_of(operand(a[1], "g"), x, x.scalar_type(), "g"),
                 ms = matrices_of(m, x, at::kFloat, "m");
  const int nesterov = PyObject_IsTrue(a[5]);
  if (nesterov < 0) throw Raised{};
  const Tensor ws = workspace(a[11], orth_bytes(c), x);
  finish(prsgd_muon_step(&c, xs.at, xs.matrix, xs.row, gs.at, gs.matrix, gs.row, static_cast<float*>(ms.at), ms.matrix, ms.row,
                         (float)number(a[3]), (float)number(a[4]), nesterov, (float)number(a[6]), (float)number(a[7]),
                         ws.data_ptr(), on.stream()));
  for (const Tensor& t : {x, m, ws}) written(t);
  Py_RETURN_NONE;
}

PyObject* bind(PyObject* const* a) {
  Py_XDECREF(g_check);
  g_check = a[0];
  Py_INCREF(g_check);
  Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*), int N> PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", N, n);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Raised&) {
  } catch (const Refused& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}
#define PRSGD_METHOD(f, n) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call<f, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {PRSGD_METHOD(bind, 1),
                         PRSGD_METHOD(rms_norm, 8),
                         PRSGD_METHOD(rms_norm_backward, 8),
                         PRSGD_METHOD(rms_norm_backward_bytes, 2),
                         PRSGD_METHOD(orthogonalize, 6),
                         PRSGD_METHOD(orthogonalize_bytes, 7),
                         PRSGD_METHOD(muon_step, 12),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops() { return PyModule_Create(&module_def); }
