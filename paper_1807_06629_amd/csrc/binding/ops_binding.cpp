// Python module _ops: torch tensors to the calls of prsgd_ops.h.  It checks types, devices and strides, allocates what is not given, and
// passes addresses and the current stream on; nothing is computed here.  The same marshalling in Python took 10 us for a call on
// one row, three times the kernel and twice the launch.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/AutogradState.h>
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
  if (c10::AutogradState::get_tls_state().get_fw_grad_mode() && t._fw_grad(0).defined())
    throw Refused(std::string(what) + " has a forward-mode tangent, which the operators would drop: call them in a torch.autograd.Function with a jvp");
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

// ---- replicas of a model over tokens -----------------------------------------------------------

// Matrices [workers][rows][cols] or [rows][cols] that go with the rows of all workers.
struct Tables { void* at; int64_t workers, rows, cols, matrix, row; };
Tables tables_of(const Tensor& t, const Tensor& like, at::ScalarType type, const char* name) {
  if (t.device() != like.device() || t.scalar_type() != type || (t.dim() != 2 && t.dim() != 3))
    throw Refused(std::string(name) + " must be [workers][rows][cols] or [rows][cols] on the device, and of the type, of the other operands");
  if (t.size(-1) > 1 && t.stride(-1) != 1) throw Refused(std::string("rows of ") + name + " must be contiguous");
  const bool many = t.dim() == 3;
  return {t.data_ptr(), many ? t.size(0) : 1, t.size(-2), t.size(-1), many && t.size(0) > 1 ? t.stride(0) : 0, t.stride(-2)};
}
const int32_t* ids_of(const Tensor& t, const Tensor& like, const char* name) {
  if (!t.is_cuda() || t.device() != like.device() || t.scalar_type() != at::kInt || t.dim() != 1 || (t.size(0) > 1 && t.stride(0) != 1))
    throw Refused(std::string(name) + " must be contiguous int32, one value a row, on the rows' device");
  return static_cast<const int32_t*>(t.data_ptr());
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v != 0;
}

prsgd_embedding_config embedding_config(const Tensor& tokens, const Tables& t, int32_t dtype, float scale) {
  prsgd_embedding_config c{};
  require(t.workers > 0 && tokens.size(0) % t.workers == 0, "every worker must have the same number of tokens");
  c.dtype = dtype;
  c.workers = size32(t.workers);
  c.rows_per_worker = tokens.size(0) / t.workers;
  c.classes = size32(t.rows);
  c.width = size32(t.cols);
  c.scale = scale;
  return c;
}
const char* const kTableType = "tables must be device tensors of float32 or bfloat16";
// tokens, table, scale, out -> out
PyObject* embedding(PyObject* const* a) {
  const Tensor& tokens = operand(a[0], "tokens");
  const Tensor& table = operand(a[1], "table");
  const int32_t dtype = operand_type(table, kTableType);
  const Tables t = tables_of(table, table, table.scalar_type(), "table");
  const int32_t* ids = ids_of(tokens, table, "tokens");
  const prsgd_embedding_config c = embedding_config(tokens, t, dtype, (float)number(a[2]));
  OnDevice on(table);
  Tensor out = a[3] == Py_None ? device_empty({tokens.size(0), t.cols}, table.scalar_type(), table) : operand(a[3], "out");
  require(out.dim() == 2 && out.device() == table.device() && out.size(0) == tokens.size(0) && out.size(1) == t.cols, "out must be [rows][width] on the table's device");
  const Rows yr = rows_of(out, out, table.scalar_type(), "out");
  finish(prsgd_embedding(&c, ids, t.at, t.matrix, t.row, yr.at, yr.distance, on.stream()));
  written(out);
  return THPVariable_Wrap(out);
}
size_t embedding_bytes(const prsgd_embedding_config& c) {
  const size_t n = prsgd_embedding_backward_workspace_bytes(&c);
  if (n == 0) finish(PRSGD_EINVAL);
  return n;
}
// tokens, table -> bytes
PyObject* embedding_backward_bytes(PyObject* const* a) {
  const Tensor& tokens = tensor(a[0], "tokens");
  const Tensor& table = tensor(a[1], "table");
  require(tokens.dim() == 1, "tokens must be [rows]");
  const int32_t dtype = operand_type(table, kTableType);
  return PyLong_FromSize_t(embedding_bytes(embedding_config(tokens, tables_of(table, table, table.scalar_type(), "table"), dtype, 1.0f)));
}
// dy, tokens, table, scale, dtable, workspace -> dtable
PyObject* embedding_backward(PyObject* const* a) {
  const Tensor& dy = operand(a[0], "dy");
  const Tensor& tokens = operand(a[1], "tokens");
  const Tensor& table = tensor(a[2], "table");             // its shape alone
  const int32_t dtype = operand_type(table, kTableType);
  const int32_t* ids = ids_of(tokens, table, "tokens");
  const prsgd_embedding_config c = embedding_config(tokens, tables_of(table, table, table.scalar_type(), "table"), dtype, (float)number(a[3]));
  require(dy.dim() == 2 && dy.device() == table.device() && dy.size(0) == tokens.size(0) && dy.size(1) == table.size(-1),
          "dy must be [rows][width] on the table's device");
  OnDevice on(table);
  const Rows dyr = rows_of(dy, dy, table.scalar_type(), "dy");
  Tensor dtable = given_or_empty(a[4], table, table.scalar_type(), "dtable");
  require(dtable.sizes() == table.sizes(), "dtable must have the table's shape");
  const Tables d = tables_of(dtable, table, table.scalar_type(), "dtable");
  const Tensor ws = workspace(a[5], embedding_bytes(c), table);
  finish(prsgd_embedding_backward(&c, ids, dyr.at, dyr.distance, d.at, d.matrix, d.row, ws.data_ptr(), on.stream()));
  written(dtable);
  written(ws);
  return THPVariable_Wrap(dtable);
}

// Sequences of a scan: given, or as many as the starts or the states say, or one.
struct ScanCall {
  prsgd_scan_config cfg;
  const int32_t* starts;
};
ScanCall scan_call(const Tensor& v, PyObject* sequences, PyObject* starts, PyObject* const* states, int n_states) {
  ScanCall c{};
  require(v.dim() == 2, "rows must be a [rows][width] tensor");
  c.cfg.dtype = operand_type(v, "rows must be a device tensor of float32 or bfloat16");
  bool known = sequences != Py_None;
  int64_t n = known ? integer(sequences) : 1;
  require(n >= 0, "the number of sequences must not be negative");
  if (starts != Py_None) {
    const Tensor& t = operand(starts, "starts");
    c.starts = ids_of(t, v, "starts");
    if (!known) n = t.size(0) - 1;
    known = true;
    require(t.size(0) == n + 1 && n >= 1, "starts must have one value more than there are sequences");
  }
  for (int i = 0; i < n_states && !known; ++i)
    if (states[i] != Py_None) {
      const Tensor& t = operand(states[i], "states");
      require(t.dim() == 2, "states must be [sequences][width]");
      n = t.size(0);
      known = true;
    }
  c.cfg.sequences = size32(n);
  c.cfg.rows = v.size(0);
  c.cfg.width = size32(v.size(1));
  return c;
}
Rows states_of(const Tensor& t, const Tensor& v, const ScanCall& c, const char* name) {
  if (t.dim() != 2 || t.device() != v.device() || t.scalar_type() != at::kFloat || t.size(0) != c.cfg.sequences || t.size(1) != v.size(1))
    throw Refused(std::string(name) + " must be float32 [sequences][width] on the rows' device");
  return rows_of(t, t, at::kFloat, name);
}
Tensor states_given_or_empty(PyObject* o, const Tensor& v, const ScanCall& c, const char* name) {
  return o == Py_None ? device_empty({c.cfg.sequences, v.size(1)}, at::kFloat, v) : operand(o, name);
}
size_t scan_workspace(const ScanCall& c) {
  const size_t n = prsgd_gated_scan_workspace_bytes(&c.cfg);
  return n;                                                // 0 of what is refused: the call says so
}
// v, sequences -> bytes
PyObject* gated_scan_bytes(PyObject* const* a) {
  return PyLong_FromSize_t(scan_workspace(scan_call(tensor(a[0], "v"), a[1], Py_None, nullptr, 0)));
}
// v, gate, sequences, starts, initial, out, last, workspace -> h, last
PyObject* gated_scan(PyObject* const* a) {
  const Tensor& v = operand(a[0], "v");
  PyObject* const states[] = {a[4], a[6]};
  ScanCall c = scan_call(v, a[2], a[3], states, 2);
  const at::ScalarType type = v.scalar_type();
  OnDevice on(v);
  const Rows vr = rows_of(v, v, type, "v"), gr = rows_of(operand(a[1], "gate"), v, type, "gate");
  Rows ir{nullptr, 0};
  if (a[4] != Py_None) ir = states_of(operand(a[4], "initial"), v, c, "initial");
  c.cfg.clear = a[5] == Py_None && c.starts != nullptr ? 1 : 0;
  Tensor h = given_or_empty(a[5], v, type, "out"), last = states_given_or_empty(a[6], v, c, "last");
  const Rows hr = rows_of(h, v, type, "out"), lr = states_of(last, v, c, "last");
  const size_t bytes = scan_workspace(c);
  const Tensor ws = bytes > 0 ? workspace(a[7], bytes, v) : Tensor();
  finish(prsgd_gated_scan(&c.cfg, c.starts, vr.at, vr.distance, gr.at, gr.distance, static_cast<const float*>(ir.at), ir.distance, hr.at,
                          hr.distance, static_cast<float*>(lr.at), lr.distance, bytes > 0 ? ws.data_ptr() : nullptr, on.stream()));
  written(h);
  written(last);
  if (bytes > 0) written(ws);
  return Py_BuildValue("(NN)", THPVariable_Wrap(h), THPVariable_Wrap(last));
}
// dh, v, gate, h, sequences, starts, initial, dlast, dv, dgate, dinitial, workspace -> dv, dgate, dinitial
PyObject* gated_scan_backward(PyObject* const* a) {
  const Tensor& v = operand(a[1], "v");
  PyObject* const states[] = {a[6], a[7], a[10]};
  ScanCall c = scan_call(v, a[4], a[5], states, 3);
  const at::ScalarType type = v.scalar_type();
  OnDevice on(v);
  const Rows dhr = rows_of(operand(a[0], "dh"), v, type, "dh"), vr = rows_of(v, v, type, "v"), gr = rows_of(operand(a[2], "gate"), v, type, "gate"),
             hr = rows_of(operand(a[3], "h"), v, type, "h");
  Rows ir{nullptr, 0}, dlr{nullptr, 0};
  if (a[6] != Py_None) ir = states_of(operand(a[6], "initial"), v, c, "initial");
  if (a[7] != Py_None) dlr = states_of(operand(a[7], "dlast"), v, c, "dlast");
  if (c.starts != nullptr) c.cfg.clear = (a[8] == Py_None ? 1 : 0) + (a[9] == Py_None ? 2 : 0);
  Tensor dv = given_or_empty(a[8], v, type, "dv"), dgate = given_or_empty(a[9], v, type, "dgate"),
         dinitial = states_given_or_empty(a[10], v, c, "dinitial");
  const Rows dvr = rows_of(dv, v, type, "dv"), dgr = rows_of(dgate, v, type, "dgate"), dir = states_of(dinitial, v, c, "dinitial");
  const size_t bytes = scan_workspace(c);
  const Tensor ws = bytes > 0 ? workspace(a[11], bytes, v) : Tensor();
  finish(prsgd_gated_scan_backward(&c.cfg, c.starts, dhr.at, dhr.distance, vr.at, vr.distance, gr.at, gr.distance, hr.at, hr.distance,
                                   static_cast<const float*>(ir.at), ir.distance, static_cast<const float*>(dlr.at), dlr.distance, dvr.at,
                                   dvr.distance, dgr.at, dgr.distance, static_cast<float*>(dir.at), dir.distance,
                                   bytes > 0 ? ws.data_ptr() : nullptr, on.stream()));
  for (const Tensor& t : {dv, dgate, dinitial}) written(t);
  if (bytes > 0) written(ws);
  return Py_BuildValue("(NNN)", THPVariable_Wrap(dv), THPVariable_Wrap(dgate), THPVariable_Wrap(dinitial));
}

// x, p, seed, step, layer, residual, out -> out
PyObject* dropout(PyObject* const* a) {
  const Tensor& x = operand(a[0], "x");
  prsgd_dropout_config c{};
  require(x.dim() == 2, "rows must be a [rows][width] tensor");
  c.dtype = operand_type(x, "rows must be a device tensor of float32 or bfloat16");
  c.layer = integer(a[4]);
  c.rows = x.size(0);
  c.width = size32(x.size(1));
  c.p = (float)number(a[1]);
  auto word = [](PyObject* o) {
    const unsigned long long v = PyLong_AsUnsignedLongLong(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) throw Raised{};
    return (uint64_t)v;
  };
  c.seed = word(a[2]);
  const int64_t* step = nullptr;
  if (THPVariable_Check(a[3])) {
    const Tensor& t = operand(a[3], "step");
    require(t.scalar_type() == at::kLong && t.device() == x.device() && t.numel() == 1, "step must be a number or an int64 tensor of one on the rows' device");
    step = static_cast<const int64_t*>(t.data_ptr());
  } else {
    c.step = word(a[3]);
  }
  OnDevice on(x);
  const Rows xr = rows_of(x, x, x.scalar_type(), "x");
  Rows rr{nullptr, 0};
  if (a[5] != Py_None) rr = rows_of(operand(a[5], "residual"), x, x.scalar_type(), "residual");
  Tensor out = given_or_empty(a[6], x, x.scalar_type(), "out");
  const Rows yr = rows_of(out, x, x.scalar_type(), "out");
  finish(prsgd_dropout(&c, step, xr.at, xr.distance, rr.at, rr.distance, yr.at, yr.distance, on.stream()));
  written(out);
  return THPVariable_Wrap(out);
}

struct XentCall {
  prsgd_xent_config cfg;
  Tables w;
};
XentCall xent_call(const Tensor& h, const Tensor& w, PyObject* classes_first) {
  XentCall c{};
  require(h.dim() == 2, "rows must be a [rows][width] tensor");
  c.cfg.dtype = operand_type(h, "rows must be a device tensor of float32 or bfloat16");
  c.w = tables_of(w, h, h.scalar_type(), "w");
  c.cfg.classes_first = truth(classes_first) ? 1 : 0;
  require(c.w.workers > 0 && h.size(0) % c.w.workers == 0, "every worker must have the same number of rows");
  require((c.cfg.classes_first != 0 ? c.w.cols : c.w.rows) == h.size(1), "w must be [width][classes], or [classes][width] with classes_first, of the rows' width");
  c.cfg.workers = size32(c.w.workers);
  c.cfg.rows_per_worker = h.size(0) / c.w.workers;
  c.cfg.width = size32(h.size(1));
  c.cfg.classes = size32(c.cfg.classes_first != 0 ? c.w.rows : c.w.cols);
  return c;
}
size_t xent_bytes(const XentCall& c, bool backward) {
  const size_t n = backward ? prsgd_linear_cross_entropy_backward_workspace_bytes(&c.cfg) : prsgd_linear_cross_entropy_workspace_bytes(&c.cfg);
  if (n == 0) finish(PRSGD_EINVAL);
  return n;
}
// h, w, classes_first, backward -> bytes
PyObject* linear_cross_entropy_bytes(PyObject* const* a) {
  return PyLong_FromSize_t(xent_bytes(xent_call(tensor(a[0], "h"), tensor(a[1], "w"), a[2]), a[3] == Py_True));
}
const int32_t* labels_of(PyObject* o, const Tensor& h) {
  const Tensor& t = operand(o, "labels");
  const int32_t* at = ids_of(t, h, "labels");
  require(t.size(0) == h.size(0), "labels must have one value a row");
  return at;
}
// h, w, labels, classes_first, loss, lse, workspace -> loss, lse
PyObject* linear_cross_entropy(PyObject* const* a) {
  const Tensor& h = operand(a[0], "h");
  const XentCall c = xent_call(h, operand(a[1], "w"), a[3]);
  const int32_t* labels = labels_of(a[2], h);
  OnDevice on(h);
  const Rows hr = rows_of(h, h, h.scalar_type(), "h");
  Tensor loss = row_vector(a[4], h, "loss"), lse = row_vector(a[5], h, "lse");
  const Tensor ws = workspace(a[6], xent_bytes(c, false), h);
  finish(prsgd_linear_cross_entropy(&c.cfg, hr.at, hr.distance, c.w.at, c.w.matrix, c.w.row, labels, static_cast<float*>(loss.data_ptr()),
                                    static_cast<float*>(lse.data_ptr()), ws.data_ptr(), on.stream()));
  for (const Tensor& t : {loss, lse, ws}) written(t);
  return Py_BuildValue("(NN)", THPVariable_Wrap(loss), THPVariable_Wrap(lse));
}
// dloss, h, w, labels, lse, classes_first, dh, dw, workspace -> dh, dw
PyObject* linear_cross_entropy_backward(PyObject* const* a) {
  const Tensor& h = operand(a[1], "h");
  const Tensor& w = operand(a[2], "w");
  const XentCall c = xent_call(h, w, a[5]);
  const int32_t* labels = labels_of(a[3], h);
  OnDevice on(h);
  const Rows hr = rows_of(h, h, h.scalar_type(), "h");
  require(a[0] != Py_None && a[4] != Py_None, "dloss and lse must be tensors");
  const Tensor dloss = row_vector(a[0], h, "dloss"), lse = row_vector(a[4], h, "lse");
  Tensor dh = given_or_empty(a[6], h, h.scalar_type(), "dh"), dw = given_or_empty(a[7], w, h.scalar_type(), "dw");
  const Rows dhr = rows_of(dh, h, h.scalar_type(), "dh");
  require(dw.sizes() == w.sizes(), "dw must have w's shape");
  const Tables d = tables_of(dw, h, h.scalar_type(), "dw");
  const Tensor ws = workspace(a[8], xent_bytes(c, true), h);
  finish(prsgd_linear_cross_entropy_backward(&c.cfg, static_cast<const float*>(dloss.data_ptr()), hr.at, hr.distance, c.w.at, c.w.matrix, c.w.row,
                                             labels, static_cast<const float*>(lse.data_ptr()), dhr.at, dhr.distance, d.at, d.matrix, d.row,
                                             ws.data_ptr(), on.stream()));
  for (const Tensor& t : {dh, dw, ws}) written(t);
  return Py_BuildValue("(NN)", THPVariable_Wrap(dh), THPVariable_Wrap(dw));
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
                         PRSGD_METHOD(embedding, 4),
                         PRSGD_METHOD(embedding_backward, 6),
                         PRSGD_METHOD(embedding_backward_bytes, 2),
                         PRSGD_METHOD(gated_scan, 8),
                         PRSGD_METHOD(gated_scan_backward, 12),
                         PRSGD_METHOD(gated_scan_bytes, 2),
                         PRSGD_METHOD(dropout, 7),
                         PRSGD_METHOD(linear_cross_entropy, 7),
                         PRSGD_METHOD(linear_cross_entropy_backward, 9),
                         PRSGD_METHOD(linear_cross_entropy_bytes, 4),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops() { return PyModule_Create(&module_def); }
