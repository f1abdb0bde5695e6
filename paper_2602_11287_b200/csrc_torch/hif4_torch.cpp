// The calls between two linears of a block for PyTorch tensors: checks, output and workspace allocation, current stream, and
// the C call, without the interpreter in between (a call of one token costs the host less than the GPU).  The Python names,
// defaults and documentation are in binding.py, which passes every argument by position.
//
// A function returns its result, or the status code (a Python int) of a C call that refused its arguments; arguments that are
// not what they should be raise ValueError or TypeError.
#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <map>
#include <stdexcept>
#include <string>
#include <tuple>

#include "hif4.h"

namespace {

struct TypeProblem : std::runtime_error { using std::runtime_error::runtime_error; };

const at::Tensor* tensor_or_null(PyObject* o, const char* what) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) throw TypeProblem(std::string(what) + ": a tensor expected");
  return &THPVariable_Unpack(o);
}
const at::Tensor& tensor(PyObject* o, const char* what) {
  const at::Tensor* t = tensor_or_null(o, what);
  if (!t) throw TypeProblem(std::string(what) + ": a tensor expected");
  return *t;
}
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw TypeProblem("an integer expected");
  return v;
}
// A code of an enumeration; one that no int holds is none of them.
int code(PyObject* o) {
  const int64_t v = integer(o);
  return v < 0 || v > 0x7FFFFFFF ? -1 : static_cast<int>(v);
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw TypeProblem("a number expected");
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw TypeProblem("true or false expected");      // the object's own exception is set, and kept
  return v == 1;
}

std::string about(const at::Tensor& t) {
  std::string s = "[";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  s += "] of " + std::string(c10::toString(t.scalar_type())) + ", strides (";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.stride(i));
  return s + ")";
}
// The device of the call: that of its first tensor, current while it runs; every other tensor has to be there as well.
thread_local int call_device = -1;
void need_cuda(const at::Tensor& t) {
  if (!t.is_cuda()) throw std::invalid_argument("the HiF4 library takes device tensors only (no CPU path exists)");
  if (t.get_device() != call_device) throw std::invalid_argument("tensors of one call must be on one device");
}
struct OnDeviceOf {
  c10::cuda::OptionalCUDAGuard guard;
  explicit OnDeviceOf(const at::Tensor& t) {
    call_device = t.is_cuda() ? t.get_device() : -1;
    need_cuda(t);
    guard.set_index(static_cast<c10::DeviceIndex>(call_device));
  }
};
int type_code(at::ScalarType t) {
  switch (t) {
    case at::kBFloat16: return HIF4_BF16;
    case at::kFloat: return HIF4_FP32;
    case at::kHalf: return HIF4_FP16;
    default: throw TypeProblem(std::string("bfloat16, float16 or float32 expected, not ") + c10::toString(t));
  }
}

struct Mat { void* p; int64_t ld; };
// A [rows, cols] operand with unit column stride; no address without one.
Mat matrix(const at::Tensor* t, int64_t rows, int64_t cols, at::ScalarType type, const char* what) {
  if (!t) return {nullptr, 0};
  need_cuda(*t);
  if (t->scalar_type() != type || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols || (cols > 1 && t->stride(1) != 1))
    throw std::invalid_argument(std::string(what) + ": [" + std::to_string(rows) + ", " + std::to_string(cols) + "] of " + c10::toString(type) +
                                " with unit column stride expected, got " + about(*t));
  const int64_t ld = t->stride(0);
  return {t->data_ptr(), rows > 1 || ld >= cols ? ld : cols};
}
void* vector(const at::Tensor* t, int64_t n, at::ScalarType type, const char* what) {
  if (!t) return nullptr;
  need_cuda(*t);
  if (t->scalar_type() != type || t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1))
    throw std::invalid_argument(std::string(what) + ": contiguous [" + std::to_string(n) + "] of " + c10::toString(type) + " expected, got " + about(*t));
  return t->data_ptr();
}
void* units(const at::Tensor* t, int64_t rows, int64_t n, const char* what) {
  if (!t) return nullptr;
  need_cuda(*t);
  if (t->scalar_type() != at::kByte || t->dim() != 3 || t->size(0) != rows || t->size(1) != n || t->size(2) != HIF4_UNIT_BYTES || !t->is_contiguous())
    throw std::invalid_argument(std::string(what) + ": contiguous uint8 units [" + std::to_string(rows) + ", " + std::to_string(n) + ", 36] expected, got " + about(*t));
  return t->data_ptr();
}
Mat gates(const at::Tensor* t, int64_t rows, int64_t cols, int64_t per, at::ScalarType type) {
  if (!t) return {nullptr, 0};
  if (per < 1) throw std::invalid_argument("a gate needs rows_per_gate >= 1");
  return matrix(t, rows / per + (rows % per != 0), cols, type, "gate");
}
at::Tensor new_rows(int64_t rows, int64_t cols, at::ScalarType type, const at::Tensor& like) {
  return at::empty({rows, cols}, like.options().dtype(type));
}
at::Tensor new_units(int64_t rows, int64_t n, const at::Tensor& like) {
  return at::empty({rows, n, HIF4_UNIT_BYTES}, like.options().dtype(at::kByte));
}
void* stream_of(const at::Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.device().index()).stream(); }
template <typename T> T* at_of(const at::Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }

PyObject* wrap(const at::Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}
PyObject* status(hif4_status s) { return PyLong_FromLong(s); }

// Calls are made with the GIL held: they only enqueue.
template <typename F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, F&& f) {
  try {
    if (given != wanted) throw TypeProblem("wrong number of arguments");
    return f();
  } catch (const TypeProblem& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.what());
  } catch (const std::invalid_argument& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// The caller's workspace, or a new one.
struct Workspace {
  at::Tensor held;
  void* p = nullptr;
  size_t bytes = 0;
  Workspace(const at::Tensor* given, size_t need, const at::Tensor& like) {
    if (given) {
      need_cuda(*given);
      if (!given->is_contiguous()) throw std::invalid_argument("workspace: contiguous memory expected, got " + about(*given));
      p = given->data_ptr();
      bytes = given->nbytes();
    } else if (need > 0) {
      held = at::empty({static_cast<int64_t>(need)}, like.options().dtype(at::kByte));
      p = held.data_ptr();
      bytes = need;
    }
  }
};

// (x, weight, bias, residual, res_scale, gate, rows_per_gate, post, post_weight, pre, eps, units, mode, out_h, out_y)
PyObject* block_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 15, [&]() -> PyObject* {
    const at::Tensor& x = tensor(a[0], "x");
    const OnDeviceOf on(x);
    if (x.dim() != 2) throw std::invalid_argument("x: a matrix expected");
    const int64_t rows = x.size(0), cols = x.size(1);
    const at::ScalarType type = x.scalar_type();
    const at::Tensor *w = tensor_or_null(a[1], "weight"), *b = tensor_or_null(a[2], "bias"), *res = tensor_or_null(a[3], "residual"),
                     *gate = tensor_or_null(a[5], "gate"), *wp = tensor_or_null(a[8], "post_weight"), *out_h = tensor_or_null(a[13], "out_h"),
                     *out_y = tensor_or_null(a[14], "out_y");
    const at::ScalarType wtype = w ? w->scalar_type() : b ? b->scalar_type() : wp ? wp->scalar_type() : type;
    hif4_block_norm_args p{};
    p.rows = rows; p.cols = cols;
    const Mat mx = matrix(&x, rows, cols, type, "x"), mr = matrix(res, rows, cols, type, "residual");
    p.dt = static_cast<hif4_dtype>(type_code(type));
    p.dt_w = static_cast<hif4_dtype>(type_code(wtype));
    p.x = mx.p; p.ld_x = mx.ld;
    p.residual = mr.p; p.ld_residual = mr.ld;
    p.res_scale = static_cast<float>(real(a[4]));
    p.rows_per_gate = integer(a[6]);
    const Mat mg = gates(gate, rows, cols, p.rows_per_gate, type);
    p.gate = mg.p; p.ld_gate = mg.ld;
    p.post = static_cast<hif4_norm_kind>(code(a[7]));
    p.post_weight = vector(wp, cols, wtype, "post_weight");
    p.pre = static_cast<hif4_norm_kind>(code(a[9]));
    p.pre_weight = vector(w, cols, wtype, "weight");
    p.pre_bias = vector(b, cols, wtype, "bias");
    p.eps = static_cast<float>(real(a[10]));
    p.y_units = truth(a[11]) ? 1 : 0;
    p.mode = static_cast<hif4_round>(code(a[12]));
    at::Tensor h, y;
    if (out_h) h = *out_h;
    else if (res || gate || p.post != HIF4_NORM_NONE) h = new_rows(rows, cols, type, x);
    if (out_y) y = *out_y;
    else if (p.pre != HIF4_NORM_NONE) y = p.y_units ? new_units(rows, cols / HIF4_UNIT_ELEMS, x) : new_rows(rows, cols, type, x);
    if (h.defined()) {
      const Mat m = matrix(&h, rows, cols, type, "out_h");
      p.h = m.p; p.ld_h = m.ld;
    }
    if (y.defined()) {
      if (p.y_units) {
        p.y = units(&y, rows, cols / HIF4_UNIT_ELEMS, "out_y");
      } else {
        const Mat m = matrix(&y, rows, cols, type, "out_y");
        p.y = m.p; p.ld_y = m.ld;
      }
    }
    if (h.defined() || y.defined()) {
      const hif4_status s = hif4_block_norm(&p, stream_of(x));
      if (s != HIF4_OK) return status(s);
    }
    PyObject* result = PyTuple_New(2);
    if (!result) return nullptr;
    if (h.defined()) PyTuple_SET_ITEM(result, 0, wrap(h));
    else { Py_INCREF(a[0]); PyTuple_SET_ITEM(result, 0, a[0]); }
    PyTuple_SET_ITEM(result, 1, wrap(y));
    return result;
  });
}

// (dy, h, weight, dh, x, bias, res_scale, gate, rows_per_gate, post, post_weight, pre, eps, wanted, workspace), `wanted` the sum of
// 1 (dx), 2 (dresidual), 4 (dgate) and 8 (weights and bias)
//   -> (dx, dresidual, dgate, dweight, dbias, dpost_weight)
PyObject* block_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 15, [&]() -> PyObject* {
    const at::Tensor *dy = tensor_or_null(a[0], "dy"), *h = tensor_or_null(a[1], "h"), *w = tensor_or_null(a[2], "weight"),
                     *dh = tensor_or_null(a[3], "dh"), *x = tensor_or_null(a[4], "x"), *gate = tensor_or_null(a[7], "gate"),
                     *wp = tensor_or_null(a[10], "post_weight"), *ws = tensor_or_null(a[14], "workspace");
    const at::Tensor* first = dy ? dy : dh;
    if (!first || first->dim() != 2) throw std::invalid_argument("dy or dh: a matrix expected");
    const OnDeviceOf on(*first);
    const int64_t rows = first->size(0), cols = first->size(1);
    const at::ScalarType type = first->scalar_type();
    const at::ScalarType wtype = w ? w->scalar_type() : wp ? wp->scalar_type() : type;
    hif4_block_norm_backward_args p{};
    p.rows = rows; p.cols = cols;
    const Mat mdy = matrix(dy, rows, cols, type, "dy"), mdh = matrix(dh, rows, cols, type, "dh"), mh = matrix(h, rows, cols, type, "h"),
              mx = matrix(x, rows, cols, type, "x");
    p.dt = static_cast<hif4_dtype>(type_code(type));
    p.dt_w = static_cast<hif4_dtype>(type_code(wtype));
    p.dy = mdy.p; p.ld_dy = mdy.ld;
    p.dh = mdh.p; p.ld_dh = mdh.ld;
    p.h = mh.p; p.ld_h = mh.ld;
    p.x = mx.p; p.ld_x = mx.ld;
    p.res_scale = static_cast<float>(real(a[6]));
    p.rows_per_gate = integer(a[8]);
    const Mat mg = gates(gate, rows, cols, p.rows_per_gate, type);
    p.gate = mg.p; p.ld_gate = mg.ld;
    p.post = static_cast<hif4_norm_kind>(code(a[9]));
    p.post_weight = vector(wp, cols, wtype, "post_weight");
    p.pre = static_cast<hif4_norm_kind>(code(a[11]));
    p.pre_weight = vector(w, cols, wtype, "weight");
    p.eps = static_cast<float>(real(a[12]));
    const auto sums = [&] { return at::empty({cols}, first->options().dtype(at::kFloat)); };
    const int64_t wanted = integer(a[13]);
    const bool weights = (wanted & 8) != 0, has_bias = truth(a[5]);
    at::Tensor d[6];
    if (wanted & 1) d[0] = new_rows(rows, cols, type, *first);
    if (wanted & 2) d[1] = new_rows(rows, cols, type, *first);
    if (gate && (wanted & 4)) d[2] = new_rows(gate->size(0), cols, type, *first);
    if (w && dy && weights) d[3] = sums();
    if (has_bias && dy && weights) d[4] = sums();
    if (wp && weights) d[5] = sums();
    p.dx = at_of<void>(d[0]); p.ld_dx = cols;
    p.dresidual = at_of<void>(d[1]); p.ld_dresidual = cols;
    p.dgate = at_of<void>(d[2]);
    p.dpre_weight = at_of<float>(d[3]);
    p.dpre_bias = at_of<float>(d[4]);
    p.dpost_weight = at_of<float>(d[5]);
    size_t need = 0;
    hif4_status s = hif4_block_norm_backward_workspace(rows, cols, &need);
    if (s != HIF4_OK) return status(s);
    const Workspace space(ws, need, *first);
    s = hif4_block_norm_backward(&p, space.p, space.bytes, stream_of(*first));
    if (s != HIF4_OK) return status(s);
    PyObject* result = PyTuple_New(6);
    if (!result) return nullptr;
    for (int i = 0; i < 6; ++i) PyTuple_SET_ITEM(result, i, wrap(d[i]));
    return result;
  });
}

// Activations [rows, K] or units [rows, K / 64, 36].
struct Activations { int64_t rows, K; Mat m; int dt, is_units; };
Activations activations(const at::Tensor& x) {
  if (x.scalar_type() == at::kByte) {
    if (x.dim() != 3) throw std::invalid_argument("x: units [rows, K / 64, 36] expected, got " + about(x));
    return {x.size(0), x.size(1) * HIF4_UNIT_ELEMS, {units(&x, x.size(0), x.size(1), "x"), 0}, HIF4_BF16, 1};
  }
  if (x.dim() != 2) throw std::invalid_argument("x: a matrix expected, got " + about(x));
  const Mat m = matrix(&x, x.size(0), x.size(1), x.scalar_type(), "x");
  return {x.size(0), x.size(1), m, type_code(x.scalar_type()), 0};
}

// What the workspace queries answered, by all that the answer depends on.
size_t workspace_bytes(int call, int device, const std::tuple<int64_t, int64_t, int64_t, int, int, int>& key, hif4_status& s,
                       hif4_status (*query)(const void*, size_t*), const void* args) {
  static std::map<std::tuple<int, int, int64_t, int64_t, int64_t, int, int, int>, size_t> known;
  const auto k = std::tuple_cat(std::make_tuple(call, device), key);
  const auto it = known.find(k);
  if (it != known.end()) { s = HIF4_OK; return it->second; }
  size_t need = 0;
  s = query(args, &need);
  if (s != HIF4_OK) return 0;
  if (known.size() >= 4096) known.clear();
  return known[k] = need;
}

// (x, w_units, w_up_units, bias, bias_up, residual, res_scale, act, dtype code or -1, units, mode, out, workspace)
PyObject* linear_act(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 13, [&]() -> PyObject* {
    const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "w_units");
    const at::Tensor *wu = tensor_or_null(a[2], "w_up_units"), *b = tensor_or_null(a[3], "bias"), *bu = tensor_or_null(a[4], "bias_up"),
                     *res = tensor_or_null(a[5], "residual"), *out = tensor_or_null(a[11], "out"), *ws = tensor_or_null(a[12], "workspace");
    const OnDeviceOf on(x);
    const Activations act = activations(x);
    if (w.dim() != 3) throw std::invalid_argument("w_units: units [N, K / 64, 36] expected, got " + about(w));
    const int64_t M = act.rows, N = w.size(0), K = act.K;
    const int64_t out_type = integer(a[8]);
    const bool to_units = truth(a[9]);
    const at::ScalarType type = out_type == HIF4_BF16 ? at::kBFloat16 : out_type == HIF4_FP32 ? at::kFloat : out_type == HIF4_FP16 ? at::kHalf
                                : out && !to_units ? out->scalar_type() : act.is_units ? at::kBFloat16 : x.scalar_type();
    hif4_linear_act_args p{};
    p.M = M; p.N = N; p.K = K;
    p.X = act.m.p; p.ld_x = act.m.ld;
    p.dt_x = static_cast<hif4_dtype>(act.dt);
    p.x_units = act.is_units;
    p.mode = static_cast<hif4_round>(code(a[10]));
    p.W_units = units(&w, N, K / HIF4_UNIT_ELEMS, "w_units");
    p.W_up_units = units(wu, N, K / HIF4_UNIT_ELEMS, "w_up_units");
    p.dt = static_cast<hif4_dtype>(type_code(type));
    p.bias = vector(b, N, type, "bias");
    p.bias_up = vector(bu, N, type, "bias_up");
    p.act = static_cast<hif4_activation>(code(a[7]));
    const Mat mr = matrix(res, M, N, type, "residual");
    p.residual = mr.p; p.ld_residual = mr.ld;
    p.res_scale = static_cast<float>(real(a[6]));
    p.y_units = to_units ? 1 : 0;
    at::Tensor y = out ? *out : to_units ? new_units(M, N / HIF4_UNIT_ELEMS, x) : new_rows(M, N, type, x);
    if (to_units) {
      p.Y = units(&y, M, N / HIF4_UNIT_ELEMS, "out");
    } else {
      const Mat m = matrix(&y, M, N, type, "out");
      p.Y = m.p; p.ld_y = m.ld;
    }
    hif4_status s;
    const size_t need = workspace_bytes(wu ? 1 : 0, x.device().index(), {M, N, K, p.x_units, p.dt, p.y_units}, s,
                                        reinterpret_cast<hif4_status (*)(const void*, size_t*)>(wu ? hif4_gated_linear_workspace : hif4_linear_act_workspace), &p);
    if (s != HIF4_OK) return status(s);
    const Workspace space(ws, need, x);
    s = (wu ? hif4_gated_linear : hif4_linear_act)(&p, space.p, space.bytes, stream_of(x));
    if (s != HIF4_OK) return status(s);
    if (out) { Py_INCREF(a[11]); return a[11]; }
    return wrap(y);
  });
}

// (dy, x, w_units, w_up_units, bias, bias_up, act, mode, want_dx, want_dbias, precise, workspace) -> (dx, dbias, dbias_up)
PyObject* linear_act_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const at::Tensor &dy = tensor(a[0], "dy"), &w = tensor(a[2], "w_units");
    const at::Tensor *x = tensor_or_null(a[1], "x"), *wu = tensor_or_null(a[3], "w_up_units"), *b = tensor_or_null(a[4], "bias"),
                     *bu = tensor_or_null(a[5], "bias_up"), *ws = tensor_or_null(a[11], "workspace");
    const OnDeviceOf on(dy);
    if (dy.dim() != 2) throw std::invalid_argument("dy: a matrix expected");
    if (w.dim() != 3) throw std::invalid_argument("w_units: units [N, K / 64, 36] expected, got " + about(w));
    const int64_t M = dy.size(0), N = dy.size(1), K = w.size(1) * HIF4_UNIT_ELEMS;
    const at::ScalarType type = dy.scalar_type();
    hif4_linear_act_backward_args p{};
    p.M = M; p.N = N; p.K = K;
    p.ld_x = K;
    if (x) {
      const Activations act = activations(*x);
      if (act.rows != M || act.K != K)
        throw std::invalid_argument("x: " + std::to_string(M) + " rows of " + std::to_string(K) + " activations expected, got " + about(*x));
      p.X = act.m.p; p.ld_x = act.m.ld;
      p.dt_x = static_cast<hif4_dtype>(act.dt);
      p.x_units = act.is_units;
    }
    p.mode = static_cast<hif4_round>(code(a[7]));
    p.W_units = units(&w, N, K / HIF4_UNIT_ELEMS, "w_units");
    p.W_up_units = units(wu, N, K / HIF4_UNIT_ELEMS, "w_up_units");
    const Mat mdy = matrix(&dy, M, N, type, "dy");
    p.dt = static_cast<hif4_dtype>(type_code(type));
    p.bias = vector(b, N, type, "bias");
    p.bias_up = vector(bu, N, type, "bias_up");
    p.act = static_cast<hif4_activation>(code(a[6]));
    p.dY = mdy.p; p.ld_dy = mdy.ld;
    at::Tensor dx, db, dbu;
    if (truth(a[8])) dx = new_rows(M, K, type, dy);
    if (truth(a[9])) {
      db = at::empty({N}, dy.options().dtype(at::kFloat));
      if (wu) dbu = at::empty({N}, dy.options().dtype(at::kFloat));
    }
    p.dX = at_of<void>(dx); p.ld_dx = K;
    p.dbias = at_of<float>(db);
    p.dbias_up = at_of<float>(dbu);
    p.precise = truth(a[10]) ? 1 : 0;
    hif4_status s;
    const size_t need = workspace_bytes(wu ? 3 : 2, dy.device().index(), {M, N, K, p.x_units, p.dt, (p.act == HIF4_ACT_NONE) + 2 * p.precise}, s,
                                        reinterpret_cast<hif4_status (*)(const void*, size_t*)>(wu ? hif4_gated_linear_backward_workspace : hif4_linear_act_backward_workspace), &p);
    if (s != HIF4_OK) return status(s);
    const Workspace space(ws, need, dy);
    s = (wu ? hif4_gated_linear_backward : hif4_linear_act_backward)(&p, space.p, space.bytes, stream_of(dy));
    if (s != HIF4_OK) return status(s);
    PyObject* result = PyTuple_New(3);
    if (!result) return nullptr;
    PyTuple_SET_ITEM(result, 0, wrap(dx));
    PyTuple_SET_ITEM(result, 1, wrap(db));
    PyTuple_SET_ITEM(result, 2, wrap(dbu));
    return result;
  });
}

PyMethodDef methods[] = {
    {"block_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(block_norm)), METH_FASTCALL, nullptr},
    {"block_norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(block_norm_backward)), METH_FASTCALL, nullptr},
    {"linear_act", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear_act)), METH_FASTCALL, nullptr},
    {"linear_act_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear_act_backward)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_hif4_torch", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__hif4_torch(void) { return PyModule_Create(&module); }
