// Python entry points of the 4-bit weights and the block residual.  These calls run beside kernels of a few
// microseconds, so their tensors are looked at here and not through Python: what the C ABI cannot see (devices,
// dtypes, shapes, the sizes of buffers) is checked, outputs and workspaces that the caller does not pass are
// allocated, and the C ABI is called on the current stream of the tensors' GPU.  A call whose GPU is not the
// current one returns None and launches nothing; flashnorm.py makes it current and calls again.  A status other
// than FN_OK comes back as an int.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <initializer_list>
#include <stdexcept>
#include <string>

#include "flashnorm.h"

namespace {

using at::Tensor;

struct TypeError : std::runtime_error {
  using std::runtime_error::runtime_error;
};

// What a call knows of its tensors: its name for messages, the GPU, the element type.
struct Call {
  const char* where;
  c10::DeviceIndex dev;
  at::ScalarType type;
  int code;     // fn_dtype
  int64_t per;  // elements of 16 bytes

  [[noreturn]] void refuse(const std::string& what) const { throw std::invalid_argument(std::string(where) + ": " + what); }
};

const Tensor* tensor_or_none(PyObject* o) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) throw TypeError("expected a tensor");
  return &THPVariable_Unpack(o);
}

const Tensor& tensor(PyObject* o) {
  const Tensor* t = tensor_or_none(o);
  if (!t) throw TypeError("expected a tensor");
  return *t;
}

int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw TypeError("expected an integer");
  return v;
}

int small(PyObject* o) {
  const int64_t v = integer(o);
  if (v != (int)v) throw std::invalid_argument("an integer is out of range");
  return (int)v;
}

bool flag(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw TypeError("expected a truth value");
  return v != 0;
}

float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw TypeError("expected a number");
  return (float)v;
}

// Begin a call by its first tensor; false where its GPU is not the current one (or it is on no GPU).
bool begin_any(Call& c, const char* where, const Tensor& t) {
  c.where = where;
  if (!t.is_cuda() || t.get_device() != c10::hip::current_device()) return false;
  c.dev = (c10::DeviceIndex)t.get_device();
  return true;
}

// The same with a matrix whose type is the call's.
bool begin(Call& c, const char* where, const Tensor& t) {
  if (!begin_any(c, where, t)) return false;
  c.type = t.scalar_type();
  if (c.type == at::kBFloat16) c.code = FN_BF16, c.per = 8;
  else if (c.type == at::kFloat) c.code = FN_F32, c.per = 4;
  else throw TypeError(std::string(where) + ": unsupported dtype " + c10::toString(c.type));
  if (t.dim() != 2) c.refuse("expected a 2-D tensor");
  return true;
}

void same_gpu(const Call& c, const Tensor& t) {
  if (!t.is_cuda() || t.get_device() != c.dev) c.refuse("every tensor must be on one GPU (one is on " + t.device().str() + ")");
}

struct Matrix {
  void* p = nullptr;
  int64_t ld = 0;
};

Matrix matrix(const Call& c, const Tensor* t, int64_t rows, int64_t cols, const char* name) {
  if (!t) return {};
  same_gpu(c, *t);
  if (t->dim() != 2 || t->size(0) != rows || t->size(1) != cols || t->scalar_type() != c.type)
    c.refuse(std::string(name) + " must be a " + std::to_string(rows) + " x " + std::to_string(cols) + " " +
             c10::toString(c.type) + " tensor");
  if (t->stride(1) != 1 && cols > 1) c.refuse(std::string(name) + " must be row-major (unit column stride)");
  // The pitch of a single row says nothing.
  return {t->data_ptr(), rows > 1 ? t->stride(0) : (cols + c.per - 1) / c.per * c.per};
}

float* vector(const Call& c, const Tensor* t, int64_t n, const char* name) {
  if (!t) return nullptr;
  if (t->scalar_type() != at::kFloat || t->numel() != n || !t->is_contiguous())
    c.refuse(std::string(name) + " must be a contiguous fp32 vector of " + std::to_string(n) + " elements");
  same_gpu(c, *t);
  return t->data_ptr<float>();
}

// A new tensor on the call's GPU, straight from torch's allocator: the operator call around it takes as long.
Tensor new_tensor(const Call& c, at::IntArrayRef size, at::ScalarType type) {
  return Tensor(at::detail::empty_cuda(size, type, c10::Device(c10::kCUDA, c.dev), std::nullopt));
}

// A new matrix, its rows padded to 16 bytes (a view of the first columns where that pads).
Tensor new_matrix(const Call& c, int64_t rows, int64_t cols) {
  const int64_t ld = (cols + c.per - 1) / c.per * c.per;
  const Tensor t = new_tensor(c, {rows, ld}, c.type);
  return ld == cols ? t : t.narrow(1, 0, cols);
}

// The caller's tensors that a call has written count as changed for autograd, which refuses a backward pass through
// values it kept of them (inference tensors have no count).
void written(std::initializer_list<const Tensor*> given) {
  for (const Tensor* t : given)
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

// The caller's workspace, checked, or a new one.
Tensor workspace(const Call& c, const Tensor* given, size_t need) {
  if (!need) return Tensor();
  if (!given) return new_tensor(c, {(int64_t)need}, at::kByte);
  same_gpu(c, *given);
  if (!given->is_contiguous() || given->nbytes() < need)
    c.refuse("the workspace must be " + std::to_string(need) + " contiguous bytes");
  return *given;
}

void* address(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
void* stream_of(const Call& c) { return c10::hip::getCurrentHIPStream(c.dev).stream(); }
PyObject* wrap(const Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
PyObject* again(PyObject* o) {
  Py_INCREF(o);
  return o;
}

template <typename F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const TypeError& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, e.what());
  } catch (const std::invalid_argument& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const c10::OutOfMemoryError& e) {
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    PyErr_Clear();
    PyErr_SetString(type ? type : PyExc_MemoryError, e.what_without_backtrace());
    Py_XDECREF(type);
    Py_XDECREF(torch);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

bool arity(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return false;
}

// The size of a 4-bit weight; refused where there is none of that shape.
int64_t w4_bytes(const Call& c, int64_t K, int64_t N, int layout, int group) {
  const size_t bytes = fold_weights_w4_size(K, N, layout, group);
  if (!bytes)
    c.refuse("no 4-bit weight of K = " + std::to_string(K) + ", N = " + std::to_string(N) + ", layout " +
             std::to_string(layout) + ", group " + std::to_string(group));
  return (int64_t)bytes;
}

// W, g, layout, group, zero_points -> the packed weight
PyObject* w4_fold(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!arity(n, 5)) return nullptr;
  return guarded([&]() -> PyObject* {
    const Tensor& W = tensor(v[0]);
    Call c;
    if (!begin(c, "fold_weights_w4", W)) Py_RETURN_NONE;
    const int64_t K = W.size(0), N = W.size(1);
    const int layout = small(v[2]), group = small(v[3]);
    const float* g = vector(c, tensor_or_none(v[1]), K, "g");
    const Tensor data = new_tensor(c, {w4_bytes(c, K, N, layout, group)}, at::kByte);
    const int s = fold_weights_w4(W.data_ptr(), W.stride(0), W.stride(1), c.code, g, K, N, layout, group, flag(v[4]),
                                  data.data_ptr(), stream_of(c));
    return s ? PyLong_FromLong(s) : wrap(data);
  });
}

// data, K, N, layout, group -> the fp32 weight
PyObject* w4_unpack(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!arity(n, 5)) return nullptr;
  return guarded([&]() -> PyObject* {
    const Tensor& data = tensor(v[0]);
    Call c;
    if (!begin_any(c, "unpack_weights_w4", data)) Py_RETURN_NONE;
    const int64_t K = integer(v[1]), N = integer(v[2]);
    const int layout = small(v[3]), group = small(v[4]);
    if (!data.is_contiguous() || (int64_t)data.nbytes() < w4_bytes(c, K, N, layout, group)) c.refuse("no whole 4-bit weight");
    const Tensor out = new_tensor(c, {K, N}, at::kFloat);
    const int s = unpack_weights_w4(data.data_ptr(), K, N, layout, group, out.data_ptr<float>(), N, stream_of(c));
    return s ? PyLong_FromLong(s) : wrap(out);
  });
}

enum { kLinear, kGlu, kRowscale };

// kind, a, data, K, N, layout, group, eps, g, bias, out, inv_rms, row_scale, workspace -> the output
PyObject* w4_product(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!arity(n, 14)) return nullptr;
  return guarded([&]() -> PyObject* {
    static const char* const names[] = {"flashnorm_linear_w4", "flashnorm_glu_w4", "rowscale_linear_w4"};
    const int64_t kind = integer(v[0]);
    if (kind < kLinear || kind > kRowscale) throw std::invalid_argument("unknown product");
    const Tensor& a = tensor(v[1]);
    Call c;
    if (!begin(c, names[kind], a)) Py_RETURN_NONE;
    const Tensor& data = tensor(v[2]);
    const int64_t K = integer(v[3]), N = integer(v[4]);
    const int layout = small(v[5]), group = small(v[6]);
    const int want = kind == kGlu ? FN_LAYOUT_GLU : FN_LAYOUT_LINEAR;
    const int64_t M = a.size(0);
    if (a.size(1) != K || layout != want)
      c.refuse("activations of width " + std::to_string(a.size(1)) + " and layout " + std::to_string(want) +
               ", a 4-bit weight of K = " + std::to_string(K) + " and layout " + std::to_string(layout));
    same_gpu(c, data);
    if (!data.is_contiguous() || (int64_t)data.nbytes() < w4_bytes(c, K, N, layout, group)) c.refuse("no whole 4-bit weight");
    const int64_t cols = kind == kGlu ? N / 2 : N;
    const Matrix A = matrix(c, &a, M, K, "the activations");
    const float* g = vector(c, tensor_or_none(v[8]), K, "g");
    const float* bias = vector(c, tensor_or_none(v[9]), N, "bias");
    const Tensor* out = tensor_or_none(v[10]);
    float* inv_rms = vector(c, tensor_or_none(v[11]), M, "inv_rms");
    const float* row_scale = vector(c, tensor_or_none(v[12]), M, "row_scale");
    const size_t need = M > FN_W4_FEW_M ? flashnorm_w4_workspace_size(M, K, N, layout, group) : 0;
    const Tensor ws = workspace(c, tensor_or_none(v[13]), need);
    const Tensor made = out ? Tensor() : new_matrix(c, M, cols);
    const Matrix Y = matrix(c, out ? out : &made, M, cols, "the output");
    const float eps = real(v[7]);
    int s;
    if (kind == kLinear)
      s = flashnorm_linear_w4(A.p, M, K, A.ld, c.code, g, data.data_ptr(), N, group, eps, bias, Y.p, Y.ld, c.code, inv_rms,
                              address(ws), need, stream_of(c));
    else if (kind == kGlu)
      s = flashnorm_glu_w4(A.p, M, K, A.ld, c.code, g, data.data_ptr(), cols, group, eps, Y.p, Y.ld, c.code, address(ws),
                           need, stream_of(c));
    else
      s = rowscale_linear_w4(A.p, M, K, A.ld, c.code, data.data_ptr(), N, group, row_scale, Y.p, Y.ld, c.code, address(ws),
                             need, stream_of(c));
    if (s) return PyLong_FromLong(s);
    written({out, tensor_or_none(v[11]), need ? tensor_or_none(v[13]) : nullptr});
    return out ? again(v[10]) : wrap(made);
  });
}

Matrix gate_of(const Call& c, const Tensor* gate, int64_t rows_per_gate, int64_t M, int64_t K) {
  if (!gate) return {};
  if (rows_per_gate < 1) c.refuse("rows_per_gate must be at least 1");
  return matrix(c, gate, M / rows_per_gate + (M % rows_per_gate != 0), K, "the gate (a row for each rows_per_gate rows)");
}

// x, h, g_post, eps_post, gate, rows_per_gate, res_scale, branch_scale, g_pre, eps_pre, out, normed, inv_rms
// -> (out, normed or None)
PyObject* block_residual(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!arity(n, 13)) return nullptr;
  return guarded([&]() -> PyObject* {
    const Tensor& x = tensor(v[0]);
    Call c;
    if (!begin(c, "flashnorm_block_residual", x)) Py_RETURN_NONE;
    const int64_t M = x.size(0), K = x.size(1), rows_per_gate = integer(v[5]);
    const Matrix X = matrix(c, &x, M, K, "x"), H = matrix(c, &tensor(v[1]), M, K, "h");
    const float* g_post = vector(c, tensor_or_none(v[2]), K, "g_post");
    const Matrix G = gate_of(c, tensor_or_none(v[4]), rows_per_gate, M, K);
    const float* g_pre = vector(c, tensor_or_none(v[8]), K, "g_pre");
    const Tensor *out = tensor_or_none(v[10]), *normed = tensor_or_none(v[11]);
    if (normed && !g_pre) c.refuse("normed needs g_pre");
    float* inv_rms = vector(c, tensor_or_none(v[12]), M, "inv_rms");
    const Tensor made = out ? Tensor() : new_matrix(c, M, K);
    const Tensor made_n = normed || !g_pre ? Tensor() : new_matrix(c, M, K);
    const Matrix O = matrix(c, out ? out : &made, M, K, "out");
    const Matrix NO = matrix(c, normed ? normed : made_n.defined() ? &made_n : nullptr, M, K, "normed");
    const int s = flashnorm_block_residual(X.p, X.ld, H.p, H.ld, M, K, c.code, g_post, real(v[3]), G.p, G.ld, rows_per_gate,
                                           real(v[6]), real(v[7]), g_pre, real(v[9]), O.p, O.ld, NO.p, NO.ld, inv_rms,
                                           stream_of(c));
    if (s) return PyLong_FromLong(s);
    written({out, normed, tensor_or_none(v[12])});
    PyObject* first = out ? again(v[10]) : wrap(made);
    PyObject* second = normed ? again(v[11]) : wrap(made_n);
    PyObject* both = first && second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_XDECREF(first);
    Py_XDECREF(second);
    return both;
  });
}

// x, h, dh_out, dn, g_post, eps_post, gate, rows_per_gate, res_scale, branch_scale, g_pre, eps_pre, workspace
// -> (dx, dh, dgate, dg_post, dg_pre), None for what the call has not
PyObject* block_residual_bwd(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (!arity(n, 13)) return nullptr;
  return guarded([&]() -> PyObject* {
    const Tensor& x = tensor(v[0]);
    Call c;
    if (!begin(c, "flashnorm_block_residual_bwd", x)) Py_RETURN_NONE;
    const int64_t M = x.size(0), K = x.size(1), rows_per_gate = integer(v[7]);
    const Tensor* gate = tensor_or_none(v[6]);
    const Matrix X = matrix(c, &x, M, K, "x"), H = matrix(c, &tensor(v[1]), M, K, "h");
    const Matrix DO = matrix(c, tensor_or_none(v[2]), M, K, "dh_out"), DN = matrix(c, tensor_or_none(v[3]), M, K, "dn");
    const float* g_post = vector(c, tensor_or_none(v[4]), K, "g_post");
    const float* g_pre = vector(c, tensor_or_none(v[10]), K, "g_pre");
    const Matrix G = gate_of(c, gate, rows_per_gate, M, K);
    const size_t need = flashnorm_block_residual_bwd_size(M, K, gate ? rows_per_gate : 0, c.code);
    const Tensor ws = workspace(c, tensor_or_none(v[12]), need);
    const Tensor dx = new_matrix(c, M, K), dh = new_matrix(c, M, K);
    const Tensor dgate = gate ? new_matrix(c, gate->size(0), K) : Tensor();
    const Tensor dpost = g_post ? new_tensor(c, {K}, at::kFloat) : Tensor();
    const Tensor dpre = g_pre ? new_tensor(c, {K}, at::kFloat) : Tensor();
    const Matrix DX = matrix(c, &dx, M, K, "dx"), DH = matrix(c, &dh, M, K, "dh");
    const Matrix DG = gate ? matrix(c, &dgate, gate->size(0), K, "dgate") : Matrix{};
    const int s = flashnorm_block_residual_bwd(
        X.p, X.ld, H.p, H.ld, DO.p, DO.ld, DN.p, DN.ld, M, K, c.code, g_post, real(v[5]), G.p, G.ld, rows_per_gate, real(v[8]),
        real(v[9]), g_pre, real(v[11]), DX.p, DX.ld, DH.p, DH.ld, DG.p, DG.ld, static_cast<float*>(address(dpost)),
        static_cast<float*>(address(dpre)), address(ws), need, stream_of(c));
    if (s) return PyLong_FromLong(s);
    written({need ? tensor_or_none(v[12]) : nullptr});
    PyObject* parts[] = {wrap(dx), wrap(dh), wrap(dgate), wrap(dpost), wrap(dpre)};
    bool whole = true;
    for (PyObject* p : parts) whole = whole && p;
    PyObject* all = whole ? PyTuple_Pack(5, parts[0], parts[1], parts[2], parts[3], parts[4]) : nullptr;
    for (PyObject* p : parts) Py_XDECREF(p);
    return all;
  });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef kMethods[] = {method<w4_fold>("w4_fold"),
                          method<w4_unpack>("w4_unpack"),
                          method<w4_product>("w4_product"),
                          method<block_residual>("block_residual"),
                          method<block_residual_bwd>("block_residual_bwd"),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&kModule); }
