// The marshalling of binding.gdn_forward, of the linear attention and of the RMS norm in native code: shape checks, the outputs, the workspace and the call, for the ordinary case of
// plain contiguous CUDA tensors on the current stream.  Whatever else comes (other types, other devices, arguments that convert) makes a function return None, and the
// Python body of the binding's function takes the call, with its conversions and its errors.
//
// A decode step is one kernel of 5.7 us; eight data pointers, a descriptor, two allocations and two calls through ctypes took 12.9 us of host time for it; a token of linear
// attention is one of 4 us (13.4 us through ctypes), an RMS norm of a few rows one of 2.5 us (13.7).
#include <torch/extension.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <c10/cuda/CUDAStream.h>

#include <climits>
#include <vector>

#include "tri_inv.h"

namespace {

using WorkspaceFn = int (*)(const tri_inv_desc*, int, size_t*);
using ForwardFn = int (*)(const void*, const void*, const void*, const float*, const float*, const float*, void*, float*, float, void*, size_t,
                          const tri_inv_desc*, int, void*);
WorkspaceFn g_workspace = nullptr;
ForwardFn g_forward = nullptr;

PyObject* bind(PyObject*, PyObject* args) {   // the addresses of tri_inv_gdn_forward_workspace and tri_inv_gdn_forward in the loaded library
  unsigned long long w = 0, f = 0;
  if (!PyArg_ParseTuple(args, "KK", &w, &f)) return nullptr;
  g_workspace = reinterpret_cast<WorkspaceFn>(w);
  g_forward = reinterpret_cast<ForwardFn>(f);
  Py_RETURN_NONE;
}

bool plain(PyObject* o, int dims) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() && t.layout() == at::kStrided && t.is_contiguous() && (dims == 0 || t.dim() == dims);
}
bool whole(PyObject* o, long lo, long hi, long* out) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  *out = PyLong_AsLongAndOverflow(o, &over);
  return !over && *out >= lo && *out <= hi;
}

// (Q, K, V, beta, g, C, scale, S0, method, cu_seqlens) -> (O, S), None (not an ordinary call), or the failing call's status (+ 256: the workspace query's)
PyObject* gdn_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  long C = 0, method = 0;
  if (n != 10 || !g_forward || !plain(a[0], 0) || !plain(a[1], 4) || !plain(a[2], 4) || !plain(a[3], 0) || !plain(a[4], 0) || !whole(a[5], INT_MIN, INT_MAX, &C) ||
      !PyFloat_CheckExact(a[6]) || !(a[7] == Py_None || plain(a[7], 0)) || !whole(a[8], INT_MIN, INT_MAX, &method))
    Py_RETURN_NONE;
  const at::Tensor &Q = THPVariable_Unpack(a[0]), &K = THPVariable_Unpack(a[1]), &V = THPVariable_Unpack(a[2]), &beta = THPVariable_Unpack(a[3]), &g = THPVariable_Unpack(a[4]);
  const bool f32 = K.scalar_type() == at::kFloat;
  if (!f32 && K.scalar_type() != at::kBFloat16) Py_RETURN_NONE;
  for (int i = 0; i < 4; ++i)
    if (K.size(i) > INT_MAX || V.size(i) > INT_MAX) Py_RETURN_NONE;
  tri_inv_desc d{};
  d.B = (int32_t)K.size(0); d.T = (int32_t)K.size(1); d.H = (int32_t)K.size(2); d.d_k = (int32_t)K.size(3); d.d_v = (int32_t)V.size(3);
  d.C = (int32_t)C;
  d.kv_dtype = f32 ? TRI_INV_F32 : TRI_INV_BF16;
  int64_t n_seqs = d.B;
  std::vector<int32_t> cu;
  if (a[9] != Py_None) {
    const bool list = PyList_CheckExact(a[9]);
    if (!list && !PyTuple_CheckExact(a[9])) Py_RETURN_NONE;
    const Py_ssize_t m = list ? PyList_GET_SIZE(a[9]) : PyTuple_GET_SIZE(a[9]);
    if (m < 1 || m > INT_MAX) Py_RETURN_NONE;
    cu.resize(m);
    for (Py_ssize_t i = 0; i < m; ++i) {
      long x = 0;
      if (!whole(list ? PyList_GET_ITEM(a[9], i) : PyTuple_GET_ITEM(a[9], i), INT_MIN, INT_MAX, &x)) Py_RETURN_NONE;
      cu[i] = (int32_t)x;
    }
    d.cu_seqlens = cu.data();
    d.n_seqs = (int32_t)(m - 1);
    n_seqs = m - 1;
  }
  size_t need = 0;
  int rc = g_workspace(&d, (int)method, &need);
  if (rc) return PyLong_FromLong(rc + 256);
  at::Tensor O = at::empty_like(V), S = at::empty({n_seqs, d.H, d.d_k, d.d_v}, K.options().dtype(at::kFloat)), work;
  if (need) work = at::empty({(int64_t)need}, K.options().dtype(at::kByte));
  const float* S0 = a[7] == Py_None ? nullptr : (const float*)THPVariable_Unpack(a[7]).data_ptr();
  const void *q = Q.data_ptr(), *k = K.data_ptr(), *v = V.data_ptr();
  const float *b = (const float*)beta.data_ptr(), *gg = (const float*)g.data_ptr();
  void *o = O.data_ptr(), *s = S.data_ptr(), *w = need ? work.data_ptr() : nullptr;
  void* stream = c10::cuda::getCurrentCUDAStream().stream();
  const float scale = (float)PyFloat_AS_DOUBLE(a[6]);
  Py_BEGIN_ALLOW_THREADS
  rc = g_forward(q, k, v, b, gg, S0, o, (float*)s, scale, w, need, &d, (int)method, stream);
  Py_END_ALLOW_THREADS
  if (rc) return PyLong_FromLong(rc);
  PyObject* out = PyTuple_New(2);
  if (!out) return nullptr;
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(O)));
  PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(std::move(S)));
  return out;
  END_HANDLE_TH_ERRORS
}

// ---- linear attention and RMS norm

using BytesFn = int (*)(const tri_inv_desc*, size_t*);
using AttentionFn = int (*)(const void*, const void*, const void*, const float*, const float*, void*, float*, float, void*, size_t, const tri_inv_desc*, void*);
using AttentionBackFn = int (*)(const void*, const void*, const void*, const void*, const float*, const float*, const float*, void*, void*, void*, float*, float, void*, size_t,
                                const tri_inv_desc*, void*);
using StepFn = int (*)(const void*, const void*, const void*, const float*, float*, const int32_t*, int32_t, void*, float, const tri_inv_desc*, void*);
using NormFn = int (*)(const void*, const void*, const void*, void*, void*, float*, int64_t, int32_t, int32_t, float, int, int, void*);
using NormBytesFn = int (*)(int64_t, int32_t, size_t*);
using NormBackFn = int (*)(const void*, const void*, const void*, const void*, void*, void*, int64_t, int32_t, float, int, void*, size_t, void*);
struct { BytesFn bytes; AttentionFn attention; BytesFn back_bytes; AttentionBackFn back; StepFn step; NormFn norm; NormBytesFn norm_bytes; NormBackFn norm_back; } g_ops = {};

PyObject* bind_operators(PyObject*, PyObject* args) {   // the addresses of the entry points above, in this order
  unsigned long long f[8];
  if (!PyArg_ParseTuple(args, "KKKKKKKK", f, f + 1, f + 2, f + 3, f + 4, f + 5, f + 6, f + 7)) return nullptr;
  g_ops = {(BytesFn)f[0], (AttentionFn)f[1], (BytesFn)f[2], (AttentionBackFn)f[3], (StepFn)f[4], (NormFn)f[5], (NormBytesFn)f[6], (NormBackFn)f[7]};
  Py_RETURN_NONE;
}

bool on_current_device(const at::Tensor& t) { return t.get_device() == c10::cuda::current_device(); }
// Whether `o` is a plain contiguous tensor of this type and shape on the current device (or, where that is allowed, None).
bool is(PyObject* o, at::ScalarType type, at::IntArrayRef shape, bool or_none = false) {
  if (o == Py_None) return or_none;
  if (!plain(o, 0)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.scalar_type() == type && t.sizes() == shape && on_current_device(t);
}
void* data(PyObject* o) { return o == Py_None ? nullptr : THPVariable_Unpack(o).data_ptr(); }
bool stored(const at::Tensor& t, int32_t* code) {
  *code = t.scalar_type() == at::kFloat ? TRI_INV_F32 : TRI_INV_BF16;
  return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16;
}
bool offsets(PyObject* o, std::vector<int32_t>* cu) {   // of a list or tuple of whole numbers
  const bool list = PyList_CheckExact(o);
  if (!list && !PyTuple_CheckExact(o)) return false;
  const Py_ssize_t m = list ? PyList_GET_SIZE(o) : PyTuple_GET_SIZE(o);
  if (m < 1 || m > INT_MAX) return false;
  cu->resize(m);
  for (Py_ssize_t i = 0; i < m; ++i) {
    long x = 0;
    if (!whole(list ? PyList_GET_ITEM(o, i) : PyTuple_GET_ITEM(o, i), INT_MIN, INT_MAX, &x)) return false;
    (*cu)[i] = (int32_t)x;
  }
  return true;
}
PyObject* tuple_of(std::initializer_list<at::Tensor> ts) {   // None for one that is not defined
  PyObject* out = PyTuple_New(ts.size());
  if (!out) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor& t : ts) {
    PyObject* o = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
    if (!o) { Py_DECREF(out); return nullptr; }
    PyTuple_SET_ITEM(out, i++, o);
  }
  return out;
}
void* current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// Q, K, V [B,T,H,d] and log_decay in a[0 .. 3], cu_seqlens: the descriptor and the shapes, or false
struct Attention {
  tri_inv_desc d{};
  std::vector<int32_t> cu;
  std::vector<int64_t> qk, vo, state;
  at::ScalarType type;
  bool take(PyObject* Q, PyObject* K, PyObject* V, PyObject* ld, PyObject* cu_seqlens) {
    if (!plain(Q, 4) || !plain(V, 4)) return false;
    const at::Tensor &q = THPVariable_Unpack(Q), &v = THPVariable_Unpack(V);
    if (!stored(q, &d.kv_dtype)) return false;
    type = q.scalar_type();
    qk = q.sizes().vec();
    vo = {qk[0], qk[1], qk[2], v.size(3)};
    for (int i = 0; i < 4; ++i)
      if (qk[i] > INT_MAX || vo[i] > INT_MAX) return false;
    d.B = (int32_t)qk[0]; d.T = (int32_t)qk[1]; d.H = (int32_t)qk[2]; d.d_k = (int32_t)qk[3]; d.d_v = (int32_t)vo[3]; d.C = 64;
    int64_t n = qk[0];
    if (cu_seqlens != Py_None) {
      if (!offsets(cu_seqlens, &cu)) return false;
      d.cu_seqlens = cu.data();
      d.n_seqs = (int32_t)cu.size() - 1;
      n = d.n_seqs;
    }
    state = {n, qk[2], qk[3], vo[3]};
    return is(Q, type, qk) && is(K, type, qk) && is(V, type, vo) && is(ld, at::kFloat, {qk[2]});
  }
};

// (Q, K, V, log_decay, scale, S0, cu_seqlens, want_state) -> (O, S or None), None, or the failing call's status (+ 256: the workspace query's)
PyObject* linear_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Attention x;
  if (n != 8 || !g_ops.attention || !PyFloat_CheckExact(a[4]) || !x.take(a[0], a[1], a[2], a[3], a[6]) || !is(a[5], at::kFloat, x.state, true)) Py_RETURN_NONE;
  size_t need = 0;
  int rc = g_ops.bytes(&x.d, &need);
  if (rc) return PyLong_FromLong(rc + 256);
  const at::Tensor& V = THPVariable_Unpack(a[2]);
  at::Tensor O = at::empty_like(V), S, work;
  if (a[7] == Py_True) S = at::empty(x.state, V.options().dtype(at::kFloat));
  if (need) work = at::empty({(int64_t)need}, V.options().dtype(at::kByte));
  void *q = data(a[0]), *k = data(a[1]), *v = data(a[2]), *ld = data(a[3]), *s0 = data(a[5]), *o = O.data_ptr(), *s = S.defined() ? S.data_ptr() : nullptr,
       *w = need ? work.data_ptr() : nullptr, *stream = current_stream();
  const float scale = (float)PyFloat_AS_DOUBLE(a[4]);
  Py_BEGIN_ALLOW_THREADS
  rc = g_ops.attention(q, k, v, (float*)ld, (float*)s0, o, (float*)s, scale, w, need, &x.d, stream);
  Py_END_ALLOW_THREADS
  return rc ? PyLong_FromLong(rc) : tuple_of({O, S});
  END_HANDLE_TH_ERRORS
}

// (dO, Q, K, V, log_decay, scale, S0, dS, cu_seqlens, want_dS0) -> (dQ, dK, dV, dS0 or None), None, or a status as above
PyObject* linear_attention_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Attention x;
  if (n != 10 || !g_ops.back || !PyFloat_CheckExact(a[5]) || !x.take(a[1], a[2], a[3], a[4], a[8]) || !is(a[0], x.type, x.vo) || !is(a[6], at::kFloat, x.state, true) ||
      !is(a[7], at::kFloat, x.state, true))
    Py_RETURN_NONE;
  size_t need = 0;
  int rc = g_ops.back_bytes(&x.d, &need);
  if (rc) return PyLong_FromLong(rc + 256);
  const at::Tensor &Q = THPVariable_Unpack(a[1]), &V = THPVariable_Unpack(a[3]);
  at::Tensor dQ = at::empty_like(Q), dK = at::empty_like(Q), dV = at::empty_like(V), dS0, work;
  if (a[9] == Py_True) dS0 = at::empty(x.state, V.options().dtype(at::kFloat));
  if (need) work = at::empty({(int64_t)need}, V.options().dtype(at::kByte));
  void *p[7], *stream = current_stream(), *w = need ? work.data_ptr() : nullptr, *gq = dQ.data_ptr(), *gk = dK.data_ptr(), *gv = dV.data_ptr(), *gs = dS0.defined() ? dS0.data_ptr() : nullptr;
  for (int i = 0; i < 5; ++i) p[i] = data(a[i]);
  p[5] = data(a[6]); p[6] = data(a[7]);
  const float scale = (float)PyFloat_AS_DOUBLE(a[5]);
  Py_BEGIN_ALLOW_THREADS
  rc = g_ops.back(p[0], p[1], p[2], p[3], (float*)p[4], (float*)p[5], (float*)p[6], gq, gk, gv, (float*)gs, scale, w, need, &x.d, stream);
  Py_END_ALLOW_THREADS
  return rc ? PyLong_FromLong(rc) : tuple_of({dQ, dK, dV, dS0});
  END_HANDLE_TH_ERRORS
}

// (Q, K, V, log_decay, S, scale, slots) -> O, None, or a status
PyObject* linear_attention_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7 || !g_ops.step || !PyFloat_CheckExact(a[5]) || !plain(a[0], 3) || !plain(a[2], 3) || !plain(a[4], 4)) Py_RETURN_NONE;
  const at::Tensor &Q = THPVariable_Unpack(a[0]), &V = THPVariable_Unpack(a[2]), &S = THPVariable_Unpack(a[4]);
  tri_inv_desc d{};
  const int64_t B = Q.size(0), H = Q.size(1), dk = Q.size(2), dv = V.size(2), slots = S.size(0);
  if (!stored(Q, &d.kv_dtype) || B < 1 || B > INT_MAX || H > INT_MAX || dk > INT_MAX || dv > INT_MAX || slots > INT_MAX) Py_RETURN_NONE;
  const at::ScalarType type = Q.scalar_type();
  if (!is(a[0], type, {B, H, dk}) || !is(a[1], type, {B, H, dk}) || !is(a[2], type, {B, H, dv}) || !is(a[3], at::kFloat, {H}) || !is(a[4], at::kFloat, {slots, H, dk, dv}) ||
      !is(a[6], at::kInt, {B}, true))
    Py_RETURN_NONE;
  d.B = (int32_t)B; d.T = 1; d.H = (int32_t)H; d.d_k = (int32_t)dk; d.d_v = (int32_t)dv; d.C = 64;
  at::Tensor O = at::empty_like(V);
  const int rc = g_ops.step(data(a[0]), data(a[1]), data(a[2]), (float*)data(a[3]), (float*)data(a[4]), (int32_t*)data(a[6]), (int32_t)slots, O.data_ptr(),
                            (float)PyFloat_AS_DOUBLE(a[5]), &d, current_stream());
  return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(O);
  END_HANDLE_TH_ERRORS
}

// Rows and columns of X (the last dimension), or false
bool rows_of(PyObject* X, int64_t* rows, int64_t* n, int32_t* code) {
  if (!plain(X, 0)) return false;
  const at::Tensor& x = THPVariable_Unpack(X);
  if (x.dim() < 1 || !stored(x, code) || !on_current_device(x)) return false;
  *n = x.size(-1);
  if (*n < 1 || *n > INT_MAX) return false;
  *rows = x.numel() / *n;
  return true;
}

// (X, w, eps, residual, coded, group) -> (Y, H or None, scales or None), None, or a status
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  int64_t rows, n;
  int32_t code;
  long group = 0;
  if (n_args != 6 || !g_ops.norm || !PyFloat_CheckExact(a[2]) || !whole(a[5], 0, INT_MAX, &group) || !rows_of(a[0], &rows, &n, &code)) Py_RETURN_NONE;
  const at::Tensor& X = THPVariable_Unpack(a[0]);
  if (!is(a[1], X.scalar_type(), {n}) || !is(a[3], X.scalar_type(), X.sizes(), true)) Py_RETURN_NONE;
  const bool coded = a[4] == Py_True;
  at::Tensor Y = coded ? at::empty(X.sizes(), X.options().dtype(at::kFloat8_e4m3fn)) : at::empty_like(X), H, scales;
  if (a[3] != Py_None) H = at::empty_like(X);
  if (coded) {
    std::vector<int64_t> shape = X.sizes().vec();
    shape.back() = group ? (n + 127) / 128 : 1;
    scales = at::empty(shape, X.options().dtype(at::kFloat));
  }
  const int rc = g_ops.norm(X.data_ptr(), data(a[3]), data(a[1]), Y.data_ptr(), H.defined() ? H.data_ptr() : nullptr, coded ? scales.data_ptr<float>() : nullptr, rows, (int32_t)n,
                            (int32_t)group, (float)PyFloat_AS_DOUBLE(a[2]), code, coded ? TRI_INV_E4M3 : code, current_stream());
  return rc ? PyLong_FromLong(rc) : tuple_of({Y, H, scales});
  END_HANDLE_TH_ERRORS
}

// (dY, X, w, eps, dH) -> (dX, dw), None, or a status
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  int64_t rows, n;
  int32_t code;
  if (n_args != 5 || !g_ops.norm_back || !PyFloat_CheckExact(a[3]) || !rows_of(a[1], &rows, &n, &code)) Py_RETURN_NONE;
  const at::Tensor& X = THPVariable_Unpack(a[1]);
  if (!is(a[0], X.scalar_type(), X.sizes()) || !is(a[2], X.scalar_type(), {n}) || !is(a[4], X.scalar_type(), X.sizes(), true)) Py_RETURN_NONE;
  size_t need = 0;
  int rc = g_ops.norm_bytes(rows, (int32_t)n, &need);
  if (rc) return PyLong_FromLong(rc + 256);
  at::Tensor dX = at::empty_like(X), dw = at::empty({n}, X.options()), work = at::empty({(int64_t)need}, X.options().dtype(at::kByte));
  rc = g_ops.norm_back(data(a[0]), X.data_ptr(), data(a[2]), data(a[4]), dX.data_ptr(), dw.data_ptr(), rows, (int32_t)n, (float)PyFloat_AS_DOUBLE(a[3]), code, work.data_ptr(), need,
                       current_stream());
  return rc ? PyLong_FromLong(rc) : tuple_of({dX, dw});
  END_HANDLE_TH_ERRORS
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         {"gdn_forward", (PyCFunction)(void (*)(void))gdn_forward, METH_FASTCALL, nullptr},
                         {"bind_operators", bind_operators, METH_VARARGS, nullptr},
                         FAST(linear_attention), FAST(linear_attention_backward), FAST(linear_attention_step), FAST(rms_norm), FAST(rms_norm_backward),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
