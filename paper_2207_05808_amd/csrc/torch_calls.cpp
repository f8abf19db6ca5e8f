// One call of a fused entry point on torch tensors, marshalled natively.
//
// The Python binding checks every argument attribute by attribute and builds
// the argument list through ctypes, about 14 us of host time per call, more
// than twice the kernel time of the small layers (1024 x 64 -> 10, C 4:
// 14.8 -> 5.1 us a call).  `fused(...)` does the same for the
// plain valid case only (exact torch.Tensor arguments, device memory, the
// documented dtypes and shapes, dense outputs) and returns None for anything
// else, an error included: the binding then takes its own path, which raises
// what it always raised.  No arithmetic of the method happens here.
//
// The library's functions come in as addresses (`init`), from the library the
// ctypes binding has loaded: there is one copy of it in the process.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdint.h>

namespace {

typedef int (*MatmulFn)(const float*, int64_t, int32_t, int64_t, const int32_t*, const float*, int32_t, const int8_t*,
                        const float*, const float*, int32_t, float*, int32_t*, uint8_t*, void*);
typedef int (*MatmulF32Fn)(const float*, int64_t, int32_t, int64_t, const int32_t*, const float*, int32_t, const float*,
                           int32_t, float*, uint8_t*, void*);
typedef int (*ActFn)(const float*, int64_t, int32_t, int64_t, const int32_t*, const float*, int32_t, const int8_t*,
                     const float*, const float*, int32_t, const float*, int32_t, float*, uint8_t*, void*);
typedef int (*ActF32Fn)(const float*, int64_t, int32_t, int64_t, const int32_t*, const float*, int32_t, const float*,
                        int32_t, const float*, int32_t, float*, uint8_t*, void*);
typedef int64_t (*IndexBytesFn)(const float*, int64_t, int32_t, int64_t, int32_t, int32_t, int32_t, int32_t);

// the output layer's
typedef int (*W4Fn)(const void*, int32_t, int64_t, int32_t, int64_t, const uint8_t*, const uint8_t*, int32_t, const float*,
                    int32_t, void*, int32_t, void*, int64_t, void*);
typedef int64_t (*W4BytesFn)(const void*, int32_t, int64_t, int32_t, int64_t, int32_t);
typedef int (*QuantizeFn)(const void*, int32_t, int32_t, int32_t, int64_t, int64_t, uint8_t*, uint8_t*, void*);
typedef int (*DequantizeFn)(const uint8_t*, const uint8_t*, int32_t, int32_t, void*, int32_t, void*);
typedef int64_t (*XentBytesFn)(int64_t, int32_t, int32_t, int32_t);
typedef int (*XentFn)(const void*, int32_t, int64_t, int32_t, int64_t, const void*, int32_t, int32_t, const float*,
                      const int64_t*, float*, float*, void*, int64_t, void*);
typedef int (*XentGradFn)(const void*, int32_t, int64_t, int32_t, int64_t, const void*, int32_t, int32_t, const float*,
                          const int64_t*, const float*, const float*, void*, void*, float*, void*, int64_t, void*);

W4Fn g_w4;
W4BytesFn g_w4_bytes;
QuantizeFn g_quantize;
DequantizeFn g_dequantize;
XentBytesFn g_xent_bytes, g_xent_grad_bytes;
XentFn g_xent;
XentGradFn g_xent_grad;

MatmulFn g_matmul;
MatmulF32Fn g_matmul_f32;
ActFn g_act;
ActF32Fn g_act_f32;
IndexBytesFn g_index_bytes;

PyObject* init(PyObject*, PyObject* args) {
  unsigned long long a, b, c, d, e, f, g, h, i, j, k, l, m;
  if (!PyArg_ParseTuple(args, "KKKKKKKKKKKKK", &a, &b, &c, &d, &e, &f, &g, &h, &i, &j, &k, &l, &m)) return nullptr;
  g_w4 = reinterpret_cast<W4Fn>(f);
  g_w4_bytes = reinterpret_cast<W4BytesFn>(g);
  g_quantize = reinterpret_cast<QuantizeFn>(h);
  g_dequantize = reinterpret_cast<DequantizeFn>(i);
  g_xent_bytes = reinterpret_cast<XentBytesFn>(j);
  g_xent = reinterpret_cast<XentFn>(k);
  g_xent_grad_bytes = reinterpret_cast<XentBytesFn>(l);
  g_xent_grad = reinterpret_cast<XentGradFn>(m);
  g_matmul = reinterpret_cast<MatmulFn>(a);
  g_matmul_f32 = reinterpret_cast<MatmulF32Fn>(b);
  g_act = reinterpret_cast<ActFn>(c);
  g_act_f32 = reinterpret_cast<ActF32Fn>(d);
  g_index_bytes = reinterpret_cast<IndexBytesFn>(e);
  Py_RETURN_NONE;
}

// the tensor behind an exact torch.Tensor (no subclass) in device memory of
// this type and rank; nullptr otherwise
const at::Tensor* plain(PyObject* o, at::ScalarType type, int64_t dim) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.scalar_type() != type || t.dim() != dim ||
      !t.has_storage())
    return nullptr;
  return &t;
}
const at::Tensor* dense(PyObject* o, at::ScalarType type, int64_t dim) {
  const at::Tensor* t = plain(o, type, dim);
  return t && t->is_contiguous() ? t : nullptr;
}

// fused(A, split, thr, lut, scale, offset, col_bias, act, y_out, acc_out,
// idx_out, want_acc, want_idx, stream) -> (y, acc, idx) or None.  scale and
// offset None: an fp32 table.  act None: the entry points without a layer
// output.
PyObject* fused(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 14 || !g_matmul) Py_RETURN_NONE;
  try {
    const bool f32 = a[4] == Py_None && a[5] == Py_None;
    const at::Tensor* A = plain(a[0], at::kFloat, 2);
    const at::Tensor* split = dense(a[1], at::kInt, 2);
    const at::Tensor* thr = dense(a[2], at::kFloat, 2);
    const at::Tensor* lut = dense(a[3], f32 ? at::kFloat : at::kChar, 3);
    if (!A || !split || !thr || !lut) Py_RETURN_NONE;
    const int64_t N = A->size(0), D = A->size(1), C = split->size(0), M = lut->size(2);
    if (N > 1 && A->stride(1) != 1) Py_RETURN_NONE;
    const int64_t lda = N > 1 ? A->stride(0) : D;
    if (split->size(1) != 4 || thr->size(0) != C || thr->size(1) != 15 || lut->size(0) != C || lut->size(1) != 16)
      Py_RETURN_NONE;
    if (N <= 0 || D <= 0 || C <= 0 || M <= 0 || lda < D || D > INT32_MAX || C > INT32_MAX || M > INT32_MAX)
      Py_RETURN_NONE;
    const at::Tensor *scale = nullptr, *offset = nullptr, *bias = nullptr;
    if (!f32) {
      scale = dense(a[4], at::kFloat, 1);
      offset = dense(a[5], at::kFloat, 1);
      if (!scale || !offset || scale->size(0) != C || offset->size(0) != C) Py_RETURN_NONE;
    }
    if (a[6] != Py_None) {
      bias = dense(a[6], at::kFloat, 1);
      if (!bias || bias->size(0) != M) Py_RETURN_NONE;
    }
    const long act = a[7] == Py_None ? -1 : PyLong_AsLong(a[7]);
    // other truth values (1, a numpy bool) are the binding's to judge
    for (int i = 11; i <= 12; ++i)
      if (a[i] != Py_True && a[i] != Py_False) Py_RETURN_NONE;
    const bool want_acc = a[11] == Py_True, want_idx = a[12] == Py_True;
    void* stream = PyLong_AsVoidPtr(a[13]);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    if (act > 3 || (act < 0 && a[7] != Py_None)) Py_RETURN_NONE;
    // outputs: the caller's, when they are what a new one would be, else new
    // (checked before any is allocated)
    const at::Tensor *y_in = nullptr, *acc_in = nullptr, *idx_in = nullptr;
    if (a[8] != Py_None && !((y_in = dense(a[8], at::kFloat, 2)) && y_in->size(0) == N && y_in->size(1) == M))
      Py_RETURN_NONE;
    if (a[9] != Py_None && !((acc_in = dense(a[9], at::kInt, 2)) && acc_in->size(0) == N && acc_in->size(1) == M))
      Py_RETURN_NONE;
    if (a[10] != Py_None && !((idx_in = dense(a[10], at::kByte, 2)) && idx_in->size(0) == N && idx_in->size(1) == C))
      Py_RETURN_NONE;
    const auto opt = A->options().requires_grad(false);
    at::Tensor y = y_in ? *y_in : at::empty({N, M}, opt);
    at::Tensor acc, idx, scratch;
    if (acc_in) acc = *acc_in;
    else if (want_acc) acc = at::empty({N, M}, opt.dtype(at::kInt));
    if (idx_in) idx = *idx_in;
    else if (want_idx) idx = at::empty({N, C}, opt.dtype(at::kByte));
    const float* pA = static_cast<const float*>(A->const_data_ptr());
    if (!idx.defined() && g_index_bytes(pA, N, (int32_t)D, lda, (int32_t)C, (int32_t)M, f32, act < 0 ? 0 : (int32_t)act) > 0)
      scratch = at::empty({N, C}, opt.dtype(at::kByte));
    uint8_t* pi = idx.defined()       ? static_cast<uint8_t*>(idx.mutable_data_ptr())
                  : scratch.defined() ? static_cast<uint8_t*>(scratch.mutable_data_ptr())
                                      : nullptr;
    const int32_t* ps = static_cast<const int32_t*>(split->const_data_ptr());
    const float* pt = static_cast<const float*>(thr->const_data_ptr());
    const void* pl = lut->const_data_ptr();
    const float* psc = scale ? static_cast<const float*>(scale->const_data_ptr()) : nullptr;
    const float* pof = offset ? static_cast<const float*>(offset->const_data_ptr()) : nullptr;
    const float* pb = bias ? static_cast<const float*>(bias->const_data_ptr()) : nullptr;
    float* py = static_cast<float*>(y.mutable_data_ptr());
    int32_t* pacc = acc.defined() ? static_cast<int32_t*>(acc.mutable_data_ptr()) : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    if (act < 0)
      rc = f32 ? g_matmul_f32(pA, N, (int32_t)D, lda, ps, pt, (int32_t)C, static_cast<const float*>(pl), (int32_t)M, py, pi,
                              stream)
               : g_matmul(pA, N, (int32_t)D, lda, ps, pt, (int32_t)C, static_cast<const int8_t*>(pl), psc, pof, (int32_t)M,
                          py, pacc, pi, stream);
    else
      rc = f32 ? g_act_f32(pA, N, (int32_t)D, lda, ps, pt, (int32_t)C, static_cast<const float*>(pl), (int32_t)M, pb,
                           (int32_t)act, py, pi, stream)
               : g_act(pA, N, (int32_t)D, lda, ps, pt, (int32_t)C, static_cast<const int8_t*>(pl), psc, pof, (int32_t)M, pb,
                       (int32_t)act, py, pi, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) Py_RETURN_NONE;
    auto out = [](PyObject* given, const at::Tensor& t) -> PyObject* {
      if (given != Py_None) {
        Py_INCREF(given);
        return given;
      }
      if (!t.defined()) Py_RETURN_NONE;
      return THPVariable_Wrap(t);
    };
    PyObject* r = PyTuple_New(3);
    if (!r) return nullptr;
    PyTuple_SET_ITEM(r, 0, out(a[8], y));
    PyTuple_SET_ITEM(r, 1, out(a[9], acc));
    PyTuple_SET_ITEM(r, 2, out(a[10], idx));
    for (int i = 0; i < 3; ++i)
      if (!PyTuple_GET_ITEM(r, i)) {
        Py_DECREF(r);
        return nullptr;
      }
    return r;
  } catch (...) {   // (a tensor without plain memory, out of device memory, ...): the binding's own path says what
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// ------------------------------------------------- the output layer's calls
// As `fused`: the plain valid case on the current device, new outputs and
// workspaces; None for anything else.  Arguments end in the current device's
// index and its current stream.

// a plain floating tensor of one of the ABI's types and its code
const at::Tensor* typed(PyObject* o, int64_t dim, int32_t& code) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.dim() != dim || !t.has_storage()) return nullptr;
  const auto s = t.scalar_type();
  if (s == at::kFloat) code = 0;
  else if (s == at::kBFloat16) code = 1;
  else if (s == at::kHalf) code = 2;
  else return nullptr;
  return &t;
}
at::ScalarType type_of(int32_t code) { return code == 0 ? at::kFloat : code == 1 ? at::kBFloat16 : at::kHalf; }

// an optional dense vector of M floats: false when it is something else
bool vector_or_none(PyObject* o, int64_t M, const at::Tensor*& t) {
  t = nullptr;
  if (o == Py_None) return true;
  t = dense(o, at::kFloat, 1);
  return t && t->size(0) == M;
}

bool on(const at::Tensor* t, int64_t device) { return !t || t->get_device() == device; }

// elements between A's rows, or -1
int64_t row_stride(const at::Tensor& A) {
  const int64_t N = A.size(0), D = A.size(1);
  if (N < 1 || D < 1 || D > INT32_MAX || (D > 1 && A.stride(1) != 1)) return -1;
  if (N == 1) return D;
  return A.stride(0) < D ? -1 : A.stride(0);
}

bool tail(PyObject* device, PyObject* stream, int64_t& d, void*& s) {
  d = PyLong_AsLongLong(device);
  s = PyLong_AsVoidPtr(stream);
  if (!PyErr_Occurred()) return true;
  PyErr_Clear();
  return false;
}

at::Tensor scratch_of(const at::Tensor& like, int64_t bytes) {
  return bytes > 0 ? at::empty({bytes}, like.options().dtype(at::kByte).requires_grad(false)) : at::Tensor();
}
void* pointer(const at::Tensor& t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }
bool aligned256(const at::Tensor& t) { return !t.defined() || (reinterpret_cast<uintptr_t>(t.const_data_ptr()) & 255) == 0; }

PyObject* pack(std::initializer_list<at::Tensor> ts) {
  PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
  if (!r) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor& t : ts) {
    PyObject* o = THPVariable_Wrap(t);
    if (!o) {
      Py_DECREF(r);
      return nullptr;
    }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

// w4(A, codes, exps, D, M, col_bias, act, y code or -1, device, stream) -> y
PyObject* w4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 10 || !g_w4) Py_RETURN_NONE;
  try {
    int32_t code;
    const at::Tensor *A = typed(a[0], 2, code), *codes = dense(a[1], at::kByte, 4), *exps = dense(a[2], at::kByte, 4), *bias;
    if (!A || !codes || !exps) Py_RETURN_NONE;
    const int64_t D = PyLong_AsLongLong(a[3]), M = PyLong_AsLongLong(a[4]);
    const long act = PyLong_AsLong(a[6]);
    long out = PyLong_AsLong(a[7]);
    int64_t device;
    void* stream;
    if (!tail(a[8], a[9], device, stream)) Py_RETURN_NONE;
    const int64_t lda = row_stride(*A), N = A->size(0);
    if (D < 1 || M < 1 || M > INT32_MAX || A->size(1) != D || lda < 0 || act < 0 || act > 3 || !vector_or_none(a[5], M, bias)) Py_RETURN_NONE;
    const int64_t mb = (M + 15) / 16, kb = (D + 127) / 128;
    if (codes->size(0) != mb || codes->size(1) != kb || codes->size(2) != 64 || codes->size(3) != 16 || exps->size(0) != mb ||
        exps->size(1) != kb || exps->size(2) != 16 || exps->size(3) != 4)
      Py_RETURN_NONE;
    if (!on(A, device) || !on(codes, device) || !on(exps, device) || !on(bias, device)) Py_RETURN_NONE;
    if (out < 0) out = act == 3 ? 0 : code;
    if (out != code && out != 0) Py_RETURN_NONE;
    const void* pA = A->const_data_ptr();
    at::Tensor y = at::empty({N, M}, A->options().dtype(type_of((int32_t)out)).requires_grad(false));
    const int64_t need = g_w4_bytes(pA, code, N, (int32_t)D, lda, (int32_t)M);
    if (need < 0) Py_RETURN_NONE;
    at::Tensor ws = scratch_of(*A, need);
    if (!aligned256(ws)) Py_RETURN_NONE;
    const uint8_t *pc = static_cast<const uint8_t*>(codes->const_data_ptr()), *pe = static_cast<const uint8_t*>(exps->const_data_ptr());
    const float* pb = bias ? static_cast<const float*>(bias->const_data_ptr()) : nullptr;
    void *py = y.mutable_data_ptr(), *pw = pointer(ws);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_w4(pA, code, N, (int32_t)D, lda, pc, pe, (int32_t)M, pb, (int32_t)act, py, (int32_t)out, pw, need, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) Py_RETURN_NONE;
    return THPVariable_Wrap(y);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// quantize(B, device, stream) -> (codes, exps)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 3 || !g_quantize) Py_RETURN_NONE;
  try {
    int32_t code;
    const at::Tensor* B = typed(a[0], 2, code);
    int64_t device;
    void* stream;
    if (!B || !tail(a[1], a[2], device, stream) || !on(B, device)) Py_RETURN_NONE;
    const int64_t D = B->size(0), M = B->size(1);
    if (D < 1 || M < 1 || D > INT32_MAX || M > INT32_MAX) Py_RETURN_NONE;
    const auto opt = B->options().dtype(at::kByte).requires_grad(false);
    at::Tensor codes = at::empty({(M + 15) / 16, (D + 127) / 128, 64, 16}, opt), exps = at::empty({(M + 15) / 16, (D + 127) / 128, 16, 4}, opt);
    const void* p = B->const_data_ptr();
    uint8_t *pc = static_cast<uint8_t*>(codes.mutable_data_ptr()), *pe = static_cast<uint8_t*>(exps.mutable_data_ptr());
    const int64_t sd = B->stride(0), sm = B->stride(1);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_quantize(p, code, (int32_t)D, (int32_t)M, sd, sm, pc, pe, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) Py_RETURN_NONE;
    return pack({codes, exps});
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// dequantize(codes, exps, D, M, code, device, stream) -> B
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7 || !g_dequantize) Py_RETURN_NONE;
  try {
    const at::Tensor *codes = dense(a[0], at::kByte, 4), *exps = dense(a[1], at::kByte, 4);
    if (!codes || !exps) Py_RETURN_NONE;
    const int64_t D = PyLong_AsLongLong(a[2]), M = PyLong_AsLongLong(a[3]);
    const long code = PyLong_AsLong(a[4]);
    int64_t device;
    void* stream;
    if (!tail(a[5], a[6], device, stream) || !on(codes, device) || !on(exps, device)) Py_RETURN_NONE;
    if (D < 1 || M < 1 || D > INT32_MAX || M > INT32_MAX || (code != 0 && code != 1)) Py_RETURN_NONE;
    const int64_t mb = (M + 15) / 16, kb = (D + 127) / 128;
    if (codes->size(0) != mb || codes->size(1) != kb || codes->size(2) != 64 || codes->size(3) != 16 || exps->size(0) != mb ||
        exps->size(1) != kb || exps->size(2) != 16 || exps->size(3) != 4)
      Py_RETURN_NONE;
    at::Tensor B = at::empty({D, M}, codes->options().dtype(type_of((int32_t)code)).requires_grad(false));
    const uint8_t *pc = static_cast<const uint8_t*>(codes->const_data_ptr()), *pe = static_cast<const uint8_t*>(exps->const_data_ptr());
    void* p = B.mutable_data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_dequantize(pc, pe, (int32_t)D, (int32_t)M, p, (int32_t)code, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) Py_RETURN_NONE;
    return THPVariable_Wrap(B);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// what both cross entropy calls take: A, B, target, col_bias
struct Xent {
  const at::Tensor *A, *B, *target, *bias;
  int32_t code, first;
  int64_t N, D, M, lda;
};
bool xent_args(PyObject* const* a, int64_t device, Xent& x) {
  int32_t code_b;
  x.A = typed(a[0], 2, x.code);
  x.B = typed(a[1], 2, code_b);
  x.target = dense(a[2], at::kLong, 1);
  if (!x.A || !x.B || !x.target || x.code == 2 || code_b != x.code) return false;
  x.N = x.A->size(0);
  x.D = x.A->size(1);
  x.M = x.B->size(1);
  x.lda = row_stride(*x.A);
  if (x.lda < 0 || x.M < 1 || x.M > INT32_MAX || x.B->size(0) != x.D || x.target->size(0) != x.N || !vector_or_none(a[3], x.M, x.bias)) return false;
  if (x.B->is_contiguous()) x.first = 0;
  else if (x.B->stride(0) == 1 && x.B->stride(1) == x.D) x.first = 1;
  else return false;
  return on(x.A, device) && on(x.B, device) && on(x.target, device) && on(x.bias, device);
}

// xent(A, B, target, col_bias, device, stream) -> (loss, lse)
PyObject* xent(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6 || !g_xent) Py_RETURN_NONE;
  try {
    Xent x;
    int64_t device;
    void* stream;
    if (!tail(a[4], a[5], device, stream) || !xent_args(a, device, x)) Py_RETURN_NONE;
    const int64_t need = g_xent_bytes(x.N, (int32_t)x.D, (int32_t)x.M, x.code);
    if (need < 0) Py_RETURN_NONE;
    const auto opt = x.A->options().dtype(at::kFloat).requires_grad(false);
    at::Tensor loss = at::empty({x.N}, opt), lse = at::empty({x.N}, opt), ws = scratch_of(*x.A, need);
    if (!aligned256(ws)) Py_RETURN_NONE;
    const void *pA = x.A->const_data_ptr(), *pB = x.B->const_data_ptr();
    const int64_t* pt = static_cast<const int64_t*>(x.target->const_data_ptr());
    const float* pb = x.bias ? static_cast<const float*>(x.bias->const_data_ptr()) : nullptr;
    float *pl = static_cast<float*>(loss.mutable_data_ptr()), *pe = static_cast<float*>(lse.mutable_data_ptr());
    void* pw = pointer(ws);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_xent(pA, x.code, x.N, (int32_t)x.D, x.lda, pB, (int32_t)x.M, x.first, pb, pt, pl, pe, pw, need, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) Py_RETURN_NONE;
    return pack({loss, lse});
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// xent_grad(A, B, target, col_bias, lse, grad_loss, device, stream) -> (dA, dB, dbias)
PyObject* xent_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 8 || !g_xent_grad) Py_RETURN_NONE;
  try {
    Xent x;
    int64_t device;
    void* stream;
    if (!tail(a[6], a[7], device, stream) || !xent_args(a, device, x)) Py_RETURN_NONE;
    const at::Tensor *lse, *g;
    if (!vector_or_none(a[4], x.N, lse) || !vector_or_none(a[5], x.N, g) || !lse || !g || !on(lse, device) || !on(g, device)) Py_RETURN_NONE;
    const int64_t need = g_xent_grad_bytes(x.N, (int32_t)x.D, (int32_t)x.M, x.code);
    if (need < 0) Py_RETURN_NONE;
    const auto opt = x.A->options().requires_grad(false);
    at::Tensor dA = at::empty({x.N, x.D}, opt), dB = x.first ? at::empty({x.M, x.D}, opt) : at::empty({x.D, x.M}, opt);
    at::Tensor db = at::empty({x.M}, opt.dtype(at::kFloat)), ws = scratch_of(*x.A, need);
    if (!aligned256(ws)) Py_RETURN_NONE;
    const void *pA = x.A->const_data_ptr(), *pB = x.B->const_data_ptr();
    const int64_t* pt = static_cast<const int64_t*>(x.target->const_data_ptr());
    const float* pb = x.bias ? static_cast<const float*>(x.bias->const_data_ptr()) : nullptr;
    const float *pe = static_cast<const float*>(lse->const_data_ptr()), *pg = static_cast<const float*>(g->const_data_ptr());
    void *p1 = dA.mutable_data_ptr(), *p2 = dB.mutable_data_ptr(), *pw = pointer(ws);
    float* p3 = static_cast<float*>(db.mutable_data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_xent_grad(pA, x.code, x.N, (int32_t)x.D, x.lda, pB, (int32_t)x.M, x.first, pb, pt, pe, pg, p1, p2, p3, pw, need, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) Py_RETURN_NONE;
    return pack({dA, x.first ? dB.as_strided({x.D, x.M}, {1, x.D}) : dB, db});
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

PyMethodDef methods[] = {
    {"init", init, METH_VARARGS, "addresses of the library's functions"},
    {"fused", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fused)), METH_FASTCALL, "one fused call"},
    {"w4", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(w4)), METH_FASTCALL, "one layer with 4-bit weights"},
    {"quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(quantize)), METH_FASTCALL, "weights to 4 bits"},
    {"dequantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(dequantize)), METH_FASTCALL, "and back"},
    {"xent", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(xent)), METH_FASTCALL, "one cross entropy"},
    {"xent_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(xent_grad)), METH_FASTCALL, "its gradient"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
