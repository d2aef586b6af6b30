// CPython module of the serving calls: checks torch tensors and passes them to the C entry points.
//
// A decode step makes a handful of these calls per layer, each a few microseconds of GPU time, so the
// checks and the marshalling of one call have to cost about one: here they do (a ctypes call with the same
// checks in Python takes 10 to 15).  Every function returns the omq_status; a tensor that does not fit is a
// ValueError, a workspace for which there is no room a torch.OutOfMemoryError, and nothing is launched.  Work
// goes to the current stream of the tensors' device; a workspace comes from torch's caching allocator on that
// stream and is handed back when the call returns, in stream order.
#include <torch/csrc/autograd/python_variable.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <exception>
#include <string>

#include "omq.h"

namespace {

struct Bad { std::string what; };

const at::Tensor* tensor(PyObject* o, const char* name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) throw Bad{std::string(name) + ": a tensor or None"};
  return &THPVariable_Unpack(o);
}

// The tensors of one call: all on one CUDA device.
struct Call {
  int device = -1;

  void place(const at::Tensor& t, const char* name) {
    if (!t.is_cuda()) throw Bad{std::string(name) + ": a CUDA tensor"};
    const int d = t.get_device();
    if (device < 0) device = d;
    if (d != device) throw Bad{std::string(name) + ": on the device of the other tensors"};
  }

  // n contiguous values
  void* vec(PyObject* o, const char* name, at::ScalarType type, int64_t n, bool required = false) {
    const at::Tensor* t = tensor(o, name);
    if (!t) {
      if (required) throw Bad{std::string(name) + ": required"};
      return nullptr;
    }
    place(*t, name);
    if (t->scalar_type() != type || t->numel() != n || !t->is_contiguous())
      throw Bad{std::string(name) + ": " + std::to_string(n) + " contiguous values of " + c10::toString(type)};
    return t->data_ptr();
  }

  // 2-D, rows contiguous; *ld is the row stride
  const at::Tensor* rows(PyObject* o, const char* name, int64_t n, int64_t cols, int64_t* ld) {
    const at::Tensor* t = tensor(o, name);
    if (!t) return nullptr;
    place(*t, name);
    if (t->dim() != 2 || (n >= 0 && t->size(0) != n) || (cols >= 0 && t->size(1) != cols) ||
        (t->size(1) > 1 && t->stride(1) != 1))
      throw Bad{std::string(name) + ": [" + (n >= 0 ? std::to_string(n) : "n") + ", " + (cols >= 0 ? std::to_string(cols) : "n") +
                "] with contiguous rows"};
    *ld = t->size(0) > 1 ? t->stride(0) : t->size(1);
    return t;
  }

  int32_t float_type(const at::Tensor& t, const char* name) {
    if (t.scalar_type() == at::kFloat) return OMQ_F32;
    if (t.scalar_type() == at::kBFloat16) return OMQ_BF16;
    throw Bad{std::string(name) + ": float32 or bfloat16"};
  }

  omq_stream_t stream() const { return (omq_stream_t)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
};

// scratch memory in stream order
struct Scratch {
  void* p = nullptr;
  Scratch(size_t n, omq_stream_t s) {
    if (n) p = c10::cuda::CUDACachingAllocator::raw_alloc_with_stream(n, (cudaStream_t)s);
  }
  ~Scratch() {
    if (p) c10::cuda::CUDACachingAllocator::raw_delete(p);
  }
};

int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Bad{""};
  return v;
}

// 32-bit argument of an entry point
int32_t integer32(PyObject* o, const char* name) {
  const int64_t v = integer(o);
  if (v < INT32_MIN || v > INT32_MAX) throw Bad{std::string(name) + ": out of range"};
  return (int32_t)v;
}

double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Bad{""};
  return v;
}

int32_t* word(PyObject* o, const char* name, Call& c) { return (int32_t*)c.vec(o, name, at::kInt, 1); }

// x, r, gain, bias, bits, rms_eps, h_eps, codes, h, z, values, residual
omq_status rmsnorm_quant(PyObject* const* a) {
  Call c;
  int64_t ldx = 0, ldr = 0, ldh = 0;
  const at::Tensor* x = c.rows(a[0], "x", -1, -1, &ldx);
  if (!x) throw Bad{"x: required"};
  const int64_t T = x->size(0), C = x->size(1);
  const int32_t xd = c.float_type(*x, "x");
  int32_t rd = OMQ_F32;
  const at::Tensor* r = c.rows(a[1], "r", T, C, &ldr);
  const at::Tensor* h = c.rows(a[11], "residual", T, C, &ldh);
  if (r) rd = c.float_type(*r, "r");
  if (h) {
    if (r && (c.float_type(*h, "residual") != rd || (ldh != ldr && T > 1)))
      throw Bad{"residual: the type and row stride of r"};
    rd = c.float_type(*h, "residual");
    ldr = ldh;
  }
  omq_qcfg cfg{};
  cfg.wbits = 16;
  cfg.abits = integer32(a[4], "bits");
  cfg.h_eps = (float)real(a[6]);
  const float* gain = (const float*)c.vec(a[2], "gain", at::kFloat, C);
  const float* bias = (const float*)c.vec(a[3], "bias", at::kFloat, C);
  uint8_t* codes = (uint8_t*)c.vec(a[7], "codes", at::kByte, T * C);
  float* step = (float*)c.vec(a[8], "h", at::kFloat, T);
  int32_t* zero = (int32_t*)c.vec(a[9], "z", at::kInt, T);
  void* values = c.vec(a[10], "values", at::kBFloat16, T * C);
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.device);
  return omq_rmsnorm_quant(c.stream(), T, C, x->data_ptr(), xd, ldx, r ? r->data_ptr() : nullptr, h ? h->data_ptr() : nullptr,
                           rd, ldr, gain, bias, (float)real(a[5]), codes, values, step, zero, &cfg);
}

// a, a_h, a_z, w, w_h, w_z, bias, out, status
omq_status qgemm(PyObject* const* a) {
  Call c;
  int64_t lda = 0, ldw = 0, ldc = 0;
  const at::Tensor* x = c.rows(a[0], "a", -1, -1, &lda);
  if (!x) throw Bad{"a: required"};
  const int64_t M = x->size(0), K = x->size(1);
  const at::Tensor* w = c.rows(a[3], "w", -1, K, &ldw);
  if (!w) throw Bad{"w: required"};
  const int64_t N = w->size(0);
  const at::Tensor* y = c.rows(a[7], "out", M, N, &ldc);
  if (!y) throw Bad{"out: required"};
  if (x->scalar_type() != at::kByte || w->scalar_type() != at::kByte) throw Bad{"a, w: uint8 codes"};
  const bool f32 = c.float_type(*y, "out") == OMQ_F32;
  const float* ah = (const float*)c.vec(a[1], "a_h", at::kFloat, M, true);
  const int32_t* az = (const int32_t*)c.vec(a[2], "a_z", at::kInt, M);
  const float* wh = (const float*)c.vec(a[4], "w_h", at::kFloat, N, true);
  const int32_t* wz = (const int32_t*)c.vec(a[5], "w_z", at::kInt, N);
  const float* bias = (const float*)c.vec(a[6], "bias", at::kFloat, N);
  int32_t* status = word(a[8], "status", c);
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.device);
  const omq_stream_t s = c.stream();
  const size_t need = omq_qgemm_i8_workspace_size(M, N, K);
  const Scratch ws(need, s);
  return omq_qgemm_i8(s, M, N, K, (const uint8_t*)x->data_ptr(), lda, ah, az, (const uint8_t*)w->data_ptr(), ldw, wh, wz, bias,
                      f32 ? (float*)y->data_ptr() : nullptr, f32 ? nullptr : y->data_ptr(), ldc, ws.p, need, status);
}

struct Rows { int32_t total, max_q; const int32_t* cu; };

// cu_q and max_q of a call on `rows` rows: without cu_q every sequence has the same number
Rows row_map(Call& c, const omq_kv_cache* kv, int64_t rows, PyObject* cu, PyObject* max_q) {
  if (kv->B <= 0) throw Bad{"cache: at least one sequence"};
  if (rows > INT32_MAX) throw Bad{"rows: too many"};
  Rows r{(int32_t)rows, 0, nullptr};
  if (cu == Py_None) {
    if (rows % kv->B != 0 || (max_q != Py_None && integer(max_q) != rows / kv->B))
      throw Bad{"rows: the same number for every sequence without cu_q"};
    r.max_q = (int32_t)(rows / kv->B);
  } else {
    if (max_q == Py_None) throw Bad{"max_q: needed with cu_q"};
    r.cu = (const int32_t*)c.vec(cu, "cu_q", at::kInt, (int64_t)kv->B + 1);
    r.max_q = integer32(max_q, "max_q");
  }
  return r;
}

// address of the omq_kv_cache, qkv, rope, n_heads, cu_q, max_q, sa, q_out, k_out, v_out, status
omq_status kv_append(PyObject* const* a) {
  Call c;
  const omq_kv_cache* kv = (const omq_kv_cache*)PyLong_AsVoidPtr(a[0]);
  if (!kv) throw Bad{PyErr_Occurred() ? "" : "cache: required"};
  const int32_t heads = integer32(a[3], "n_heads");
  const int64_t qw = (int64_t)heads * 128, kw = (int64_t)kv->n_kv * 128;
  int64_t ld = 0, ldq = 0, ldk = 0, ldv = 0;
  const at::Tensor* x = c.rows(a[1], "qkv", -1, qw + 2 * kw, &ld);
  if (!x) throw Bad{"qkv: required"};
  const int64_t n = x->size(0);
  const Rows r = row_map(c, kv, n, a[4], a[5]);
  const at::Tensor* rope = tensor(a[2], "rope");
  if (!rope || rope->dim() != 3 || rope->size(1) != 64 || rope->size(2) != 2 || rope->scalar_type() != at::kFloat ||
      !rope->is_contiguous() || rope->size(0) > INT32_MAX)
    throw Bad{"rope: contiguous float32 [n_pos, 64, 2]"};
  c.place(*rope, "rope");
  const float* sa = (const float*)c.vec(a[6], "sa", at::kFloat, kw);
  const at::Tensor* q = c.rows(a[7], "q_out", n, qw, &ldq);
  if (!q) throw Bad{"q_out: required"};
  const at::Tensor* k = c.rows(a[8], "k_out", n, kw, &ldk);
  const at::Tensor* v = c.rows(a[9], "v_out", n, kw, &ldv);
  if (!k != !v || (k && ldk != ldv)) throw Bad{"k_out, v_out: both or neither, of one row stride"};
  if (q->scalar_type() != at::kBFloat16 || (k && (k->scalar_type() != at::kBFloat16 || v->scalar_type() != at::kBFloat16)))
    throw Bad{"q_out, k_out, v_out: bfloat16"};
  int32_t* status = word(a[10], "status", c);
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.device);
  return omq_kv_append(c.stream(), kv, r.total, r.max_q, r.cu, heads, x->data_ptr(), c.float_type(*x, "qkv"), ld,
                       (const float*)rope->data_ptr(), (int32_t)rope->size(0), sa, q->data_ptr(), ldq,
                       k ? k->data_ptr() : nullptr, v ? v->data_ptr() : nullptr, ldk, status);
}

// address of the omq_kv_cache, q, n_heads, cu_q, max_q, max_kv, out, lse, status
omq_status kv_attention(PyObject* const* a) {
  Call c;
  const omq_kv_cache* kv = (const omq_kv_cache*)PyLong_AsVoidPtr(a[0]);
  if (!kv) throw Bad{PyErr_Occurred() ? "" : "cache: required"};
  const int32_t heads = integer32(a[2], "n_heads");
  const int64_t qw = (int64_t)heads * 128;
  int64_t ldq = 0, ldo = 0;
  const at::Tensor* q = c.rows(a[1], "q", -1, qw, &ldq);
  if (!q || q->scalar_type() != at::kBFloat16) throw Bad{"q: bfloat16 [rows, n_heads * 128]"};
  const int64_t n = q->size(0);
  const Rows r = row_map(c, kv, n, a[3], a[4]);
  const int32_t max_kv = integer32(a[5], "max_kv");
  const at::Tensor* o = c.rows(a[6], "out", n, qw, &ldo);
  if (!o) throw Bad{"out: required"};
  const bool f32 = c.float_type(*o, "out") == OMQ_F32;
  float* lse = (float*)c.vec(a[7], "lse", at::kFloat, n * heads);
  int32_t* status = word(a[8], "status", c);
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)c.device);
  const omq_stream_t s = c.stream();
  const size_t need = omq_kv_attention_workspace_size(kv->B, r.total, r.max_q, max_kv, heads, kv->n_kv);
  const Scratch ws(need, s);
  return omq_kv_attention(s, kv, r.total, r.max_q, r.cu, max_kv, heads, q->data_ptr(), ldq,
                          f32 ? (float*)o->data_ptr() : nullptr, f32 ? nullptr : o->data_ptr(), ldo, lse, ws.p, need, status);
}

template <omq_status (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", N, n);
    return nullptr;
  }
  try {
    const omq_status s = F(args);
    return PyLong_FromLong((long)s);
  } catch (const Bad& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what.c_str());
  } catch (const c10::OutOfMemoryError& e) {       // as torch's own allocations report it
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* kind = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    if (kind) PyErr_SetString(kind, e.what_without_backtrace());
    Py_XDECREF(kind);
    Py_XDECREF(torch);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

#define ENTRY(name, n) {#name, (PyCFunction)(void (*)(void))entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(rmsnorm_quant, 12), ENTRY(qgemm, 9), ENTRY(kv_append, 11), ENTRY(kv_attention, 9),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bind(void) { return PyModule_Create(&module); }
