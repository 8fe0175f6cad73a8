// The usual case of the calls between the linear layers, without the interpreter: a decode step makes dozens of
// them, a few microseconds of GPU time each, and argument checks, an allocation and a foreign call from Python cost
// more than that.  Each function here takes what the function of the same name in binding.py takes, checks it
// through torch's DLPack exchange interface (a C structure of function pointers: no libtorch is linked) and makes
// the same call of libtq.  Whatever is not plainly in order (another device or type, a refusal by the library) is
// answered with None, and binding.py goes through its own checks, which say what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/dlpack.h>

#include <cstdint>

#include "tq.h"

namespace {

const DLPackExchangeAPI* g_api = nullptr;
PyTypeObject* g_tensor = nullptr;    // torch.Tensor
PyObject* g_device = nullptr;        // torch._C._cuda_getDevice
PyObject* g_empty_like = nullptr;    // torch.empty_like
PyObject* g_empty = nullptr;         // torch.empty
PyObject* g_bf16 = nullptr;          // torch.bfloat16
PyObject* g_int8 = nullptr;
PyObject* g_f32 = nullptr;
PyObject* g_kwnames = nullptr;       // ("dtype", "device")
PyObject* g_kwdtype = nullptr;       // ("dtype",)
PyObject* g_device_attr = nullptr;   // "device"

decltype(&tq_rmsnorm) f_rmsnorm = nullptr;
decltype(&tq_rmsnorm_q8) f_rmsnorm_q8 = nullptr;
decltype(&tq_rope_append) f_rope = nullptr;
decltype(&tq_paged_attention) f_paged = nullptr;
decltype(&tq_cross_attention) f_cross = nullptr;

struct T {
  DLTensor d;
  bool is(int code, int bits) const { return d.dtype.code == code && d.dtype.bits == bits && d.dtype.lanes == 1; }
  bool bf16() const { return is(kDLBfloat, 16); }
  bool f32() const { return is(kDLFloat, 32); }
  bool i32() const { return is(kDLInt, 32); }
  int type() const { return bf16() ? TQ_TYPE_BF16 : (f32() ? TQ_TYPE_F32 : -1); }
  int64_t n(int i) const { return d.shape[i]; }
  int64_t stride(int i) const { return d.shape[i] > 1 ? d.strides[i] : 0; }  // of a dimension of size 1 it means nothing
  char* ptr() const { return static_cast<char*>(d.data) + d.byte_offset; }
  int64_t numel() const {
    int64_t k = 1;
    for (int i = 0; i < d.ndim; ++i) k *= d.shape[i];
    return k;
  }
  bool contiguous() const {
    int64_t k = 1;
    for (int i = d.ndim - 1; i >= 0; --i) {
      if (d.shape[i] > 1 && d.strides[i] != k) return false;
      k *= d.shape[i];
    }
    return true;
  }
};

// A CUDA tensor on `device` (or on any, where it is -1) with so many dimensions.
bool get(PyObject* o, T& t, int ndim, int device) {
  if (!PyObject_TypeCheck(o, g_tensor)) return false;
  if (g_api->dltensor_from_py_object_no_sync(o, &t.d) != 0) {
    PyErr_Clear();
    return false;
  }
  return t.d.device.device_type == kDLCUDA && (device < 0 || t.d.device.device_id == device) && (ndim < 0 || t.d.ndim == ndim) &&
         (t.d.ndim == 0 || t.d.strides != nullptr);
}

bool current(int device, void** stream) {
  PyObject* r = PyObject_CallNoArgs(g_device);
  const long now = r ? PyLong_AsLong(r) : -1;
  Py_XDECREF(r);
  if (now != device || g_api->current_work_stream(kDLCUDA, device, stream) != 0) {
    PyErr_Clear();
    return false;
  }
  return true;
}

// A new tensor of the given shape on like's device.
PyObject* empty(const int64_t* shape, int ndim, PyObject* dtype, PyObject* like) {
  PyObject* dev = PyObject_GetAttr(like, g_device_attr);
  PyObject* size = PyTuple_New(ndim);
  PyObject* r = nullptr;
  if (dev && size) {
    for (int i = 0; i < ndim; ++i) PyTuple_SET_ITEM(size, i, PyLong_FromLongLong(shape[i]));
    PyObject* args[3] = {size, dtype, dev};
    r = PyObject_Vectorcall(g_empty, args, 1, g_kwnames);
  }
  Py_XDECREF(dev);
  Py_XDECREF(size);
  return r;
}

PyObject* none() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

// out as given, or a new bf16 tensor of this shape; owned by the caller.
PyObject* result(PyObject* out, PyObject* like, const T& like_t, const int64_t* shape, int ndim, int device, T& t) {
  if (out != Py_None) {
    int64_t k = 1;
    for (int i = 0; i < ndim; ++i) k *= shape[i];
    if (!get(out, t, -1, device) || !t.bf16() || !t.contiguous() || t.numel() != k) return nullptr;
    Py_INCREF(out);
    return out;
  }
  bool same = like_t.contiguous() && like_t.d.ndim == ndim;
  for (int i = 0; same && i < ndim; ++i) same = like_t.n(i) == shape[i];
  PyObject* args[2] = {like, g_bf16};
  PyObject* r = !same ? empty(shape, ndim, g_bf16, like)
                      : (like_t.bf16() ? PyObject_CallOneArg(g_empty_like, like) : PyObject_Vectorcall(g_empty_like, args, 1, g_kwdtype));
  if (r && !get(r, t, ndim, device)) {
    Py_DECREF(r);
    return nullptr;
  }
  return r;
}

// h, weight, delta, h_out of the norms
struct Norm {
  T h, w, d, ho;
  const void* dp = nullptr;
  int dt = 0, device = 0;
  int64_t ds = 0;
  void* hop = nullptr;
  uint32_t rows = 0, cols = 0;
  void* stream = nullptr;
};
bool norm_args(PyObject* const* a, PyObject* h_out, Norm& n) {
  if (!get(a[0], n.h, 2, -1)) return false;
  n.device = n.h.d.device.device_id;
  if (n.h.type() < 0 || n.h.n(0) > 0x7FFFFFFF || n.h.n(1) > 0x7FFFFFFF || n.h.n(1) == 0) return false;
  n.rows = (uint32_t)n.h.n(0);
  n.cols = (uint32_t)n.h.n(1);
  if (n.cols > 1 && n.h.d.strides[1] != 1) return false;
  if (!get(a[1], n.w, 1, n.device) || !n.w.f32() || !n.w.contiguous() || n.w.n(0) != n.cols) return false;
  if (a[2] != Py_None) {
    if (!get(a[2], n.d, 2, n.device) || n.d.type() < 0 || n.d.n(0) != n.rows || n.d.n(1) != n.cols || (n.cols > 1 && n.d.d.strides[1] != 1)) return false;
    n.dp = n.d.ptr();
    n.dt = n.d.type();
    n.ds = n.d.stride(0);
    n.hop = n.h.ptr();
  }
  if (h_out != Py_None) {
    if (!get(h_out, n.ho, 2, n.device) || n.ho.type() != n.h.type() || n.ho.n(0) != n.rows || n.ho.n(1) != n.cols) return false;
    if (n.ho.stride(0) != n.h.stride(0) || n.ho.stride(1) != n.h.stride(1)) return false;
    n.hop = n.ho.ptr();
  }
  return current(n.device, &n.stream);
}

// (h, weight, delta, eps, out, h_out)
PyObject* py_rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t count) {
  Norm n;
  T o;
  if (count != 6 || !norm_args(a, a[5], n)) return none();
  const double eps = PyFloat_AsDouble(a[3]);
  if (eps == -1.0 && PyErr_Occurred()) return none();
  const int64_t shape[2] = {n.rows, n.cols};
  PyObject* out = result(a[4], a[0], n.h, shape, 2, n.device, o);
  if (!out) return none();
  if (f_rmsnorm(n.h.ptr(), n.h.type(), n.h.stride(0), n.dp, n.dt, n.ds, (const float*)n.w.ptr(), (float)eps, n.rows, n.cols, n.hop, o.ptr(),
                n.stream) == TQ_OK)
    return out;
  Py_DECREF(out);
  return none();
}

// (h, weight, delta, eps, h_out) -> (q, scale)
PyObject* py_rmsnorm_q8(PyObject*, PyObject* const* a, Py_ssize_t count) {
  Norm n;
  T q, s;
  if (count != 5 || !norm_args(a, a[4], n)) return none();
  const double eps = PyFloat_AsDouble(a[3]);
  if (eps == -1.0 && PyErr_Occurred()) return none();
  const int64_t shape[2] = {n.rows, n.cols};
  PyObject* qo = empty(shape, 2, g_int8, a[0]);
  PyObject* so = qo ? empty(shape, 1, g_f32, a[0]) : nullptr;
  if (so && get(qo, q, 2, n.device) && get(so, s, 1, n.device) &&
      f_rmsnorm_q8(n.h.ptr(), n.h.type(), n.h.stride(0), n.dp, n.dt, n.ds, (const float*)n.w.ptr(), (float)eps, n.rows, n.cols, n.hop,
                   (int8_t*)q.ptr(), (float*)s.ptr(), n.stream) == TQ_OK) {
    PyObject* r = PyTuple_Pack(2, qo, so);
    Py_DECREF(qo);
    Py_DECREF(so);
    return r;
  }
  Py_XDECREF(qo);
  Py_XDECREF(so);
  return none();
}

const tq_kv_cache* cache_of(PyObject* address) { return static_cast<const tq_kv_cache*>(PyLong_AsVoidPtr(address)); }

// token stride of [tokens][n * dim] or [tokens][n][dim], -1: not one of them
int64_t heads(PyObject* o, T& t, int64_t tokens, int64_t n, int64_t dim, int type, int device) {
  if (!get(o, t, -1, device) || (t.d.ndim != 2 && t.d.ndim != 3) || t.type() != type || t.n(0) != tokens) return -1;
  const int last = t.d.ndim - 1;
  if (t.d.strides[last] != 1) return -1;
  if (t.d.ndim == 2 ? t.n(1) != n * dim : (t.n(1) != n || t.n(2) != dim || (n > 1 && t.d.strides[1] != dim))) return -1;
  return t.stride(0) < 0 ? -1 : t.stride(0);
}

// (q, k, v, table, positions, slots, cache address, cache device, sections or None, interleaved, out)
PyObject* py_rope_append(PyObject*, PyObject* const* a, Py_ssize_t count) {
  T q, k, v, table, pos, slots, o;
  if (count != 11 || !get(a[0], q, -1, -1) || (q.d.ndim != 2 && q.d.ndim != 3)) return none();
  const tq_kv_cache* c = cache_of(a[6]);
  const int device = q.d.device.device_id, type = q.type();
  if (!c || PyLong_AsLong(a[7]) != device || type < 0 || q.n(0) > 0x7FFFFFFF) return none();
  const int64_t D = c->head_dim, K = c->n_kv_heads, tokens = q.n(0), H = q.d.ndim == 3 ? q.n(1) : q.n(1) / D;
  const int64_t qs = heads(a[0], q, tokens, H, D, type, device), ks = heads(a[1], k, tokens, K, D, type, device),
                vs = heads(a[2], v, tokens, K, D, type, device);
  if (qs < 0 || ks < 0 || vs < 0 || H <= 0 || H > 65536) return none();
  if (!get(a[3], table, 2, device) || !table.f32() || !table.contiguous() || table.n(0) > 0x7FFFFFFF || table.n(1) > 0x7FFFFFFF) return none();
  if (!get(a[4], pos, -1, device) || !pos.i32() || !pos.contiguous() || pos.d.ndim < 1 || pos.d.ndim > 2) return none();
  const int64_t axes = pos.d.ndim == 1 ? 1 : pos.n(0);
  if (axes < 1 || axes > (int64_t)TQ_ROPE_MAX_AXES || pos.numel() != axes * tokens) return none();
  if (!get(a[5], slots, -1, device) || !slots.i32() || !slots.contiguous() || slots.numel() != tokens) return none();
  uint32_t sections[TQ_ROPE_MAX_AXES] = {(uint32_t)(table.n(1) / 2)};
  if (a[8] != Py_None) {
    const bool list = PyList_Check(a[8]);
    if ((!list && !PyTuple_Check(a[8])) || PySequence_Fast_GET_SIZE(a[8]) != axes) return none();
    for (int64_t i = 0; i < axes; ++i) {
      const long x = PyLong_AsLong(PySequence_Fast_GET_ITEM(a[8], i));
      if (x < 0 || x > 0x7FFFFFFF) return none();
      sections[i] = (uint32_t)x;
    }
  } else if (axes != 1) {
    return none();
  }
  const int inter = PyObject_IsTrue(a[9]);
  void* stream;
  if (inter < 0 || !current(device, &stream)) return none();
  const int64_t shape[3] = {tokens, H, D};
  PyObject* out = result(a[10], a[0], q, shape, 3, device, o);
  if (!out) return none();
  if (f_rope(q.ptr(), k.ptr(), v.ptr(), type, qs, ks, vs, (uint32_t)tokens, (uint32_t)H, (const float*)table.ptr(), (uint32_t)table.n(0),
             (uint32_t)table.n(1), (const int32_t*)pos.ptr(), sections, (uint32_t)axes, inter, (const int32_t*)slots.ptr(), c, o.ptr(), stream) == TQ_OK)
    return out;
  Py_DECREF(out);
  return none();
}

// out and lse of an attention call with queries q
PyObject* attn_result(PyObject* out, PyObject* lse, PyObject* q, const T& qt, int device, T& o, float** lse_ptr) {
  T l;
  *lse_ptr = nullptr;
  if (lse != Py_None) {
    if (!get(lse, l, qt.d.ndim - 1, device) || !l.f32() || !l.contiguous()) return nullptr;
    for (int i = 0; i < qt.d.ndim - 1; ++i)
      if (l.n(i) != qt.n(i)) return nullptr;
    *lse_ptr = (float*)l.ptr();
  }
  if (out != Py_None) {  // the shape itself, not its size alone
    if (!get(out, o, qt.d.ndim, device)) return nullptr;
    for (int i = 0; i < qt.d.ndim; ++i)
      if (o.n(i) != qt.n(i)) return nullptr;
  }
  return result(out, q, qt, qt.d.shape, qt.d.ndim, device, o);
}

// (q, cache address, cache device, page_table, lens, workspace address, bytes, workspace device, scale, out, lse)
PyObject* py_paged_attention(PyObject*, PyObject* const* a, Py_ssize_t count) {
  T q, table, lens, o;
  if (count != 11 || !get(a[0], q, 3, -1) || !q.bf16()) return none();
  const tq_kv_cache* c = cache_of(a[1]);
  const int device = q.d.device.device_id;
  if (!c || PyLong_AsLong(a[2]) != device || PyLong_AsLong(a[7]) != device) return none();
  const int64_t B = q.n(0), H = q.n(1), D = q.n(2);
  if (D != c->head_dim || q.d.strides[2] != 1 || (H > 1 && q.d.strides[1] != D) || B > 0x7FFFFFFF || H > 65536) return none();
  if (!get(a[3], table, 2, device) || !table.i32() || !table.contiguous() || table.n(0) != B || table.n(1) > 0x7FFFFFFF) return none();
  if (!get(a[4], lens, -1, device) || !lens.i32() || !lens.contiguous() || lens.numel() != B) return none();
  const double scale = PyFloat_AsDouble(a[8]);
  void* ws = PyLong_AsVoidPtr(a[5]);
  const uint64_t bytes = PyLong_AsUnsignedLongLong(a[6]);
  void* stream;
  if (PyErr_Occurred() || !current(device, &stream)) return none();
  float* lse;
  PyObject* out = attn_result(a[9], a[10], a[0], q, device, o, &lse);
  if (!out) return none();
  if (f_paged(c, q.ptr(), q.stride(0), (uint32_t)B, (uint32_t)H, (const int32_t*)table.ptr(), (uint32_t)table.n(1), (const int32_t*)lens.ptr(),
              (float)scale, o.ptr(), lse, ws, bytes, stream) == TQ_OK)
    return out;
  Py_DECREF(out);
  return none();
}

// (q, k, v, workspace address, bytes, workspace device, kv_len, mask, block_len, scale, out, lse)
PyObject* py_cross_attention(PyObject*, PyObject* const* a, Py_ssize_t count) {
  T q, k, v, o, t;
  if (count != 12 || !get(a[0], q, 4, -1) || !q.bf16()) return none();
  const int device = q.d.device.device_id;
  const int64_t B = q.n(0), tokens = q.n(1), H = q.n(2), D = q.n(3);
  if (PyLong_AsLong(a[5]) != device || q.d.strides[3] != 1 || (H > 1 && q.d.strides[2] != D) || B > 0x7FFFFFFF || tokens > 0x7FFFFFFF || H > 65536) return none();
  if (!get(a[1], k, 4, device) || !get(a[2], v, 4, device) || !k.bf16() || !v.bf16() || k.n(0) != B || k.n(3) != D || k.d.strides[3] != 1) return none();
  for (int i = 0; i < 4; ++i)
    if (k.n(i) != v.n(i) || k.stride(i) != v.stride(i)) return none();
  const int64_t S = k.n(1);
  if (S > 0x7FFFFFFF || k.n(2) > 65536) return none();
  const int32_t* kv_len = nullptr;
  if (a[6] != Py_None) {
    if (!get(a[6], t, -1, device) || !t.i32() || !t.contiguous() || t.numel() != B) return none();
    kv_len = (const int32_t*)t.ptr();
  }
  const int64_t block = PyLong_AsLongLong(a[8]);
  const uint8_t* mask = nullptr;
  if (a[7] != Py_None) {
    if (block < 1 || block > 0x7FFFFFFF || !get(a[7], t, 3, device) || !(t.is(kDLUInt, 8) || t.is(kDLBool, 8)) || !t.contiguous()) return none();
    if (t.n(0) != B || t.n(1) != tokens || t.n(2) != (S + block - 1) / block) return none();
    mask = (const uint8_t*)t.ptr();
  }
  const double scale = PyFloat_AsDouble(a[9]);
  void* ws = PyLong_AsVoidPtr(a[3]);
  const uint64_t bytes = PyLong_AsUnsignedLongLong(a[4]);
  void* stream;
  if (PyErr_Occurred() || !current(device, &stream)) return none();
  float* lse;
  PyObject* out = attn_result(a[10], a[11], a[0], q, device, o, &lse);
  if (!out) return none();
  const tq_encoder_kv kv{k.ptr(), v.ptr(), (uint32_t)B, (uint32_t)S, (uint32_t)k.n(2), (uint32_t)D, k.stride(0), k.stride(1), k.stride(2)};
  if (f_cross(&kv, q.ptr(), q.stride(0), q.stride(1), (uint32_t)tokens, (uint32_t)H, kv_len, mask, (uint32_t)(mask ? block : 0), (float)scale, o.ptr(),
              lse, ws, bytes, stream) == TQ_OK)
    return out;
  Py_DECREF(out);
  return none();
}

// setup(torch, addresses of the five library functions): True if this torch has the exchange interface
PyObject* py_setup(PyObject*, PyObject* const* a, Py_ssize_t count) {
  if (count != 6) {
    PyErr_SetString(PyExc_TypeError, "setup(torch, rmsnorm, rmsnorm_q8, rope_append, paged_attention, cross_attention)");
    return nullptr;
  }
  PyObject* torch = a[0];
  PyObject* tensor = PyObject_GetAttrString(torch, "Tensor");
  PyObject* c = PyObject_GetAttrString(torch, "_C");
  if (!tensor || !c) return nullptr;
  PyObject* capsule = PyObject_GetAttrString(tensor, "__dlpack_c_exchange_api__");
  const DLPackExchangeAPI* api = capsule ? (const DLPackExchangeAPI*)PyCapsule_GetPointer(capsule, "dlpack_exchange_api") : nullptr;
  Py_XDECREF(capsule);
  if (!api || api->header.version.major != DLPACK_MAJOR_VERSION || !api->dltensor_from_py_object_no_sync || !api->current_work_stream) {
    PyErr_Clear();
    Py_RETURN_FALSE;
  }
  g_tensor = (PyTypeObject*)tensor;
  g_device = PyObject_GetAttrString(c, "_cuda_getDevice");
  g_empty_like = PyObject_GetAttrString(torch, "empty_like");
  g_empty = PyObject_GetAttrString(torch, "empty");
  g_bf16 = PyObject_GetAttrString(torch, "bfloat16");
  g_int8 = PyObject_GetAttrString(torch, "int8");
  g_f32 = PyObject_GetAttrString(torch, "float32");
  g_kwnames = Py_BuildValue("(ss)", "dtype", "device");
  g_kwdtype = Py_BuildValue("(s)", "dtype");
  g_device_attr = PyUnicode_InternFromString("device");
  if (!g_kwdtype || !g_device || !g_empty_like || !g_empty || !g_bf16 || !g_int8 || !g_f32 || !g_kwnames || !g_device_attr) {
    PyErr_Clear();
    Py_RETURN_FALSE;
  }
  f_rmsnorm = (decltype(f_rmsnorm))PyLong_AsVoidPtr(a[1]);
  f_rmsnorm_q8 = (decltype(f_rmsnorm_q8))PyLong_AsVoidPtr(a[2]);
  f_rope = (decltype(f_rope))PyLong_AsVoidPtr(a[3]);
  f_paged = (decltype(f_paged))PyLong_AsVoidPtr(a[4]);
  f_cross = (decltype(f_cross))PyLong_AsVoidPtr(a[5]);
  if (PyErr_Occurred()) return nullptr;
  g_api = api;
  Py_RETURN_TRUE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(setup),           FAST(rmsnorm),         FAST(rmsnorm_q8), FAST(rope_append),
                         FAST(paged_attention), FAST(cross_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tqfast", "The usual case of the calls between the linear layers.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tqfast() { return PyModule_Create(&module); }
