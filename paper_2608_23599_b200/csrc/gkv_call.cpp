// The calls of a decode step without ctypes: a Python extension that takes the arguments of the binding's methods
// (tensors, device addresses or None), makes the pointers of them and calls the C ABI with the interpreter lock released, as ctypes
// does.  An argument that it cannot convert is not judged here: the function returns NotImplemented and the binding goes through
// ctypes, which converts it or raises what it always raised.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/gkv.h"

namespace {

// the library's entry points, handed over by the binding, which has loaded it
decltype(&gkv_append_demote) f_append = nullptr;
decltype(&gkv_decode_attn) f_decode = nullptr;
decltype(&gkv_decode_attn_observe) f_observe = nullptr;
decltype(&gkv_quest_select) f_select = nullptr;
PyObject* s_data_ptr = nullptr;      // "data_ptr"
PyObject* s_value = nullptr;         // "value"
PyObject* void_p = nullptr;          // ctypes.c_void_p

// an int or None
bool as_plain(PyObject* o, void** out) {
  if (o != Py_None && !PyLong_Check(o)) return false;
  *out = o == Py_None ? nullptr : reinterpret_cast<void*>(static_cast<uintptr_t>(PyLong_AsUnsignedLongLongMask(o)));
  return !PyErr_Occurred();
}
// an int, None, or a tensor
bool as_address(PyObject* o, void** out) {
  if (o == Py_None || PyLong_Check(o)) return as_plain(o, out);
  PyObject* v = PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (!v) return false;
  const bool ok = as_plain(v, out);
  Py_DECREF(v);
  return ok;
}
// a ctypes.c_void_p, an int or None
bool as_handle(PyObject* o, gkv_cache** out) {
  void* p = nullptr;
  bool ok;
  if (reinterpret_cast<PyObject*>(Py_TYPE(o)) == void_p) {
    PyObject* v = PyObject_GetAttr(o, s_value);
    if (!v) return false;
    ok = as_plain(v, &p);
    Py_DECREF(v);
  } else {
    ok = as_plain(o, &p);
  }
  *out = static_cast<gkv_cache*>(p);
  return ok;
}
bool as_int(PyObject* o, int32_t* out) {
  if (!PyLong_Check(o)) return false;
  *out = static_cast<int32_t>(PyLong_AsUnsignedLongMask(o));
  return !PyErr_Occurred();
}
// An exception of the conversion is raised again, or not, by the binding's second attempt (an interrupt is not one).
PyObject* refuse() {
  if (PyErr_Occurred()) {
    if (!PyErr_ExceptionMatches(PyExc_Exception)) return nullptr;
    PyErr_Clear();
  }
  Py_RETURN_NOTIMPLEMENTED;
}
bool want(Py_ssize_t n, Py_ssize_t need) {
  if (n == need) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments are needed, not %zd", need, n);
  return false;
}

// bind(append, decode, observe, select, c_void_p): addresses, and ctypes' type of a handle
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* p[4];
  if (!want(n, 5)) return nullptr;
  for (int i = 0; i < 4; ++i)
    if (!as_plain(a[i], &p[i])) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_TypeError, "an address is needed");
  Py_INCREF(a[4]);
  Py_XSETREF(void_p, a[4]);
  f_append = reinterpret_cast<decltype(f_append)>(p[0]);
  f_decode = reinterpret_cast<decltype(f_decode)>(p[1]);
  f_observe = reinterpret_cast<decltype(f_observe)>(p[2]);
  f_select = reinterpret_cast<decltype(f_select)>(p[3]);
  Py_RETURN_NONE;
}

// append(handle, layer, k, v, n_new, token_mass, level_plan, stream)
PyObject* py_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  gkv_cache* h;
  int32_t layer, n_new;
  void *k, *v, *mass, *plan, *st;
  if (!want(n, 8)) return nullptr;
  if (!as_handle(a[0], &h) || !as_int(a[1], &layer) || !as_address(a[2], &k) || !as_address(a[3], &v) || !as_int(a[4], &n_new) ||
      !as_address(a[5], &mass) || !as_address(a[6], &plan) || !as_plain(a[7], &st))
    return refuse();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f_append(h, layer, k, v, n_new, static_cast<const float*>(mass), static_cast<const int8_t*>(plan), st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// decode(handle, layer, q, page_idx, n_sel, out, lse, stream)
PyObject* py_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  gkv_cache* h;
  int32_t layer, n_sel;
  void *q, *pages, *out, *lse, *st;
  if (!want(n, 8)) return nullptr;
  if (!as_handle(a[0], &h) || !as_int(a[1], &layer) || !as_address(a[2], &q) || !as_address(a[3], &pages) || !as_int(a[4], &n_sel) ||
      !as_address(a[5], &out) || !as_address(a[6], &lse) || !as_plain(a[7], &st))
    return refuse();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f_decode(h, layer, q, static_cast<const int32_t*>(pages), n_sel, static_cast<float*>(out), static_cast<float*>(lse), st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// observe(handle, layer, q, out, lse, block_mass, certificate, stream)
PyObject* py_observe(PyObject*, PyObject* const* a, Py_ssize_t n) {
  gkv_cache* h;
  int32_t layer;
  void *q, *out, *lse, *mass, *cert, *st;
  if (!want(n, 8)) return nullptr;
  if (!as_handle(a[0], &h) || !as_int(a[1], &layer) || !as_address(a[2], &q) || !as_address(a[3], &out) || !as_address(a[4], &lse) ||
      !as_address(a[5], &mass) || !as_address(a[6], &cert) || !as_plain(a[7], &st))
    return refuse();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f_observe(h, layer, q, static_cast<float*>(out), static_cast<float*>(lse), static_cast<float*>(mass), static_cast<float*>(cert), st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// select(handle, layer, q, budget_tokens, page_idx_out, stream) -> (status, pages selected)
PyObject* py_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
  gkv_cache* h;
  int32_t layer, budget, n_sel = 0;
  void *q, *pages, *st;
  if (!want(n, 6)) return nullptr;
  if (!as_handle(a[0], &h) || !as_int(a[1], &layer) || !as_address(a[2], &q) || !as_int(a[3], &budget) || !as_address(a[4], &pages) ||
      !as_plain(a[5], &st))
    return refuse();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f_select(h, layer, q, budget, static_cast<int32_t*>(pages), &n_sel, st);
  Py_END_ALLOW_THREADS
  return Py_BuildValue("(ii)", rc, static_cast<int>(n_sel));
}

// ---- calls whose tensors are looked at here: prompts and chunks -------------------------------------
// Everything that the binding asks of the arguments is asked here too, without its messages: what is not in order makes the function return
// NotImplemented, and the binding finds and names the fault.
decltype(&gkv_prompt_attn) f_prompt_attn = nullptr;
decltype(&gkv_prompt_workspace_bytes) f_prompt_bytes = nullptr;
decltype(&gkv_prompt_mass) f_prompt_mass = nullptr;
decltype(&gkv_chunk_attn) f_chunk = nullptr;
PyObject* tensor_type = nullptr;     // torch.Tensor
PyObject* bf16_type = nullptr;       // torch.bfloat16
PyObject* f32_type = nullptr;        // torch.float32
PyObject* get_device = nullptr;      // the current device
PyObject* get_stream = nullptr;      // a device's current stream
PyObject* capturing = nullptr;       // is it being captured?
PyObject *s_shape = nullptr, *s_stride = nullptr, *s_dtype = nullptr, *s_get_device = nullptr;

// bind_rows(prompt_attn, prompt_workspace_bytes, prompt_mass, chunk_attn, Tensor, bfloat16, float32, current device, current stream, is it captured)
PyObject* py_bind_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* p[4];
  if (!want(n, 10)) return nullptr;
  for (int i = 0; i < 4; ++i)
    if (!as_plain(a[i], &p[i])) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_TypeError, "an address is needed");
  f_prompt_attn = reinterpret_cast<decltype(f_prompt_attn)>(p[0]);
  f_prompt_bytes = reinterpret_cast<decltype(f_prompt_bytes)>(p[1]);
  f_prompt_mass = reinterpret_cast<decltype(f_prompt_mass)>(p[2]);
  f_chunk = reinterpret_cast<decltype(f_chunk)>(p[3]);
  PyObject** const kept[6] = {&tensor_type, &bf16_type, &f32_type, &get_device, &get_stream, &capturing};
  for (int i = 0; i < 6; ++i) {
    Py_INCREF(a[4 + i]);
    Py_XSETREF(*kept[i], a[4 + i]);
  }
  Py_RETURN_NONE;
}

struct Rows {
  void* ptr;
  int64_t shape[4], stride[4];
  int dims;
};
bool as_i64s(PyObject* o, int64_t* out, int dims) {
  if (!o) return false;
  bool ok = PyTuple_Check(o) && PyTuple_GET_SIZE(o) == dims;
  for (int i = 0; ok && i < dims; ++i) {
    out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
    ok = out[i] >= 0;
  }
  Py_DECREF(o);
  return ok && !PyErr_Occurred();
}
// a plain CUDA tensor of that type and device with so many dimensions
bool as_rows(PyObject* o, PyObject* dtype, long dev, int dims, Rows* r) {
  if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != tensor_type) return false;
  PyObject* v = PyObject_GetAttr(o, s_dtype);
  Py_XDECREF(v);                     // (types are singletons)
  if (v != dtype) return false;
  if (!(v = PyObject_CallMethodNoArgs(o, s_get_device))) return false;
  const long on = PyLong_AsLong(v);
  Py_DECREF(v);
  r->dims = dims;
  return on == dev && as_i64s(PyObject_GetAttr(o, s_shape), r->shape, dims) && as_i64s(PyObject_CallMethodNoArgs(o, s_stride), r->stride, dims) &&
         as_address(o, &r->ptr);
}
bool packed(const Rows& r) {
  int64_t step = 1;
  for (int i = r.dims; i-- > 0; step *= r.shape[i])
    if (r.shape[i] != 1 && r.stride[i] != step) return false;
  return true;
}
bool shaped(const Rows& r, int64_t a, int64_t b, int64_t c, int64_t d = 0) {
  return r.shape[0] == a && r.shape[1] == b && (r.dims < 3 || r.shape[2] == c) && (r.dims < 4 || r.shape[3] == d);
}
// [rows][heads][128] whose heads follow one another, and how far its rows are apart
bool heads_together(const Rows& r, int64_t* step) {
  if (r.shape[0] == 0 || r.shape[1] == 0 || r.shape[2] != 128 || r.stride[2] != 1 || (r.shape[1] > 1 && r.stride[1] != 128)) return false;
  *step = r.shape[0] > 1 ? r.stride[0] : r.shape[1] * 128;
  if (*step < r.shape[1] * 128) return false;      // (rows that share memory; 0 would mean packed rows)
  return true;
}
// a contiguous array of 32-bit integers (numpy's, as a rule)
struct Ints {
  Py_buffer view{};
  const int32_t* data = nullptr;
  int64_t n = 0;
  bool take(PyObject* o) {
    if (PyObject_GetBuffer(o, &view, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) != 0) return false;
    data = static_cast<const int32_t*>(view.buf);
    n = view.len / 4;
    return view.ndim == 1 && view.itemsize == 4 && view.format && (view.format[0] == 'i' || view.format[0] == 'l') && !view.format[1];
  }
  ~Ints() {
    if (view.obj) PyBuffer_Release(&view);
  }
};
bool here(long* dev, void** st) {
  PyObject* d = PyObject_CallNoArgs(get_device);
  if (!d) return false;
  *dev = PyLong_AsLong(d);
  PyObject* v = PyObject_CallOneArg(get_stream, d);
  Py_DECREF(d);
  if (!v) return false;
  const bool ok = as_plain(v, st);
  Py_DECREF(v);
  return ok && *dev >= 0;
}
bool describe(gkv_prompt* d, const Rows& q, const Rows& k, const Ints& off, PyObject* scale) {
  if (off.n < 1 || off.data[off.n - 1] > q.shape[0] || k.shape[0] != q.shape[0]) return false;
  *d = gkv_prompt{};
  d->struct_size = sizeof(gkv_prompt);
  d->abi_version = GKV_ABI_VERSION;
  d->n_seqs = static_cast<int32_t>(off.n - 1);
  d->n_q_heads = static_cast<int32_t>(q.shape[1]);
  d->n_kv_heads = static_cast<int32_t>(k.shape[1]);
  d->head_dim = 128;
  d->offsets = off.data;
  const double x = PyFloat_AsDouble(scale);
  d->softmax_scale = static_cast<float>(x);
  return !PyErr_Occurred();
}

// prompt_attn(q, k, v, out, offsets, lse, softmax_scale, workspaces) -> status, or the bytes of workspace that the caller has to bring.
// workspaces: a tuple (address, bytes, ...), or a dict of them by 64 * stream + device, which is not looked at while the stream is captured
PyObject* py_prompt_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!want(n, 8)) return nullptr;
  long dev;
  void* st;
  Rows q, k, v, out, lse{};
  Ints off;
  gkv_prompt d;
  if (!here(&dev, &st) || !as_rows(a[0], bf16_type, dev, 3, &q) || !as_rows(a[1], bf16_type, dev, 3, &k) || !as_rows(a[2], bf16_type, dev, 3, &v) ||
      !as_rows(a[3], bf16_type, dev, 3, &out) || !off.take(a[4]) || (a[5] != Py_None && !as_rows(a[5], f32_type, dev, 2, &lse)) ||
      !describe(&d, q, k, off, a[6]) || !heads_together(q, &d.q_stride) || !heads_together(k, &d.k_stride) || !heads_together(v, &d.v_stride) ||
      !heads_together(out, &d.out_stride) || !shaped(v, k.shape[0], k.shape[1], 128) || !shaped(out, q.shape[0], q.shape[1], 128) ||
      (a[5] != Py_None && (!packed(lse) || !shaped(lse, q.shape[0], q.shape[1], 0))))
    return refuse();
  size_t need = 0, have = 0;
  void* ws = nullptr;
  PyObject* held = nullptr;                // the workspace's owner: while the launches are made another thread may put a new one into its place
  int rc = f_prompt_bytes(&d, &need);
  if (rc == GKV_OK && need > 0) {
    PyObject* space = a[7];
    if (PyDict_Check(space)) {
      PyObject* busy = PyObject_CallNoArgs(capturing);
      if (!busy) return nullptr;
      const bool captured = PyObject_IsTrue(busy) != 0;
      Py_DECREF(busy);
      PyObject* key = PyLong_FromUnsignedLongLong((reinterpret_cast<unsigned long long>(st) << 6) + static_cast<unsigned long long>(dev));
      if (!key) return nullptr;
      space = captured ? nullptr : PyDict_GetItemWithError(a[7], key);
      Py_DECREF(key);
    }
    if (space && PyTuple_Check(space) && PyTuple_GET_SIZE(space) >= 2 && as_plain(PyTuple_GET_ITEM(space, 0), &ws)) have = PyLong_AsSize_t(PyTuple_GET_ITEM(space, 1));
    if (PyErr_Occurred()) return refuse();
    if (have < need) return PyLong_FromSize_t(need);
    held = space;
    Py_INCREF(held);
  }
  if (rc == GKV_OK) {
    Py_BEGIN_ALLOW_THREADS
    rc = f_prompt_attn(&d, q.ptr, k.ptr, v.ptr, out.ptr, static_cast<float*>(lse.ptr), ws, have, st);
    Py_END_ALLOW_THREADS
  }
  Py_XDECREF(held);
  return PyLong_FromLong(rc);
}

// prompt_mass(q, k, lse, mass, mass's dimensions, offsets, n_obs, softmax_scale)
PyObject* py_prompt_mass(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!want(n, 8)) return nullptr;
  long dev;
  void* st;
  Rows q, k, lse, mass{};
  Ints off;
  gkv_prompt d;
  int32_t dims, n_obs;
  if (!here(&dev, &st) || !as_int(a[4], &dims) || dims < 1 || dims > 4 || !as_int(a[6], &n_obs) || !as_rows(a[0], bf16_type, dev, 3, &q) ||
      !as_rows(a[1], bf16_type, dev, 3, &k) || !as_rows(a[2], f32_type, dev, 2, &lse) || !as_rows(a[3], f32_type, dev, dims, &mass) || !off.take(a[5]) ||
      !describe(&d, q, k, off, a[7]) || !heads_together(q, &d.q_stride) || !heads_together(k, &d.k_stride) || !packed(lse) ||
      !shaped(lse, q.shape[0], q.shape[1], 0) || !packed(mass))
    return refuse();
  int64_t room = 1;
  for (int i = 0; i < dims; ++i) room *= mass.shape[i];
  if (room < (static_cast<int64_t>(off.data[off.n - 1]) - off.data[0]) * k.shape[1]) return refuse();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f_prompt_mass(&d, q.ptr, k.ptr, static_cast<const float*>(lse.ptr), n_obs, static_cast<float*>(mass.ptr), st);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// chunk(handle, layer, q, k_new, v_new, out, lse, lengths, workspace, its bytes, batch, query heads, KV heads, stream or None = the current one, device)
PyObject* py_chunk(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!want(n, 15)) return nullptr;
  gkv_cache* h;
  int32_t layer, b, hq, hkv, on;
  long dev;
  void *st, *ws, *given;
  Rows q, k, v, out, lse{};
  Ints len;
  if (!here(&dev, &st) || !as_handle(a[0], &h) || !as_int(a[1], &layer) || !as_rows(a[2], bf16_type, dev, 4, &q) || !as_rows(a[3], bf16_type, dev, 4, &k) ||
      !as_rows(a[4], bf16_type, dev, 4, &v) || !as_rows(a[5], bf16_type, dev, 4, &out) || (a[6] != Py_None && !as_rows(a[6], f32_type, dev, 3, &lse)) ||
      (a[7] != Py_None && !len.take(a[7])) || !as_plain(a[8], &ws) || !PyLong_Check(a[9]) || !as_int(a[10], &b) || !as_int(a[11], &hq) || !as_int(a[12], &hkv) ||
      !as_plain(a[13], &given) || !as_int(a[14], &on) || on != dev || q.shape[1] > INT32_MAX)
    return refuse();
  const int64_t m = q.shape[1];
  if (!shaped(q, b, m, hq, 128) || !shaped(k, b, m, hkv, 128) || !shaped(v, b, m, hkv, 128) || !shaped(out, b, m, hq, 128) || !packed(q) || !packed(k) ||
      !packed(v) || !packed(out) || (a[6] != Py_None && (!shaped(lse, b, m, hq) || !packed(lse))) || (a[7] != Py_None && len.n != b))
    return refuse();
  const size_t bytes = PyLong_AsSize_t(a[9]);
  if (PyErr_Occurred()) return refuse();
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f_chunk(h, layer, q.ptr, k.ptr, v.ptr, static_cast<int32_t>(m), len.data, out.ptr, static_cast<float*>(lse.ptr), ws, bytes, a[13] == Py_None ? st : given);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

#define GKV_FAST(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {GKV_FAST("bind", py_bind),       GKV_FAST("append", py_append), GKV_FAST("decode", py_decode),
                         GKV_FAST("observe", py_observe), GKV_FAST("select", py_select),
                         GKV_FAST("bind_rows", py_bind_rows), GKV_FAST("prompt_attn", py_prompt_attn), GKV_FAST("prompt_mass", py_prompt_mass),
                         GKV_FAST("chunk", py_chunk),     {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_gkv_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__gkv_call() {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_value = PyUnicode_InternFromString("value");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_get_device = PyUnicode_InternFromString("get_device");
  return s_data_ptr && s_value && s_shape && s_stride && s_dtype && s_get_device ? PyModule_Create(&module) : nullptr;
}
