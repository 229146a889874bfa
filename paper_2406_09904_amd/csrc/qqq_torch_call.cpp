// The two linear calls of binding.py, and those of qqq_layer.h, from tensors to the C ABI in one step of native code.  A one-row call takes the GPU 4.8 us and
// took Python 6.3 to marshal (a method call per data pointer, contiguity, type and size, ctypes' conversions): calls in a row 6.34 us each, 5.35 so.
// Only the plain case is handled: dense tensors that are exactly torch.Tensor, on the GPU, as the call wants them.  Anything else (a subclass, a
// wrapper without storage, a function mode, a wrong type or stride, a failed allocation) returns None, and binding.py's own path, which decides what is
// accepted and raises, takes the call.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <exception>
#include <type_traits>

#include "qqq_layer.h"

namespace {

using PerChannel = int (*)(const void*, int64_t, const void*, const void*, void*, int32_t*, int64_t, int64_t, int64_t, void*, size_t, void*);
using PerGroup = int (*)(const void*, int64_t, const void*, const int8_t*, const void*, int, int, void*, int32_t*, int64_t, int64_t, int64_t, void*,
                         size_t, void*);
PerChannel per_channel = nullptr;
PerGroup per_group = nullptr;

const at::Tensor* plain(PyObject* o, at::ScalarType type) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.has_storage() || !t.is_cuda() || t.layout() != at::kStrided || t.scalar_type() != type ||
      t.unsafeGetTensorImpl()->is_python_dispatch())
    return nullptr;
  return &t;
}
const at::Tensor* dense(PyObject* o, at::ScalarType type) {
  const at::Tensor* t = plain(o, type);
  return t && t->is_contiguous() ? t : nullptr;
}

// linear(a_fp16, w_packed, s_g or None, s_w, workspace, y or None, acc_out or None, group, sg_max, stream)
// -> the output, an error code, or None: not a plain call
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 10) Py_RETURN_NONE;
  const bool grouped = args[2] != Py_None;
  if (!(grouped ? per_group != nullptr : per_channel != nullptr)) Py_RETURN_NONE;
  try {
    if (at::impl::PythonTorchFunctionTLS::stack_len() > 0) Py_RETURN_NONE;
    const at::Tensor* a = plain(args[0], at::kHalf);
    const at::Tensor* w = dense(args[1], at::kByte);
    const at::Tensor* s_g = grouped ? dense(args[2], at::kChar) : nullptr;
    const at::Tensor* s_w = dense(args[3], at::kHalf);
    const at::Tensor* ws = dense(args[4], at::kByte);
    const at::Tensor* acc = args[6] == Py_None ? nullptr : dense(args[6], at::kInt);
    if (!a || !w || !s_w || !ws || (grouped && !s_g) || (args[6] != Py_None && !acc) || a->dim() != 2 || s_w->dim() < 1 || a->stride(1) != 1)
      Py_RETURN_NONE;
    const int64_t M = a->size(0), K = a->size(1), N = s_w->size(0);
    const int64_t lda = M > 1 || a->stride(0) > K ? a->stride(0) : K;
    const long group = PyLong_AsLong(args[7]), sg_max = PyLong_AsLong(args[8]);
    void* const stream = PyLong_AsVoidPtr(args[9]);
    if (PyErr_Occurred() || group != (int)group || sg_max != (int)sg_max) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    at::Tensor made;
    const at::Tensor* y = nullptr;
    if (args[5] == Py_None) {
      made = at::empty({M, N}, a->options());
      y = &made;
    } else {
      y = dense(args[5], at::kHalf);
    }
    if (!y) Py_RETURN_NONE;
    void *pa = a->data_ptr(), *pw = w->data_ptr(), *ps = s_w->data_ptr(), *py = y->data_ptr(), *pws = ws->data_ptr();
    const int8_t* pg = grouped ? static_cast<const int8_t*>(s_g->data_ptr()) : nullptr;
    int32_t* pacc = acc ? static_cast<int32_t*>(acc->data_ptr()) : nullptr;
    const size_t bytes = static_cast<size_t>(ws->numel());
    int rc;
    Py_BEGIN_ALLOW_THREADS;  // (as ctypes does)
    rc = grouped ? per_group(pa, lda, pw, pg, ps, (int)group, (int)sg_max, py, pacc, M, N, K, pws, bytes, stream)
                 : per_channel(pa, lda, pw, ps, py, pacc, M, N, K, pws, bytes, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    if (args[5] != Py_None) {
      Py_INCREF(args[5]);
      return args[5];
    }
    return THPVariable_Wrap(made);
  } catch (const std::exception&) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// bind(address of qqq_linear_w4a8_perchannel, of qqq_linear_w4a8_pergroup)
PyObject* bind(PyObject*, PyObject* args) {
  unsigned long long pc = 0, pg = 0;
  if (!PyArg_ParseTuple(args, "KK", &pc, &pg)) return nullptr;
  per_channel = reinterpret_cast<PerChannel>(static_cast<uintptr_t>(pc));
  per_group = reinterpret_cast<PerGroup>(static_cast<uintptr_t>(pg));
  Py_RETURN_NONE;
}

// ---- qqq_layer.h, in the same way: what a decoder layer does between its linear calls takes a few microseconds of the GPU for one token, and
// Python took 6 (norm) to 19 (attention: twelve tensors) to marshal

struct {
  decltype(&qqq_add_rmsnorm) norm;
  decltype(&qqq_add_rmsnorm_quant) norm_quant;
  decltype(&qqq_gated_act_quant) gated;
  decltype(&qqq_kv8_append) append;
  decltype(&qqq_kv8_read) read;
  decltype(&qqq_attention_kv8_workspace_bytes) attention_bytes;
  decltype(&qqq_attention_kv8) attention;
} layer = {};

bool plain_world() { return at::impl::PythonTorchFunctionTLS::stack_len() == 0; }

// rows of unit inner stride
const at::Tensor* rows(PyObject* o, at::ScalarType type) {
  const at::Tensor* t = plain(o, type);
  return t && t->dim() == 2 && t->stride(1) == 1 ? t : nullptr;
}
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 || t.stride(0) > t.size(1) ? t.stride(0) : t.size(1); }
bool is_shape(const at::Tensor& t, at::IntArrayRef shape) { return t.sizes() == shape; }

// the given output, or a new one; nullptr: not a plain one
const at::Tensor* output(PyObject* o, at::ScalarType type, at::IntArrayRef shape, const at::Tensor& like, at::Tensor& made) {
  if (o == Py_None) {
    made = at::empty(shape, like.options().dtype(type));
    return &made;
  }
  const at::Tensor* t = dense(o, type);
  return t && is_shape(*t, shape) ? t : nullptr;
}
PyObject* given_or(PyObject* o, at::Tensor& made) {
  if (o == Py_None) return THPVariable_Wrap(made);
  Py_INCREF(o);
  return o;
}
PyObject* none() {
  Py_INCREF(Py_None);
  return Py_None;
}
PyObject* tuple_of(PyObject* a, PyObject* b, PyObject* c = nullptr) {
  PyObject* t = a && b ? PyTuple_New(c ? 3 : 2) : nullptr;
  if (!t) {
    Py_XDECREF(a);
    Py_XDECREF(b);
    Py_XDECREF(c);
    return nullptr;
  }
  PyTuple_SET_ITEM(t, 0, a);
  PyTuple_SET_ITEM(t, 1, b);
  if (c) PyTuple_SET_ITEM(t, 2, c);
  return t;
}

// rmsnorm(x, gain, residual or None, eps, sum_out or None, y or a_q or None, s_a or None, quantise, stream)
// -> (sum or None, y) or (sum or None, a_q, s_a), an error code, or None: not a plain call
PyObject* rmsnorm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 9 || !layer.norm || !layer.norm_quant) Py_RETURN_NONE;
  try {
    if (!plain_world()) Py_RETURN_NONE;
    const bool quantise = args[7] == Py_True, has = args[2] != Py_None;
    const at::Tensor *x = rows(args[0], at::kHalf), *gain = dense(args[1], at::kHalf);
    if (!x || !gain || !PyFloat_CheckExact(args[3]) || (!has && args[4] != Py_None)) Py_RETURN_NONE;
    const int64_t M = x->size(0), K = x->size(1);
    if (!is_shape(*gain, {K})) Py_RETURN_NONE;
    const at::Tensor *res = nullptr, *sum = nullptr;
    at::Tensor made_sum, made_out, made_s;
    if (has) {
      res = rows(args[2], at::kHalf);
      if (!res) res = rows(args[2], at::kFloat);
      if (!res || !is_shape(*res, x->sizes())) Py_RETURN_NONE;
      if (args[4] == Py_None) {
        made_sum = at::empty({M, K}, res->options());
        sum = &made_sum;
      } else {
        sum = rows(args[4], res->scalar_type());
      }
      if (!sum || !is_shape(*sum, x->sizes())) Py_RETURN_NONE;
    }
    const at::Tensor* out = output(args[5], quantise ? at::kChar : at::kHalf, {M, K}, *x, made_out);
    const at::Tensor* s_a = quantise ? output(args[6], at::kFloat, {M}, *x, made_s) : nullptr;
    void* const stream = PyLong_AsVoidPtr(args[8]);
    const float eps = (float)PyFloat_AS_DOUBLE(args[3]);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    if (!out || (quantise && !s_a)) Py_RETURN_NONE;
    const int kind = !has ? QQQ_RESIDUAL_NONE : res->scalar_type() == at::kHalf ? QQQ_RESIDUAL_FP16 : QQQ_RESIDUAL_FP32;
    const void *px = x->data_ptr(), *pr = has ? res->data_ptr() : nullptr, *pg = gain->data_ptr();
    void *ps = has ? sum->data_ptr() : nullptr, *po = out->data_ptr();
    float* pa = quantise ? static_cast<float*>(s_a->data_ptr()) : nullptr;
    const int64_t ldx = row_stride(*x), ldr = has ? row_stride(*res) : 0, lds = has ? row_stride(*sum) : 0;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = quantise ? layer.norm_quant(px, ldx, pr, ldr, kind, pg, eps, M, K, ps, lds, static_cast<int8_t*>(po), pa, stream)
                  : layer.norm(px, ldx, pr, ldr, kind, pg, eps, M, K, ps, lds, po, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    PyObject* total = has ? given_or(args[4], made_sum) : none();
    return quantise ? tuple_of(total, given_or(args[5], made_out), given_or(args[6], made_s)) : tuple_of(total, given_or(args[5], made_out));
  } catch (const std::exception&) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// gated(gate, up, act, a_q or None, s_a or None, stream) -> (a_q, s_a), an error code, or None
PyObject* gated(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 6 || !layer.gated) Py_RETURN_NONE;
  try {
    if (!plain_world()) Py_RETURN_NONE;
    const at::Tensor *gate = rows(args[0], at::kHalf), *up = rows(args[1], at::kHalf);
    if (!gate || !up || !is_shape(*up, gate->sizes())) Py_RETURN_NONE;
    const int64_t M = gate->size(0), F = gate->size(1);
    at::Tensor made_q, made_s;
    const at::Tensor *a_q = output(args[3], at::kChar, {M, F}, *gate, made_q), *s_a = output(args[4], at::kFloat, {M}, *gate, made_s);
    const long act = PyLong_AsLong(args[2]);
    void* const stream = PyLong_AsVoidPtr(args[5]);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    if (!a_q || !s_a) Py_RETURN_NONE;
    const void *pg = gate->data_ptr(), *pu = up->data_ptr();
    int8_t* pq = static_cast<int8_t*>(a_q->data_ptr());
    float* ps = static_cast<float*>(s_a->data_ptr());
    const int64_t ldg = row_stride(*gate), ldu = row_stride(*up);
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = layer.gated(pg, ldg, pu, ldu, (int)act, M, F, pq, ps, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    return tuple_of(given_or(args[3], made_q), given_or(args[4], made_s));
  } catch (const std::exception&) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// the structs of a KV8Cache and a KV8Batch; false: not plain ones
bool kv8_structs(PyObject* cache, PyObject* batch, qqq_kv8_cache& c, qqq_kv8_batch& b, const at::Tensor** codes) {
  if (!PyTuple_Check(cache) || PyTuple_GET_SIZE(cache) != 6 || !PyTuple_Check(batch) || PyTuple_GET_SIZE(batch) != 6) return false;
  const at::Tensor *kc = dense(PyTuple_GET_ITEM(cache, 0), at::kByte), *ks = dense(PyTuple_GET_ITEM(cache, 1), at::kFloat);
  const at::Tensor *vc = dense(PyTuple_GET_ITEM(cache, 2), at::kByte), *vs = dense(PyTuple_GET_ITEM(cache, 3), at::kFloat);
  const at::Tensor *kt = dense(PyTuple_GET_ITEM(cache, 4), at::kHalf), *vt = dense(PyTuple_GET_ITEM(cache, 5), at::kHalf);
  PyObject* const slots_o = PyTuple_GET_ITEM(batch, 3);
  const at::Tensor *table = rows(PyTuple_GET_ITEM(batch, 0), at::kInt), *len = dense(PyTuple_GET_ITEM(batch, 1), at::kInt);
  const at::Tensor *cu = dense(PyTuple_GET_ITEM(batch, 2), at::kInt), *slots = slots_o == Py_None ? nullptr : dense(slots_o, at::kInt);
  if (!kc || !ks || !vc || !vs || !kt || !vt || !table || !len || !cu || (slots_o != Py_None && !slots) || kc->dim() != 4 || kt->dim() != 4) return false;
  const int64_t pages = kc->size(0), H = kc->size(1), P = kc->size(2), D = kc->size(3), B = table->size(0), nslots = kt->size(0);
  if (!is_shape(*vc, {pages, H, D, P}) || !is_shape(*ks, {pages, H}) || !is_shape(*vs, {pages, H}) || !is_shape(*kt, {nslots, H, P, D}) ||
      !is_shape(*vt, {nslots, H, D, P}) || !is_shape(*len, {B}) || !is_shape(*cu, {B + 1}) || (slots ? !is_shape(*slots, {B}) : nslots < B) ||
      H > 0x7FFFFFFF || P > 64 || D > 256 || B > 0x7FFFFFFF || nslots > 0x7FFFFFFF || table->size(1) > 0x7FFFFFFF)
    return false;
  const long max_new = PyLong_AsLong(PyTuple_GET_ITEM(batch, 4)), max_len = PyLong_AsLong(PyTuple_GET_ITEM(batch, 5));
  if (PyErr_Occurred() || max_new != (int32_t)max_new || max_len != (int32_t)max_len) {
    PyErr_Clear();
    return false;
  }
  c = {static_cast<uint8_t*>(kc->data_ptr()), static_cast<float*>(ks->data_ptr()), static_cast<uint8_t*>(vc->data_ptr()), static_cast<float*>(vs->data_ptr()),
       kt->data_ptr(), vt->data_ptr(), pages, (int32_t)nslots, (int32_t)H, (int32_t)D, (int32_t)P};
  b = {static_cast<int32_t*>(table->data_ptr()), row_stride(*table), static_cast<int32_t*>(len->data_ptr()), static_cast<int32_t*>(cu->data_ptr()),
       slots ? static_cast<int32_t*>(slots->data_ptr()) : nullptr, (int32_t)table->size(1), (int32_t)B, (int32_t)max_new, (int32_t)max_len};
  *codes = kc;
  return true;
}
const at::Tensor* heads_of(PyObject* o, int64_t heads, int64_t D) {
  const at::Tensor* t = plain(o, at::kHalf);
  return t && t->dim() == 3 && t->stride(2) == 1 && t->size(2) == D && (heads == 0 || t->size(1) == heads) ? t : nullptr;
}

// strides of [tokens, heads, D]; of an axis of one entry it may be anything, and is not used
int64_t token_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : 0; }
int64_t head_stride(const at::Tensor& t) { return t.size(1) > 1 ? t.stride(1) : 0; }

// append(cache, batch, k, v, stream) -> an error code (0 too), or None
PyObject* append(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 5 || !layer.append) Py_RETURN_NONE;
  try {
    qqq_kv8_cache c;
    qqq_kv8_batch b;
    const at::Tensor* codes;
    if (!plain_world() || !kv8_structs(args[0], args[1], c, b, &codes)) Py_RETURN_NONE;
    const at::Tensor *k = heads_of(args[2], c.kv_heads, c.head_dim), *v = heads_of(args[3], c.kv_heads, c.head_dim);
    void* const stream = PyLong_AsVoidPtr(args[4]);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    if (!k || !v || k->size(0) != v->size(0)) Py_RETURN_NONE;
    const void *pk = k->data_ptr(), *pv = v->data_ptr();
    const int64_t kt = token_stride(*k), kh = head_stride(*k), vt = token_stride(*v), vh = head_stride(*v), T = k->size(0);
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = layer.append(&c, &b, pk, kt, kh, pv, vt, vh, T, stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
  } catch (const std::exception&) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// read(cache, batch, k, v, stream) -> an error code (0 too), or None
PyObject* read(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 5 || !layer.read) Py_RETURN_NONE;
  try {
    qqq_kv8_cache c;
    qqq_kv8_batch b;
    const at::Tensor* codes;
    if (!plain_world() || !kv8_structs(args[0], args[1], c, b, &codes)) Py_RETURN_NONE;
    const at::Tensor *k = dense(args[2], at::kHalf), *v = dense(args[3], at::kHalf);
    void* const stream = PyLong_AsVoidPtr(args[4]);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    if (!k || !v || k->dim() != 3 || !is_shape(*k, {k->size(0), c.kv_heads, c.head_dim}) || !is_shape(*v, k->sizes())) Py_RETURN_NONE;
    void *pk = k->data_ptr(), *pv = v->data_ptr();
    const int64_t T = k->size(0);
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = layer.read(&c, &b, pk, pv, T, stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
  } catch (const std::exception&) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// attention(cache, batch, q, scale or None, causal, window, out or None, lse or None, workspace or None, stream)
// -> (out, lse or None), an error code, or None
PyObject* attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 10 || !layer.attention || !layer.attention_bytes) Py_RETURN_NONE;
  try {
    qqq_kv8_cache c;
    qqq_kv8_batch b;
    const at::Tensor* codes;
    if (!plain_world() || !kv8_structs(args[0], args[1], c, b, &codes)) Py_RETURN_NONE;
    const at::Tensor* q = heads_of(args[2], 0, c.head_dim);
    if (!q || !(args[3] == Py_None || PyFloat_CheckExact(args[3])) || !PyBool_Check(args[4]) || !PyLong_CheckExact(args[5])) Py_RETURN_NONE;
    const int64_t T = q->size(0), Hq = q->size(1);
    const float scale = args[3] == Py_None ? (float)(1.0 / std::sqrt((double)c.head_dim)) : (float)PyFloat_AS_DOUBLE(args[3]);
    const long window = PyLong_AsLong(args[5]);
    void* const stream = PyLong_AsVoidPtr(args[9]);
    if (PyErr_Occurred() || window != (int)window || Hq != (int)Hq) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    at::Tensor made, lent;
    const at::Tensor* out = output(args[6], at::kHalf, q->sizes(), *q, made);
    const at::Tensor* lse = args[7] == Py_None ? nullptr : dense(args[7], at::kFloat);
    if (!out || (args[7] != Py_None && (!lse || !is_shape(*lse, {T, Hq})))) Py_RETURN_NONE;
    void* work = nullptr;
    size_t bytes = 0;
    if (args[8] == Py_None) {
      bytes = layer.attention_bytes(&c, &b, (int)Hq, T);
      if (bytes) {
        lent = at::empty({(int64_t)bytes}, q->options().dtype(at::kByte));
        work = lent.data_ptr();
      }
    } else {
      const at::Tensor* w = dense(args[8], at::kByte);
      if (!w) Py_RETURN_NONE;
      work = w->data_ptr();
      bytes = (size_t)w->numel();
    }
    const void* pq = q->data_ptr();
    void* po = out->data_ptr();
    float* pl = lse ? static_cast<float*>(lse->data_ptr()) : nullptr;
    const int64_t qt = token_stride(*q), qh = head_stride(*q);
    const int causal = args[4] == Py_True;
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = layer.attention(&c, &b, pq, qt, qh, (int)Hq, T, scale, causal, (int)window, po, pl, work, bytes, stream);
    Py_END_ALLOW_THREADS;
    if (rc != 0) return PyLong_FromLong(rc);
    Py_INCREF(args[7]);
    return tuple_of(given_or(args[6], made), args[7]);
  } catch (const std::exception&) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// bind_layer(addresses of the seven entry points, in the order of `layer`)
PyObject* bind_layer(PyObject*, PyObject* args) {
  unsigned long long a[7] = {};
  if (!PyArg_ParseTuple(args, "KKKKKKK", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6)) return nullptr;
  auto set = [&](auto& f, int i) { f = reinterpret_cast<std::decay_t<decltype(f)>>(static_cast<uintptr_t>(a[i])); };
  set(layer.norm, 0);
  set(layer.norm_quant, 1);
  set(layer.gated, 2);
  set(layer.append, 3);
  set(layer.read, 4);
  set(layer.attention_bytes, 5);
  set(layer.attention, 6);
  Py_RETURN_NONE;
}

template <typename F>
PyMethodDef fast(const char* name, F f) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {fast("rmsnorm", rmsnorm), fast("gated", gated), fast("append", append), fast("read", read), fast("attention", attention),
                         {"bind_layer", bind_layer, METH_VARARGS, nullptr},
                         {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(linear)), METH_FASTCALL, nullptr},
                         {"bind", bind, METH_VARARGS, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_qqq_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__qqq_call(void) { return PyModule_Create(&module); }
