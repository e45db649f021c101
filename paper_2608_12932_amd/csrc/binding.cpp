// Native fast path of the Python binding: the hot entry points of w4a8.h on
// torch tensors, on the current stream.
//
// The calls of the decode and verify steps run for 2 - 10 us on the GPU, and
// argument checks, the stream lookup, the output's allocation and the
// foreign-function call took 9 - 18 us of interpreted Python per call, so
// consecutive calls were bound by the host.  Here they take about 1 us
// beyond the launches.
//
// Each function returns None for anything but the plain case (a tensor
// subclass, another stream's workspace, a wrong type or shape ...): the
// interpreted path in __init__.py then takes the call, grows the workspace
// or raises the error.  An int is a nonzero status of the library call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "w4a8.h"

namespace {

// a plain, contiguous device tensor of the given type; nullptr otherwise
const at::Tensor* plain(PyObject* o, at::ScalarType type) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() && t.scalar_type() == type && t.is_contiguous() ? &t : nullptr;
}

bool is_int(PyObject* o) { return PyLong_CheckExact(o); }
int64_t as_int(PyObject* o) { return PyLong_AsLongLong(o); }  // -1 with an error set past 64 bits

hipStream_t current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// Runs f without the interpreter's lock, also where it throws: launches may
// wait for room in the queue, allocations for the allocator's lock, whose
// holder may itself be waiting for the interpreter's.
template <class F>
w4a8_status without_gil(F f) {
  struct Released {
    PyThreadState* state = PyEval_SaveThread();
    ~Released() { PyEval_RestoreThread(state); }
  } released;
  return f();
}

// linear(swiglu, x, w_packed, w_scale, N, x_scale, scale_mode, out_kind, out,
//        workspace, workspace_stream, is_workspace)
// workspace_stream: the stream that a Workspace's buffer (is_workspace)
// belongs to, None while it is empty or that is not known (a copy's).  A
// negative int is the size that an
// otherwise plain call's Workspace has to grow to.
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 12 || !is_int(a[0]) || !is_int(a[4]) || !is_int(a[6]) || !is_int(a[7])) Py_RETURN_NONE;
  const bool swiglu = as_int(a[0]) != 0;
  const int64_t N = as_int(a[4]), mode = as_int(a[6]), kind = as_int(a[7]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  if (mode < 0 || mode > 1 || kind < 0 || kind > 2 || N <= 0) Py_RETURN_NONE;
  const at::Tensor* x = plain(a[1], at::kBFloat16);
  const at::Tensor* xs = nullptr;
  int in_kind = W4A8_IN_BF16;
  if (!x) {
    x = plain(a[1], at::kChar);
    xs = x ? plain(a[5], at::kFloat) : nullptr;
    if (!xs) Py_RETURN_NONE;
    in_kind = W4A8_IN_I8;
  }
  const at::Tensor* wp = plain(a[2], at::kByte);
  if (!wp || x->dim() != 2) Py_RETURN_NONE;
  const at::Tensor* ws = nullptr;
  if (a[3] != Py_None && !(ws = plain(a[3], mode == W4A8_SCALE_CHANNEL_F32 ? at::kFloat : at::kHalf))) Py_RETURN_NONE;
  const int64_t M = x->size(0), K = x->size(1), cols = swiglu ? N / 2 : N;
  const at::ScalarType out_type = kind == W4A8_OUT_BF16 ? at::kBFloat16 : kind == W4A8_OUT_F32 ? at::kFloat : at::kInt;

  const at::Tensor* out = nullptr;
  if (a[8] != Py_None) {
    out = plain(a[8], out_type);
    if (!out || out->dim() != 2 || out->size(0) != M || out->size(1) != cols) Py_RETURN_NONE;
  }

  const size_t need = swiglu ? w4a8_linear_swiglu_workspace_bytes(M, N, K, (int)mode, in_kind)
                             : w4a8_linear_workspace_bytes(M, N, K, (int)mode, in_kind);
  const hipStream_t stream = current_stream();
  void* wk = nullptr;
  size_t wk_bytes = 0;
  const bool temporary = need && a[9] == Py_None && a[11] != Py_True;
  if (need && !temporary) {
    const at::Tensor* buf = plain(a[9], at::kByte);
    if (!buf) Py_RETURN_NONE;
    if (a[11] == Py_True) {  // a Workspace: of this stream (its memory is ordered on it), and large enough
      if (a[10] != Py_None && (!is_int(a[10]) || PyLong_AsVoidPtr(a[10]) != (void*)stream)) {
        PyErr_Clear();
        Py_RETURN_NONE;
      }
      if ((size_t)buf->numel() < need) return PyLong_FromLongLong(-(long long)need);
      if (a[10] == Py_None) Py_RETURN_NONE;
    }
    wk = buf->data_ptr();
    wk_bytes = (size_t)buf->numel();
  }

  const void *xp = x->data_ptr(), *sp = ws ? ws->data_ptr() : nullptr;
  const float* xsp = xs ? static_cast<const float*>(xs->data_ptr()) : nullptr;
  const uint8_t* wpp = static_cast<const uint8_t*>(wp->data_ptr());
  at::Tensor y;
  const w4a8_status s = without_gil([&] {
    y = out ? *out : at::empty({M, cols}, x->options().dtype(out_type));
    at::Tensor tmp;  // released to the allocator on this stream, which orders its next use
    if (temporary) {
      tmp = at::zeros({(int64_t)need}, x->options().dtype(at::kByte));
      wk = tmp.data_ptr();
      wk_bytes = need;
    }
    return (swiglu ? w4a8_linear_swiglu : w4a8_linear)(xp, in_kind, xsp, M, K, wpp, sp, (int)mode, N, y.data_ptr(), (int)kind,
                                                       wk, wk_bytes, stream);
  });
  if (s != W4A8_OK) return PyLong_FromLong(s);
  if (out) return Py_NewRef(a[8]);
  return THPVariable_Wrap(std::move(y));
  END_HANDLE_TH_ERRORS
}

// The current device, where the call's first tensor is on it; -1 otherwise.
c10::DeviceIndex device_of(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return -1;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() && t.get_device() == c10::hip::current_device() ? (c10::DeviceIndex)t.get_device() : -1;
}
// A tensor of the type, of `dim` axes, on the device that the call runs on;
// its last axis alone has to be contiguous.  nullptr otherwise.
const at::Tensor* rows_of(PyObject* o, at::ScalarType type, int64_t dim, c10::DeviceIndex device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() && t.scalar_type() == type && t.dim() == dim && t.get_device() == device &&
                 (t.numel() == 0 || t.stride(dim - 1) == 1)
             ? &t
             : nullptr;
}
// The same, contiguous throughout.
const at::Tensor* whole(PyObject* o, at::ScalarType type, int64_t dim, c10::DeviceIndex device) {
  const at::Tensor* t = rows_of(o, type, dim, device);
  return t && t->is_contiguous() ? t : nullptr;
}
template <class T>
T* ptr(const at::Tensor* t) {
  return t ? static_cast<T*>(t->data_ptr()) : nullptr;
}

// add_norm(x, residual, gamma, eps, out) -> (codes, scales, sum)
PyObject* add_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 5 || !PyFloat_CheckExact(a[3])) Py_RETURN_NONE;
  const c10::DeviceIndex device = device_of(a[0]);
  if (device < 0) Py_RETURN_NONE;
  const at::Tensor *x = whole(a[0], at::kBFloat16, 2, device), *r = whole(a[1], at::kBFloat16, 2, device),
                   *g = whole(a[2], at::kBFloat16, 1, device), *out = nullptr;
  if (!x || !r || !g) Py_RETURN_NONE;
  const int64_t M = x->size(0), K = x->size(1);
  auto fits = [&](const at::Tensor& t) { return t.size(0) == M && t.size(1) == K; };
  if (!fits(*r) || g->size(0) != K) Py_RETURN_NONE;
  if (a[4] != Py_None && (!(out = whole(a[4], at::kBFloat16, 2, device)) || !fits(*out))) Py_RETURN_NONE;
  const float eps = (float)PyFloat_AS_DOUBLE(a[3]);
  at::Tensor q, s, sum;
  const hipStream_t stream = current_stream();
  const w4a8_status st = without_gil([&] {
    q = at::empty({M, K}, x->options().dtype(at::kChar));
    s = at::empty({M}, x->options().dtype(at::kFloat));
    sum = out ? *out : at::empty({M, K}, x->options());
    return w4a8_add_rmsnorm_quantize_act(ptr<uint16_t>(x), ptr<uint16_t>(r), ptr<uint16_t>(g), eps, M, K, ptr<uint16_t>(&sum),
                                         ptr<int8_t>(&q), ptr<float>(&s), stream);
  });
  if (st != W4A8_OK) return PyLong_FromLong(st);
  PyObject* t = PyTuple_New(3);
  if (!t) return nullptr;
  PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(std::move(q)));
  PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(std::move(s)));
  PyTuple_SET_ITEM(t, 2, out ? Py_NewRef(a[4]) : THPVariable_Wrap(std::move(sum)));
  return t;
  END_HANDLE_TH_ERRORS
}

// The library's view of a KVCache (k_codes, v_codes, scales, k_recent,
// v_recent) and of a batch (starts, lengths, table, pos, rope_cos, rope_sin
// at b[0] ..) of T tokens; false for anything but the plain case.
bool cache_view(PyObject* o, bool rings, c10::DeviceIndex device, w4a8_cache& c) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 5) return false;
  auto item = [&](int i) { return PyTuple_GET_ITEM(o, i); };
  const at::Tensor *k = whole(item(0), at::kChar, 4, device), *v = whole(item(1), at::kChar, 4, device),
                   *s = whole(item(2), at::kFloat, 3, device);
  if (!k || !v || !s) return false;
  const int64_t pages = k->size(0), Hkv = k->size(1), D = k->size(3);
  if (k->size(2) != W4A8_CACHE_BLOCK || D != 128 || v->size(0) != pages || v->size(1) != Hkv || v->size(2) != D ||
      v->size(3) != W4A8_CACHE_BLOCK || s->size(0) != pages || s->size(1) != Hkv || s->size(2) != 2)
    return false;
  c = {ptr<int8_t>(k), ptr<int8_t>(v), ptr<float>(s), pages, Hkv, nullptr, nullptr, 0};
  if (rings) {
    const at::Tensor *kr = whole(item(3), at::kBFloat16, 4, device), *vr = whole(item(4), at::kBFloat16, 4, device);
    if (!kr || !vr || kr->sizes() != vr->sizes() || kr->size(1) != Hkv || kr->size(2) != W4A8_CACHE_RECENT || kr->size(3) != D)
      return false;
    c.k_recent = ptr<uint16_t>(kr);
    c.v_recent = ptr<uint16_t>(vr);
    c.n_slots = kr->size(0);
  }
  return true;
}
bool batch_view(PyObject* const* b, int64_t T, c10::DeviceIndex device, w4a8_batch& out) {
  const at::Tensor *starts = whole(b[0], at::kInt, 1, device), *lengths = whole(b[1], at::kInt, 1, device),
                   *table = whole(b[2], at::kInt, 2, device), *pos = whole(b[3], at::kInt, 1, device),
                   *cs = whole(b[4], at::kFloat, 2, device), *sn = whole(b[5], at::kFloat, 2, device);
  if (!starts || !lengths || !table || !pos || !cs || !sn) return false;
  const int64_t B = lengths->size(0);
  if (starts->size(0) != B + 1 || table->size(0) != B || pos->size(0) != T || cs->sizes() != sn->sizes() || cs->size(1) != 64)
    return false;
  out = {ptr<int32_t>(starts), ptr<int32_t>(lengths), ptr<int32_t>(table), table->size(1), B, T, ptr<int32_t>(pos),
         ptr<float>(cs), ptr<float>(sn), cs->size(0)};
  return true;
}
// Token rows [T][heads][128]: the strides, that of an axis of one being free.
int64_t stride_of(const at::Tensor* t, int axis) { return t->size(axis) <= 1 ? 128 : t->stride(axis); }

// cache_append(k, v, cache, starts, lengths, table, pos, rope_cos, rope_sin, slots) -> True
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const c10::DeviceIndex device = n == 10 ? device_of(a[0]) : -1;
  if (device < 0) Py_RETURN_NONE;
  const at::Tensor *k = rows_of(a[0], at::kBFloat16, 3, device), *v = rows_of(a[1], at::kBFloat16, 3, device), *slots = nullptr;
  w4a8_cache c;
  w4a8_batch b;
  if (!k || !v || k->sizes() != v->sizes() || k->size(2) != 128 || !cache_view(a[2], true, device, c) || k->size(1) != c.Hkv ||
      !batch_view(a + 3, k->size(0), device, b))
    Py_RETURN_NONE;
  if (a[9] != Py_None && (!(slots = whole(a[9], at::kInt, 1, device)) || slots->size(0) != b.B)) Py_RETURN_NONE;
  const hipStream_t stream = current_stream();
  const w4a8_status s = without_gil([&] {
    return w4a8_cache_append(&c, &b, ptr<uint16_t>(k), stride_of(k, 0), stride_of(k, 1), ptr<uint16_t>(v), stride_of(v, 0),
                             stride_of(v, 1), ptr<int32_t>(slots), stream);
  });
  if (s != W4A8_OK) return PyLong_FromLong(s);
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

// cache_attention(q, cache, starts, lengths, table, pos, rope_cos, rope_sin,
//                 scale, max_len, out, workspace, workspace_stream, is_workspace)
// The last three and a negative answer are as for linear.
PyObject* cache_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const c10::DeviceIndex device = n == 14 ? device_of(a[0]) : -1;
  if (device < 0) Py_RETURN_NONE;
  const at::Tensor *q = rows_of(a[0], at::kBFloat16, 3, device), *out = nullptr;
  w4a8_cache c;
  w4a8_batch b;
  if (!q || q->size(2) != 128 || !cache_view(a[1], false, device, c) || !batch_view(a + 2, q->size(0), device, b) ||
      !PyFloat_CheckExact(a[8]))
    Py_RETURN_NONE;
  const int64_t T = b.T, H = q->size(1);
  int64_t max_len = b.max_blocks * W4A8_CACHE_BLOCK;
  if (a[9] != Py_None) {
    if (!is_int(a[9])) Py_RETURN_NONE;
    max_len = as_int(a[9]);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
  }
  if (a[10] != Py_None && (!(out = rows_of(a[10], at::kBFloat16, 3, device)) || out->sizes() != q->sizes())) Py_RETURN_NONE;
  const float scale = (float)PyFloat_AS_DOUBLE(a[8]);
  const hipStream_t stream = current_stream();
  const size_t need = w4a8_cache_attention_workspace_bytes(b.B, T, H, c.Hkv, max_len);
  void* wk = nullptr;
  size_t wk_bytes = 0;
  const bool temporary = need && a[11] == Py_None && a[13] != Py_True;
  if (need && !temporary) {
    const at::Tensor* buf = plain(a[11], at::kByte);
    if (!buf || buf->get_device() != device) Py_RETURN_NONE;
    if (a[13] == Py_True) {
      if (a[12] != Py_None && (!is_int(a[12]) || PyLong_AsVoidPtr(a[12]) != (void*)stream)) {
        PyErr_Clear();
        Py_RETURN_NONE;
      }
      if ((size_t)buf->numel() < need) return PyLong_FromLongLong(-(long long)need);
      if (a[12] == Py_None) Py_RETURN_NONE;
    }
    wk = buf->data_ptr();
    wk_bytes = (size_t)buf->numel();
  }
  at::Tensor y;
  const w4a8_status s = without_gil([&] {
    y = out ? *out : at::empty({T, H, 128}, q->options());
    at::Tensor tmp;  // released to the allocator on this stream, which orders its next use
    if (temporary) {
      tmp = at::empty({(int64_t)need}, q->options().dtype(at::kByte));
      wk = tmp.data_ptr();
      wk_bytes = need;
    }
    return w4a8_cache_attention(&c, &b, ptr<uint16_t>(q), stride_of(q, 0), stride_of(q, 1), H, scale, max_len, ptr<uint16_t>(&y),
                                stride_of(&y, 0), stride_of(&y, 1), wk, wk_bytes, stream);
  });
  if (s != W4A8_OK) return PyLong_FromLong(s);
  if (out) return Py_NewRef(a[10]);
  return THPVariable_Wrap(std::move(y));
  END_HANDLE_TH_ERRORS
}

// The 4-bit cache's: (k_codes, v_codes, k_params, v_params), and a batch's
// (starts, lengths, table).
bool cache4_view(PyObject* o, c10::DeviceIndex device, w4a8_cache4& c) {
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) return false;
  auto item = [&](int i) { return PyTuple_GET_ITEM(o, i); };
  const at::Tensor *k = whole(item(0), at::kInt, 5, device), *v = whole(item(1), at::kInt, 6, device),
                   *kp = whole(item(2), at::kHalf, 5, device), *vp = whole(item(3), at::kHalf, 5, device);
  if (!k || !v || !kp || !vp) return false;
  const int64_t pages = k->size(0), Hkv = k->size(1);
  auto is = [&](const at::Tensor* t, std::initializer_list<int64_t> shape) {
    int64_t i = 2;
    for (int64_t n : shape)
      if (t->size(i++) != n) return false;
    return t->size(0) == pages && t->size(1) == Hkv;
  };
  if (!is(k, {4, 16, 16}) || !is(v, {8, 2, 16, 4}) || !is(kp, {2, W4A8_CACHE_BLOCK, 2}) || !is(vp, {2, 2, W4A8_CACHE_BLOCK}))
    return false;
  c = {ptr<uint32_t>(k), ptr<uint32_t>(v), ptr<uint16_t>(kp), ptr<uint16_t>(vp), pages, Hkv};
  return true;
}
bool batch4_view(PyObject* const* b, int64_t T, c10::DeviceIndex device, w4a8_batch& out) {
  const at::Tensor *starts = whole(b[0], at::kInt, 1, device), *lengths = whole(b[1], at::kInt, 1, device),
                   *table = whole(b[2], at::kInt, 2, device);
  if (!starts || !lengths || !table) return false;
  const int64_t B = lengths->size(0);
  if (starts->size(0) != B + 1 || table->size(0) != B) return false;
  out = {ptr<int32_t>(starts), ptr<int32_t>(lengths), ptr<int32_t>(table), table->size(1), B, T, nullptr, nullptr, nullptr, 0};
  return true;
}
const at::Tensor* token_rows(PyObject* o, c10::DeviceIndex device) {
  const at::Tensor* t = rows_of(o, at::kBFloat16, 3, device);
  return t && t->size(2) == 128 ? t : nullptr;
}

// cache4_append(k, v, cache, starts, lengths, table) -> True
PyObject* cache4_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const c10::DeviceIndex device = n == 6 ? device_of(a[0]) : -1;
  if (device < 0) Py_RETURN_NONE;
  const at::Tensor *k = token_rows(a[0], device), *v = token_rows(a[1], device);
  w4a8_cache4 c;
  w4a8_batch b;
  if (!k || !v || k->sizes() != v->sizes() || !cache4_view(a[2], device, c) || k->size(1) != c.Hkv ||
      !batch4_view(a + 3, k->size(0), device, b))
    Py_RETURN_NONE;
  const hipStream_t stream = current_stream();
  const w4a8_status s = without_gil([&] {
    return w4a8_cache4_append(&c, &b, ptr<uint16_t>(k), stride_of(k, 0), stride_of(k, 1), ptr<uint16_t>(v), stride_of(v, 0),
                              stride_of(v, 1), stream);
  });
  if (s != W4A8_OK) return PyLong_FromLong(s);
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

// Two results: the caller's own tensors, or the call's.
PyObject* pair_of(PyObject* own0, const at::Tensor& t0, PyObject* own1, const at::Tensor& t1) {
  PyObject* r = PyTuple_New(2);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, own0 != Py_None || !t0.defined() ? Py_NewRef(own0) : THPVariable_Wrap(t0));
  PyTuple_SET_ITEM(r, 1, own1 != Py_None || !t1.defined() ? Py_NewRef(own1) : THPVariable_Wrap(t1));
  return r;
}

// cache4_read(cache, starts, lengths, table, rows, k_out, v_out) -> (k, v)
PyObject* cache4_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7 || !is_int(a[4]) || !PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != 4) Py_RETURN_NONE;
  const c10::DeviceIndex device = device_of(PyTuple_GET_ITEM(a[0], 0));
  const int64_t T = as_int(a[4]);
  if (PyErr_Occurred()) PyErr_Clear();
  if (device < 0 || T < 0) Py_RETURN_NONE;
  w4a8_cache4 c;
  w4a8_batch b;
  if (!cache4_view(a[0], device, c) || !batch4_view(a + 1, T, device, b)) Py_RETURN_NONE;
  const at::Tensor* own[2] = {nullptr, nullptr};
  for (int i = 0; i < 2; ++i)
    if (a[5 + i] != Py_None &&
        (!(own[i] = token_rows(a[5 + i], device)) || own[i]->size(0) != T || own[i]->size(1) != c.Hkv))
      Py_RETURN_NONE;
  const at::Tensor& codes = THPVariable_Unpack(PyTuple_GET_ITEM(a[0], 0));
  const hipStream_t stream = current_stream();
  at::Tensor k, v;
  const w4a8_status s = without_gil([&] {
    k = own[0] ? *own[0] : at::empty({T, c.Hkv, 128}, codes.options().dtype(at::kBFloat16));
    v = own[1] ? *own[1] : at::empty({T, c.Hkv, 128}, codes.options().dtype(at::kBFloat16));
    return w4a8_cache4_read(&c, &b, ptr<uint16_t>(&k), stride_of(&k, 0), stride_of(&k, 1), ptr<uint16_t>(&v), stride_of(&v, 0),
                            stride_of(&v, 1), stream);
  });
  if (s != W4A8_OK) return PyLong_FromLong(s);
  return pair_of(a[5], k, a[6], v);
  END_HANDLE_TH_ERRORS
}

// qk_norm_rope(q, k, gamma_q, gamma_k, eps, pos, rope_cos, rope_sin, axes, q_out, k_out) -> (q, k)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 11 || !PyFloat_CheckExact(a[4])) Py_RETURN_NONE;
  const c10::DeviceIndex device = device_of(a[0] != Py_None ? a[0] : a[1]);
  if (device < 0) Py_RETURN_NONE;
  w4a8_heads heads[2] = {};
  const at::Tensor *x[2] = {nullptr, nullptr}, *own[2] = {nullptr, nullptr};
  int64_t T = -1;
  for (int i = 0; i < 2; ++i) {
    if (a[i] == Py_None) continue;
    if (!(x[i] = token_rows(a[i], device)) || (T >= 0 && x[i]->size(0) != T)) Py_RETURN_NONE;
    T = x[i]->size(0);
    heads[i] = {ptr<uint16_t>(x[i]), stride_of(x[i], 0), stride_of(x[i], 1), x[i]->size(1), nullptr, nullptr, 0, 0};
    if (a[2 + i] != Py_None) {
      const at::Tensor* gamma = whole(a[2 + i], at::kBFloat16, 1, device);
      if (!gamma || gamma->size(0) != 128) Py_RETURN_NONE;
      heads[i].gamma = ptr<uint16_t>(gamma);
    }
    if (a[9 + i] != Py_None && (!(own[i] = token_rows(a[9 + i], device)) || own[i]->sizes() != x[i]->sizes())) Py_RETURN_NONE;
  }
  w4a8_rope rope = {};
  if (a[5] != Py_None) {
    const at::Tensor* pos = whole(a[5], at::kInt, 2, device);
    if (!pos) pos = whole(a[5], at::kInt, 1, device);
    const at::Tensor *cs = whole(a[6], at::kFloat, 2, device), *sn = whole(a[7], at::kFloat, 2, device);
    if (!pos || !cs || !sn || pos->size(pos->dim() - 1) != T || cs->sizes() != sn->sizes() || cs->size(1) != 64) Py_RETURN_NONE;
    if (a[8] != Py_None && (!PyBytes_CheckExact(a[8]) || PyBytes_GET_SIZE(a[8]) != 64)) Py_RETURN_NONE;
    rope = {ptr<int32_t>(pos), pos->dim() == 2 ? pos->size(0) : 1,
            a[8] == Py_None ? nullptr : reinterpret_cast<const uint8_t*>(PyBytes_AS_STRING(a[8])), ptr<float>(cs), ptr<float>(sn),
            cs->size(0)};
  }
  const float eps = (float)PyFloat_AS_DOUBLE(a[4]);
  const hipStream_t stream = current_stream();
  at::Tensor y[2];
  const w4a8_status s = without_gil([&] {
    for (int i = 0; i < 2; ++i)
      if (x[i]) {
        y[i] = own[i] ? *own[i] : at::empty(x[i]->sizes(), x[i]->options());
        heads[i].out = ptr<uint16_t>(&y[i]);
        heads[i].out_row = stride_of(&y[i], 0);
        heads[i].out_head = stride_of(&y[i], 1);
      }
    return w4a8_qk_norm_rope(x[0] ? &heads[0] : nullptr, x[1] ? &heads[1] : nullptr, T, eps, a[5] == Py_None ? nullptr : &rope, stream);
  });
  if (s != W4A8_OK) return PyLong_FromLong(s);
  return pair_of(x[0] ? a[9] : Py_None, y[0], x[1] ? a[10] : Py_None, y[1]);
  END_HANDLE_TH_ERRORS
}

// cache4_attention(q, cache, starts, lengths, table, scale, max_len, out,
//                  workspace, workspace_stream, is_workspace)
// The last three and a negative answer are as for linear.
PyObject* cache4_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const c10::DeviceIndex device = n == 11 ? device_of(a[0]) : -1;
  if (device < 0) Py_RETURN_NONE;
  const at::Tensor *q = token_rows(a[0], device), *out = nullptr;
  w4a8_cache4 c;
  w4a8_batch b;
  if (!q || !cache4_view(a[1], device, c) || !batch4_view(a + 2, q->size(0), device, b) || !PyFloat_CheckExact(a[5])) Py_RETURN_NONE;
  const int64_t T = b.T, H = q->size(1);
  int64_t max_len = b.max_blocks * W4A8_CACHE_BLOCK;
  if (a[6] != Py_None) {
    if (!is_int(a[6])) Py_RETURN_NONE;
    max_len = as_int(a[6]);
    if (PyErr_Occurred()) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
  }
  if (a[7] != Py_None && (!(out = token_rows(a[7], device)) || out->sizes() != q->sizes())) Py_RETURN_NONE;
  const float scale = (float)PyFloat_AS_DOUBLE(a[5]);
  const hipStream_t stream = current_stream();
  const size_t need = w4a8_cache4_attention_workspace_bytes(b.B, T, H, c.Hkv, max_len);
  void* wk = nullptr;
  size_t wk_bytes = 0;
  const bool temporary = need && a[8] == Py_None && a[10] != Py_True;
  if (need && !temporary) {
    const at::Tensor* buf = plain(a[8], at::kByte);
    if (!buf || buf->get_device() != device) Py_RETURN_NONE;
    if (a[10] == Py_True) {
      if (a[9] != Py_None && (!is_int(a[9]) || PyLong_AsVoidPtr(a[9]) != (void*)stream)) {
        PyErr_Clear();
        Py_RETURN_NONE;
      }
      if ((size_t)buf->numel() < need) return PyLong_FromLongLong(-(long long)need);
      if (a[9] == Py_None) Py_RETURN_NONE;
    }
    wk = buf->data_ptr();
    wk_bytes = (size_t)buf->numel();
  }
  at::Tensor y;
  const w4a8_status s = without_gil([&] {
    y = out ? *out : at::empty({T, H, 128}, q->options());
    at::Tensor tmp;  // released to the allocator on this stream, which orders its next use
    if (temporary) {
      tmp = at::empty({(int64_t)need}, q->options().dtype(at::kByte));
      wk = tmp.data_ptr();
      wk_bytes = need;
    }
    return w4a8_cache4_attention(&c, &b, ptr<uint16_t>(q), stride_of(q, 0), stride_of(q, 1), H, scale, max_len, ptr<uint16_t>(&y),
                                 stride_of(&y, 0), stride_of(&y, 1), wk, wk_bytes, stream);
  });
  if (s != W4A8_OK) return PyLong_FromLong(s);
  if (out) return Py_NewRef(a[7]);
  return THPVariable_Wrap(std::move(y));
  END_HANDLE_TH_ERRORS
}

PyObject* pair(at::Tensor q, at::Tensor s) {
  PyObject* t = PyTuple_New(2);
  if (!t) return nullptr;
  PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(std::move(q)));
  PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(std::move(s)));
  return t;
}

// quantize(x) / rmsnorm_quantize(x, gamma, eps)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor* x = n == 1 || n == 3 ? plain(a[0], at::kBFloat16) : nullptr;
  if (!x || x->dim() != 2) Py_RETURN_NONE;
  const int64_t M = x->size(0), K = x->size(1);
  const at::Tensor* g = nullptr;
  float eps = 0.0f;
  if (n == 3) {
    g = plain(a[1], at::kBFloat16);
    if (!g || g->dim() != 1 || g->size(0) != K || !PyFloat_CheckExact(a[2])) Py_RETURN_NONE;
    eps = (float)PyFloat_AS_DOUBLE(a[2]);
  }
  at::Tensor q, s;
  const uint16_t *xp = static_cast<const uint16_t*>(x->data_ptr()), *gp = g ? static_cast<const uint16_t*>(g->data_ptr()) : nullptr;
  const hipStream_t stream = current_stream();
  const w4a8_status st = without_gil([&] {
    q = at::empty({M, K}, x->options().dtype(at::kChar));
    s = at::empty({M}, x->options().dtype(at::kFloat));
    int8_t* qp = static_cast<int8_t*>(q.data_ptr());
    float* sp = static_cast<float*>(s.data_ptr());
    return g ? w4a8_rmsnorm_quantize_act(xp, gp, eps, M, K, qp, sp, stream) : w4a8_quantize_act(xp, M, K, qp, sp, stream);
  });
  if (st != W4A8_OK) return PyLong_FromLong(st);
  return pair(std::move(q), std::move(s));
  END_HANDLE_TH_ERRORS
}

// flow_step(x, v_new, v_cache, dt, stats, repeat) -> the stats tensor, True
// without stats
PyObject* flow_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 6 || !PyFloat_CheckExact(a[3]) || !PyBool_Check(a[4]) || !is_int(a[5])) Py_RETURN_NONE;
  const at::Tensor *x = plain(a[0], at::kFloat), *c = plain(a[2], at::kBFloat16), *v = nullptr;
  if (!x || !c || x->dim() != 2) Py_RETURN_NONE;
  const int64_t B = x->size(0), len = x->size(1), repeat = as_int(a[5]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  auto fits = [&](const at::Tensor& t) { return t.dim() == 2 && t.size(0) == B && t.size(1) == len; };
  if (!fits(*c)) Py_RETURN_NONE;
  if (a[1] != Py_None) {
    v = plain(a[1], at::kBFloat16);
    if (!v || !fits(*v)) Py_RETURN_NONE;
  }
  const bool stats = a[4] == Py_True;
  at::Tensor st;
  float* xp = static_cast<float*>(x->data_ptr());
  const uint16_t* vp = v ? static_cast<const uint16_t*>(v->data_ptr()) : nullptr;
  uint16_t* cp = static_cast<uint16_t*>(c->data_ptr());
  const float dt = (float)PyFloat_AS_DOUBLE(a[3]);
  const hipStream_t stream = current_stream();
  const w4a8_status s = without_gil([&] {
    if (stats) st = at::empty({B, 4}, x->options().dtype(at::kDouble));
    double* stp = stats ? static_cast<double*>(st.data_ptr()) : nullptr;
    return w4a8_flow_step(xp, vp, cp, B, len, dt, repeat, stp, stream);
  });
  if (s != W4A8_OK) return PyLong_FromLong(s);
  if (!stats) Py_RETURN_TRUE;
  return THPVariable_Wrap(std::move(st));
  END_HANDLE_TH_ERRORS
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL
PyMethodDef methods[] = {{"linear", FAST(linear), nullptr},
                         {"quantize", FAST(quantize), nullptr},
                         {"flow_step", FAST(flow_step), nullptr},
                         {"add_norm", FAST(add_norm), nullptr},
                         {"cache_append", FAST(cache_append), nullptr},
                         {"cache_attention", FAST(cache_attention), nullptr},
                         {"qk_norm_rope", FAST(qk_norm_rope), nullptr},
                         {"cache4_append", FAST(cache4_append), nullptr},
                         {"cache4_read", FAST(cache4_read), nullptr},
                         {"cache4_attention", FAST(cache4_attention), nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
