// Argument marshalling of the binding's tensor calls in native code: the ordinary call (plain contiguous CUDA tensors, torch's
// current stream, the binding's own scratch) without the Python statements and the ctypes conversion around the C entry point.
// It does what binding.py does for the same call, in the same order, and returns NotImplemented, with nothing done, for every
// call that it does not know in full: binding.py then takes it, with its checks and errors.
//
// Why: a decode step of one sequence is 10 us on the GPU and was 12.3 us on the host, 5 of them the two launches (a small fp32
// call 8.9 and 10.0).  The tensors' attributes alone are some twenty Python calls.
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <cuda_runtime_api.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

#include "../../include/kata.h"

namespace {

PyObject* not_implemented() { Py_RETURN_NOTIMPLEMENTED; }

struct Held {                    // a reference until the end of the call (or null)
  PyObject* o;
  ~Held() { Py_XDECREF(o); }
};

// A tensor whose attributes are what they seem: no subclass, in memory of its own, on a CUDA device.
const at::Tensor* plain(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.has_storage() ? &t : nullptr;
}
const at::Tensor* plain_contiguous(PyObject* o) {
  const at::Tensor* t = plain(o);
  return t != nullptr && t->is_contiguous() ? t : nullptr;
}

bool dtype_code(const at::Tensor& t, int32_t& code) {
  if (t.scalar_type() == at::kFloat) code = KATA_F32;
  else if (t.scalar_type() == at::kBFloat16) code = KATA_BF16;
  else return false;
  return true;
}

// The keyword options of a call; false: one that is not an int of 32 bits, or not known here.
bool read_options(PyObject* kw, kata_opts& o) {
  o = kata_opts{};
  o.struct_size = sizeof(kata_opts);
  o.feature_order = 2;
  if (!PyDict_CheckExact(kw)) return false;
  PyObject *key, *value;
  Py_ssize_t pos = 0;
  while (PyDict_Next(kw, &pos, &key, &value)) {
    static const struct { const char* name; int32_t kata_opts::* field; } kFields[] = {
        {"feature_groups", &kata_opts::feature_groups}, {"state_layout", &kata_opts::state_layout},
        {"inter_chunk", &kata_opts::inter_chunk},       {"feature_order", &kata_opts::feature_order},
        {"impl", &kata_opts::impl},                     {"scan_group", &kata_opts::scan_group}};
    if (!PyUnicode_Check(key) || !PyLong_CheckExact(value)) return false;
    int overflow = 0;
    const long long x = PyLong_AsLongLongAndOverflow(value, &overflow);
    if (overflow != 0 || x < INT_MIN || x > INT_MAX) return false;
    bool known = false;
    for (const auto& f : kFields)
      if (PyUnicode_CompareWithASCIIString(key, f.name) == 0) {
        o.*(f.field) = (int32_t)x;
        known = true;
        break;
      }
    if (!known) return false;
  }
  return true;
}

bool int_size(int64_t x, int& out) {
  out = (int)x;
  return x >= 0 && x <= INT_MAX;
}

// The stream of the call and, where it needs scratch, the buffer that binding.py keeps for this thread, device and stream.
// `held` is a new reference to hold until the call is made (or null).  false: binding.py has to make a buffer first.
bool stream_and_scratch(PyObject* owner, const at::Tensor& q, int fn, int B, int H, int T, int d_k, int d_v, int C, kata_opts& o,
                        PyObject*& held) {
  held = nullptr;
  const c10::DeviceIndex dev = q.device().index();
  cudaStream_t stream = c10::cuda::getCurrentCUDAStream(dev).stream();
  o.stream = stream;
  const size_t need = kata_workspace_bytes(fn, B, H, T, d_k, d_v, C, &o);
  if (need == 0) return true;
  if (stream != nullptr) {
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(stream, &status) != cudaSuccess) {
      cudaGetLastError();
      return false;
    }
    if (status != cudaStreamCaptureStatusNone) return false;
  }
  static PyObject* const name = PyUnicode_InternFromString("bufs");
  PyObject* bufs = PyObject_GetAttr(owner, name);
  PyObject* key = stream != nullptr ? Py_BuildValue("(iN)", (int)dev, PyLong_FromVoidPtr(stream)) : Py_BuildValue("(iO)", (int)dev, Py_None);
  PyObject* entry = bufs != nullptr && key != nullptr && PyDict_Check(bufs) ? PyDict_GetItemWithError(bufs, key) : nullptr;
  Py_XINCREF(entry);
  Py_XDECREF(key);
  Py_XDECREF(bufs);
  if (entry != nullptr && PyTuple_CheckExact(entry) && PyTuple_GET_SIZE(entry) == 3) {
    const size_t size = PyLong_AsSize_t(PyTuple_GET_ITEM(entry, 2));
    void* ptr = PyLong_AsVoidPtr(PyTuple_GET_ITEM(entry, 1));
    if (!PyErr_Occurred() && size >= need) {
      o.workspace = ptr;
      o.workspace_bytes = size;
      held = entry;
      return true;
    }
  }
  Py_XDECREF(entry);
  PyErr_Clear();
  return false;
}

// Room for what the kernels read or write behind a pointer, which take sizes, type and device from q (binding.py _check_room).
bool has_room(const at::Tensor& t, const at::Tensor& q, at::ScalarType type, int64_t n) {
  return t.numel() >= n && t.scalar_type() == type && t.device() == q.device() && t.is_contiguous();
}
bool input_fits(const at::Tensor& t, const at::Tensor& q, int64_t heads, int64_t n) {
  return has_room(t, q, q.scalar_type(), n) && (t.numel() == n || heads == 1);
}

// The result of a call: the tensors, or the status as an int.
PyObject* result(int status, std::initializer_list<const at::Tensor*> out) {
  if (status != KATA_OK) return PyLong_FromLong(status);
  if (out.size() == 1) return THPVariable_Wrap(**out.begin());
  PyObject* tuple = PyTuple_New((Py_ssize_t)out.size());
  Py_ssize_t i = 0;
  for (const at::Tensor* t : out) {
    PyObject* x = tuple != nullptr ? THPVariable_Wrap(*t) : nullptr;
    if (x == nullptr) {
      Py_XDECREF(tuple);
      return nullptr;
    }
    PyTuple_SET_ITEM(tuple, i++, x);
  }
  return tuple;
}

// The tensor that was passed for an output of n elements, or a new one like `like`; false: one that is not plain, or too small.
bool output_ok(PyObject* o, const at::Tensor& q, int64_t n) {
  if (o == Py_None) return true;
  const at::Tensor* p = plain(o);
  return p != nullptr && has_room(*p, q, q.scalar_type(), n);
}
at::Tensor output(PyObject* o, const at::Tensor& like) { return o == Py_None ? at::empty_like(like) : THPVariable_Unpack(o); }

bool pointer(PyObject* o, const at::Tensor& q, at::ScalarType type, int64_t n, void*& p) {
  p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = plain(o);
  if (t == nullptr || !has_room(*t, q, type, n)) return false;
  p = t->data_ptr();
  return true;
}

// Feature rows of a state (binding.py decode_n_psi).
int64_t state_rows(const kata_opts& o, int d_k) {
  const int g = o.feature_groups > 1 ? o.feature_groups : 1, m = d_k / g;
  return o.feature_order == 1 ? d_k : (int64_t)g * (o.state_layout == KATA_LAYOUT_PACKED ? (int64_t)m * (m + 1) / 2 : (int64_t)m * m);
}

// The three calls.  With None for the scratch owner they only look the tensors over: True, they are plain and have room.

// forward(fn, scratch owner, q, k, v, out, C, s_pre, z_pre, s_init, z_init, device_status, options)
PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 13 || !PyLong_CheckExact(a[0]) || !PyLong_CheckExact(a[6]) || at::impl::torch_function_mode_enabled()) return not_implemented();
  const int fn = (int)PyLong_AsLong(a[0]);
  int overflow = 0;
  const long c_arg = PyLong_AsLongAndOverflow(a[6], &overflow);
  kata_opts o;
  if (overflow != 0 || c_arg < INT_MIN || c_arg > INT_MAX || !read_options(a[12], o)) return not_implemented();
  const at::Tensor *q = plain_contiguous(a[2]), *k = plain_contiguous(a[3]), *v = plain_contiguous(a[4]);
  if (q == nullptr || k == nullptr || v == nullptr || q->dim() != 4 || v->dim() < 1 || !dtype_code(*q, o.dtype)) return not_implemented();
  int B, H, T, d_k, d_v;
  if (!int_size(q->size(0), B) || !int_size(q->size(1), H) || !int_size(q->size(2), T) || !int_size(q->size(3), d_k) ||
      !int_size(v->size(-1), d_v))
    return not_implemented();
  const int64_t heads = (int64_t)B * H, nv = heads * T * d_v;
  if (!input_fits(*k, *q, heads, q->numel()) || !input_fits(*v, *q, heads, nv) || !output_ok(a[5], *q, nv)) return not_implemented();
  void *s_pre, *z_pre, *s_init, *z_init, *device_status;
  const int64_t rows = heads * state_rows(o, d_k);
  const int64_t rows_pre = fn == KATA_FN_CHUNK_STATE_SCAN && c_arg > 0 ? rows * ((T + c_arg - 1) / c_arg) : rows;
  if (!pointer(a[7], *q, at::kFloat, rows_pre * d_v, s_pre) || !pointer(a[8], *q, at::kFloat, rows_pre, z_pre) ||
      !pointer(a[9], *q, at::kFloat, rows * d_v, s_init) || !pointer(a[10], *q, at::kFloat, rows, z_init) ||
      !pointer(a[11], *q, at::kInt, 1, device_status))
    return not_implemented();
  o.s_pre = static_cast<float*>(s_pre);
  o.z_pre = static_cast<float*>(z_pre);
  o.s_init = static_cast<const float*>(s_init);
  o.z_init = static_cast<const float*>(z_init);
  o.device_status = static_cast<int*>(device_status);
  if (a[1] == Py_None) Py_RETURN_TRUE;
  PyObject* held;
  if (!stream_and_scratch(a[1], *q, fn, B, H, T, d_k, d_v, (int)c_arg, o, held)) return not_implemented();
  const Held hold{held};
  const at::Tensor out = output(a[5], *v);
  const auto call = fn == KATA_FN_QUADRATIC ? kata_fwd_quadratic : fn == KATA_FN_CHUNKED ? kata_fwd_chunked : kata_chunk_state_scan;
  const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr();
  void* op = out.data_ptr();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = call(qp, kp, vp, op, B, H, T, d_k, d_v, (int)c_arg, &o);
  Py_END_ALLOW_THREADS
  return result(st, {&out});
  END_HANDLE_TH_ERRORS
}

// decode(scratch owner, q, k, v, S, Z, out, options)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  kata_opts o;
  if (n != 8 || !read_options(a[7], o) || at::impl::torch_function_mode_enabled()) return not_implemented();
  const at::Tensor *q = plain_contiguous(a[1]), *k = plain_contiguous(a[2]), *v = plain_contiguous(a[3]), *S = plain_contiguous(a[4]),
                   *Z = plain_contiguous(a[5]);
  if (q == nullptr || k == nullptr || v == nullptr || S == nullptr || Z == nullptr || q->dim() != 3 || v->dim() < 1 ||
      !dtype_code(*q, o.dtype) || S->scalar_type() != at::kFloat || Z->scalar_type() != at::kFloat || S->dim() != 4 || Z->dim() != 3)
    return not_implemented();
  int B, H, d_k, d_v;
  if (!int_size(q->size(0), B) || !int_size(q->size(1), H) || !int_size(q->size(2), d_k) || !int_size(v->size(-1), d_v)) return not_implemented();
  const int64_t heads = (int64_t)B * H, rows = state_rows(o, d_k);
  if (!input_fits(*k, *q, heads, q->numel()) || !input_fits(*v, *q, heads, heads * d_v) || !output_ok(a[6], *q, heads * d_v) ||
      S->device() != q->device() || Z->device() != q->device())
    return not_implemented();
  if (S->size(0) != B || S->size(1) != H || S->size(2) != rows || S->size(3) != d_v || Z->size(0) != B || Z->size(1) != H || Z->size(2) != rows)
    return not_implemented();
  if (a[0] == Py_None) Py_RETURN_TRUE;
  PyObject* held;
  if (!stream_and_scratch(a[0], *q, KATA_FN_DECODE_STEP, B, H, 1, d_k, d_v, 0, o, held)) return not_implemented();
  const Held hold{held};
  const at::Tensor out = output(a[6], *v);
  const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr();
  void *op = out.data_ptr(), *sp = S->data_ptr(), *zp = Z->data_ptr();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = kata_decode_step(qp, kp, vp, op, static_cast<float*>(sp), static_cast<float*>(zp), B, H, d_k, d_v, &o);
  Py_END_ALLOW_THREADS
  return result(st, {&out});
  END_HANDLE_TH_ERRORS
}

// backward(fn, scratch owner, q, k, v, dout, dq, dk, dv, C, options)
PyObject* backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  kata_opts o;
  if (n != 11 || !PyLong_CheckExact(a[0]) || !PyLong_CheckExact(a[9]) || !read_options(a[10], o) || at::impl::torch_function_mode_enabled())
    return not_implemented();
  const int fn = (int)PyLong_AsLong(a[0]);
  int overflow = 0;
  const long c_arg = PyLong_AsLongAndOverflow(a[9], &overflow);
  if (overflow != 0 || c_arg < INT_MIN || c_arg > INT_MAX) return not_implemented();
  const at::Tensor *q = plain_contiguous(a[2]), *k = plain_contiguous(a[3]), *v = plain_contiguous(a[4]), *dout = plain_contiguous(a[5]);
  if (q == nullptr || k == nullptr || v == nullptr || dout == nullptr || q->dim() != 4 || v->dim() < 1 || !dtype_code(*q, o.dtype))
    return not_implemented();
  int B, H, T, d_k, d_v;
  if (!int_size(q->size(0), B) || !int_size(q->size(1), H) || !int_size(q->size(2), T) || !int_size(q->size(3), d_k) ||
      !int_size(v->size(-1), d_v))
    return not_implemented();
  const int64_t heads = (int64_t)B * H, nk = q->numel(), nv = heads * T * d_v;
  if (!input_fits(*k, *q, heads, nk) || !input_fits(*v, *q, heads, nv) || !input_fits(*dout, *q, heads, nv) || !output_ok(a[6], *q, nk) ||
      !output_ok(a[7], *q, nk) || !output_ok(a[8], *q, nv))
    return not_implemented();
  if (a[1] == Py_None) Py_RETURN_TRUE;
  PyObject* held;
  if (!stream_and_scratch(a[1], *q, fn, B, H, T, d_k, d_v, (int)c_arg, o, held)) return not_implemented();
  const Held hold{held};
  const at::Tensor dq = output(a[6], *q), dk = output(a[7], *k), dv = output(a[8], *v);
  const void *qp = q->data_ptr(), *kp = k->data_ptr(), *vp = v->data_ptr(), *gp = dout->data_ptr();
  void *dqp = dq.data_ptr(), *dkp = dk.data_ptr(), *dvp = dv.data_ptr();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = fn == KATA_FN_BWD_QUADRATIC ? kata_bwd_quadratic(qp, kp, vp, gp, dqp, dkp, dvp, B, H, T, d_k, d_v, &o)
                                   : kata_bwd_chunked(qp, kp, vp, gp, dqp, dkp, dvp, B, H, T, d_k, d_v, (int)c_arg, &o);
  Py_END_ALLOW_THREADS
  return result(st, {&dq, &dk, &dv});
  END_HANDLE_TH_ERRORS
}

// ---- rows around the attention and the decayed recurrence (binding.py: the functions of the same names) ----
// Strided views whose rows lie side by side, on the current device; everything else is left to binding.py.

// The truth of an option; false: it has none (binding.py raises what asking for it raises).
bool truth(PyObject* o, int32_t& to) {
  const int x = PyObject_IsTrue(o);
  if (x < 0) PyErr_Clear();
  to = x == 1;
  return x >= 0;
}
// The tensor if it is plain, has these sizes and this type, and lies on main's device (main: itself).
const at::Tensor* view(PyObject* o, const at::Tensor* main, std::initializer_list<int64_t> sizes, at::ScalarType type, bool contiguous = false) {
  const at::Tensor* t = plain(o);
  if (t == nullptr || t->scalar_type() != type || t->dim() != (int64_t)sizes.size() || (main != nullptr && t->device() != main->device())) return nullptr;
  int64_t i = 0;
  for (int64_t n : sizes)
    if (t->size(i++) != n) return nullptr;
  if (contiguous) return t->is_contiguous() ? t : nullptr;
  return t->size(-1) == 1 || t->stride(-1) == 1 ? t : nullptr;
}
bool main_tensor(PyObject* o, int64_t dim, const at::Tensor*& t, kata_opts& opts) {
  t = plain(o);
  opts = kata_opts{};
  opts.struct_size = sizeof(kata_opts);
  if (t == nullptr || t->dim() != dim || !dtype_code(*t, opts.dtype) || t->numel() == 0 || t->device().index() != c10::cuda::current_device()) return false;
  for (int64_t i = 0; i < dim; ++i)
    if (t->size(i) > INT_MAX) return false;
  return t->size(-1) == 1 || t->stride(-1) == 1;
}
// An optional contiguous tensor's pointer; false: one that is left to binding.py.
template <typename T> bool optional(PyObject* o, const at::Tensor& main, std::initializer_list<int64_t> sizes, at::ScalarType type, T*& p) {
  p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = view(o, &main, sizes, type, true);
  if (t == nullptr) return false;
  p = static_cast<T*>(const_cast<void*>(static_cast<const void*>(t->data_ptr())));
  return true;
}
void strides(const at::Tensor& t, int64_t* to, int n) {
  for (int i = 0; i < n; ++i) to[i] = t.stride(i);
}
at::Tensor make_output(PyObject* o, const at::Tensor& like, bool same_layout) {
  return o != Py_None ? THPVariable_Unpack(o) : same_layout ? at::empty_like(like) : at::empty(like.sizes(), like.options());
}
bool given_fits(PyObject* o, const at::Tensor& like) {
  if (o == Py_None) return true;
  const at::Tensor* t = plain(o);
  return t != nullptr && t->sizes() == like.sizes() && t->scalar_type() == like.scalar_type() && t->device() == like.device() &&
         (t->size(-1) == 1 || t->stride(-1) == 1);
}
PyObject* tuple_of(int status, std::initializer_list<const at::Tensor*> out) {
  if (status != KATA_OK) return PyLong_FromLong(status);
  PyObject* tuple = PyTuple_New((Py_ssize_t)out.size());
  Py_ssize_t i = 0;
  for (const at::Tensor* t : out) {
    PyObject* x = tuple == nullptr ? nullptr : t->defined() ? THPVariable_Wrap(*t) : (Py_INCREF(Py_None), Py_None);
    if (x == nullptr) {
      Py_XDECREF(tuple);
      return nullptr;
    }
    PyTuple_SET_ITEM(tuple, i++, x);
  }
  return tuple;
}

// q, k, q_weight, k_weight, positions, offset, frequencies (tuple or list of floats), interleaved, eps: the arguments of both calls
bool rope_args(PyObject* const* a, kata_norm_rope_args& r, double (&freq)[64], kata_opts& o, const at::Tensor*& q, const at::Tensor*& k) {
  if (at::impl::torch_function_mode_enabled() || !main_tensor(a[0], 4, q, o)) return false;
  r = kata_norm_rope_args{};
  r.struct_size = sizeof r;
  r.B = (int)q->size(0); r.H_q = (int)q->size(1); r.T = (int)q->size(2); r.d = (int)q->size(3);
  k = nullptr;
  if (a[1] != Py_None) {
    const at::Tensor* t = plain(a[1]);
    if (t == nullptr || t->dim() != 4 || t->size(1) > INT_MAX) return false;
    k = view(a[1], q, {r.B, t->size(1), r.T, r.d}, q->scalar_type());
    if (k == nullptr) return false;
    r.H_k = (int)k->size(1);
  } else if (a[3] != Py_None) {
    return false;
  }
  if (!optional(a[2], *q, {r.d}, q->scalar_type(), r.q_weight) || !optional(a[3], *q, {r.d}, q->scalar_type(), r.k_weight)) return false;
  if (a[4] != Py_None) {
    const at::Tensor* p = plain(a[4]);
    if (p == nullptr || p->scalar_type() != at::kLong || p->device() != q->device() || p->dim() < 1 || p->dim() > 2 || p->size(-1) != r.T ||
        (p->dim() == 2 && p->size(0) != r.B))
      return false;
    r.positions = p->data_ptr<int64_t>();
    r.pos_stride[0] = p->dim() == 2 ? p->stride(0) : 0;
    r.pos_stride[1] = p->stride(-1);
  }
  int overflow = 0;
  if (!PyLong_CheckExact(a[5])) return false;
  r.pos_offset = PyLong_AsLongLongAndOverflow(a[5], &overflow);
  if (overflow != 0 || !(PyTuple_CheckExact(a[6]) || PyList_CheckExact(a[6])) || !PyFloat_CheckExact(a[8])) return false;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[6]);
  if (n > 64) return false;
  PyObject** items = PySequence_Fast_ITEMS(a[6]);
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (!PyFloat_CheckExact(items[i])) return false;
    freq[i] = PyFloat_AS_DOUBLE(items[i]);
  }
  r.inv_freq = freq;
  r.rotary_dim = (int)(2 * n);
  if (!truth(a[7], r.interleaved)) return false;
  r.eps = PyFloat_AS_DOUBLE(a[8]);
  r.q = q->data_ptr();
  strides(*q, r.q_stride, 3);
  if (k != nullptr) {
    r.k = k->data_ptr();
    strides(*k, r.k_stride, 3);
  }
  return true;
}

// norm_rope(q, k, q_weight, k_weight, positions, offset, frequencies, interleaved, eps, q_out, k_out)
PyObject* norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  kata_norm_rope_args r;
  kata_opts o;
  double freq[64];
  const at::Tensor *q, *k;
  if (n != 11 || !rope_args(a, r, freq, o, q, k) || !given_fits(a[9], *q) || (k == nullptr ? a[10] != Py_None : !given_fits(a[10], *k))) return not_implemented();
  const at::Tensor qo = make_output(a[9], *q, false), ko = k != nullptr ? make_output(a[10], *k, false) : at::Tensor();
  r.q_out = qo.data_ptr();
  strides(qo, r.q_out_stride, 3);
  if (k != nullptr) {
    r.k_out = ko.data_ptr();
    strides(ko, r.k_out_stride, 3);
  }
  o.stream = c10::cuda::getCurrentCUDAStream(q->device().index()).stream();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = kata_fwd_norm_rope(&r, &o);
  Py_END_ALLOW_THREADS
  return tuple_of(st, {&qo, &ko});
  END_HANDLE_TH_ERRORS
}

// norm_rope_bwd(q, k, q_weight, k_weight, positions, offset, frequencies, interleaved, eps, scratch owner, dq_out, dk_out, dq, dk)
PyObject* norm_rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  kata_norm_rope_args r;
  kata_opts o;
  double freq[64];
  const at::Tensor *q, *k;
  if (n != 14 || !rope_args(a, r, freq, o, q, k) || a[10] == Py_None || !given_fits(a[10], *q) || !given_fits(a[12], *q)) return not_implemented();
  if (k == nullptr ? a[11] != Py_None || a[13] != Py_None : a[11] == Py_None || !given_fits(a[11], *k) || !given_fits(a[13], *k)) return not_implemented();
  PyObject* held;
  if (!stream_and_scratch(a[9], *q, KATA_FN_BWD_NORM_ROPE, r.B, r.H_q + r.H_k, r.T, r.d, 0, 0, o, held)) return not_implemented();
  const Held hold{held};
  const at::Tensor &go = THPVariable_Unpack(a[10]), dq = make_output(a[12], *q, true);
  at::Tensor dk, dqw, dkw;
  r.q_out = go.data_ptr();
  strides(go, r.q_out_stride, 3);
  r.dq = dq.data_ptr();
  strides(dq, r.dq_stride, 3);
  if (r.q_weight != nullptr) {
    dqw = at::empty({r.d}, q->options().dtype(at::kFloat));
    r.dq_weight = dqw.data_ptr<float>();
  }
  if (k != nullptr) {
    const at::Tensor& gk = THPVariable_Unpack(a[11]);
    dk = make_output(a[13], *k, true);
    r.k_out = gk.data_ptr();
    strides(gk, r.k_out_stride, 3);
    r.dk = dk.data_ptr();
    strides(dk, r.dk_stride, 3);
    if (r.k_weight != nullptr) {
      dkw = at::empty({r.d}, q->options().dtype(at::kFloat));
      r.dk_weight = dkw.data_ptr<float>();
    }
  }
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = kata_bwd_norm_rope(&r, &o);
  Py_END_ALLOW_THREADS
  return tuple_of(st, {&dq, &dk, &dqw, &dkw});
  END_HANDLE_TH_ERRORS
}

// x, weight, bias, silu, lengths: the arguments of the three calls; `dim`: axes of x (2: one token)
bool conv_args(PyObject* const* a, int64_t dim, kata_short_conv_args& r, kata_opts& o, const at::Tensor*& x, const at::Tensor*& w) {
  if (at::impl::torch_function_mode_enabled() || !main_tensor(a[0], dim, x, o)) return false;
  r = kata_short_conv_args{};
  r.struct_size = sizeof r;
  r.B = (int)x->size(0); r.T = dim == 3 ? (int)x->size(1) : 1; r.D = (int)x->size(-1);
  const at::Tensor* t = plain(a[1]);
  if (t == nullptr || t->dim() != 2 || t->size(1) > INT_MAX) return false;
  w = view(a[1], x, {r.D, t->size(1)}, x->scalar_type(), true);
  if (w == nullptr) return false;
  r.width = (int)w->size(1);
  r.weight = w->data_ptr();
  if (!optional(a[2], *x, {r.D}, x->scalar_type(), r.bias) || !optional(a[4], *x, {r.B}, at::kInt, r.lengths)) return false;
  if (!truth(a[3], r.silu)) return false;
  r.x = x->data_ptr();
  strides(*x, r.x_stride, (int)dim - 1);
  return true;
}

// short_conv(x, weight, bias, silu, lengths, s_init, s_final, out); x of two axes: one token
PyObject* short_conv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  kata_short_conv_args r;
  kata_opts o;
  const at::Tensor *x, *w;
  if (n != 8 || !THPVariable_CheckExact(a[0])) return not_implemented();
  const int64_t dim = THPVariable_Unpack(a[0]).dim();
  if ((dim != 2 && dim != 3) || !conv_args(a, dim, r, o, x, w) || !given_fits(a[7], *x)) return not_implemented();
  if (!optional(a[5], *x, {r.B, r.D, r.width - 1}, x->scalar_type(), r.s_init) || !optional(a[6], *x, {r.B, r.D, r.width - 1}, x->scalar_type(), r.s_final))
    return not_implemented();
  const at::Tensor out = make_output(a[7], *x, false);
  r.out = out.data_ptr();
  strides(out, r.out_stride, (int)dim - 1);
  o.stream = c10::cuda::getCurrentCUDAStream(x->device().index()).stream();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = dim == 2 ? kata_decode_short_conv(&r, &o) : kata_fwd_short_conv(&r, &o);
  Py_END_ALLOW_THREADS
  return result(st, {&out});
  END_HANDLE_TH_ERRORS
}

// short_conv_bwd(x, weight, bias, silu, lengths, scratch owner, dout, dx)
PyObject* short_conv_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  kata_short_conv_args r;
  kata_opts o;
  const at::Tensor *x, *w;
  if (n != 8 || !conv_args(a, 3, r, o, x, w) || a[6] == Py_None || !given_fits(a[6], *x) || !given_fits(a[7], *x)) return not_implemented();
  PyObject* held;
  if (!stream_and_scratch(a[5], *x, KATA_FN_BWD_SHORT_CONV, r.B, r.D, r.T, r.width, 0, 0, o, held)) return not_implemented();
  const Held hold{held};
  const at::Tensor &g = THPVariable_Unpack(a[6]), dx = make_output(a[7], *x, false), dw = at::empty(w->sizes(), w->options().dtype(at::kFloat)),
                   db = r.bias != nullptr ? at::empty({r.D}, w->options().dtype(at::kFloat)) : at::Tensor();
  r.dout = g.data_ptr();
  strides(g, r.dout_stride, 2);
  r.dx = dx.data_ptr();
  strides(dx, r.dx_stride, 2);
  r.dweight = dw.data_ptr<float>();
  r.dbias = db.defined() ? db.data_ptr<float>() : nullptr;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = kata_bwd_short_conv(&r, &o);
  Py_END_ALLOW_THREADS
  return tuple_of(st, {&dx, &dw, &db});
  END_HANDLE_TH_ERRORS
}

// ssm(scratch owner, q, k, v, dt, A, D, dt_bias, dt_softplus, s_init, s_final, lengths, out, impl); v of three axes: one token
PyObject* ssm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  kata_opts o;
  const at::Tensor *v, *q, *k, *dt;
  if (n != 14 || !THPVariable_CheckExact(a[3]) || !PyLong_CheckExact(a[13]) || at::impl::torch_function_mode_enabled()) return not_implemented();
  const int64_t dim = THPVariable_Unpack(a[3]).dim();
  if ((dim != 3 && dim != 4) || !main_tensor(a[3], dim, v, o)) return not_implemented();
  const bool step = dim == 3;
  q = plain(a[1]);
  if (q == nullptr || q->dim() != dim || q->size(1) > INT_MAX || q->size(-1) > INT_MAX) return not_implemented();
  kata_ssm_args r{};
  r.struct_size = sizeof r;
  r.B = (int)v->size(0); r.H = (int)v->size(1); r.T = step ? 1 : (int)v->size(2); r.d_v = (int)v->size(-1);
  r.G = (int)q->size(1); r.n = (int)q->size(-1);
  const at::ScalarType type = v->scalar_type();
  q = step ? view(a[1], v, {r.B, r.G, r.n}, type) : view(a[1], v, {r.B, r.G, r.T, r.n}, type);
  k = step ? view(a[2], v, {r.B, r.G, r.n}, type) : view(a[2], v, {r.B, r.G, r.T, r.n}, type);
  dt = plain(a[4]);
  if (q == nullptr || k == nullptr || dt == nullptr || dt->dim() != dim - 1 || dt->scalar_type() != type || dt->device() != v->device() || dt->size(0) != r.B ||
      dt->size(1) != r.H || (!step && dt->size(2) != r.T))
    return not_implemented();
  if (a[5] == Py_None || !optional(a[5], *v, {r.H}, at::kFloat, r.A) || !optional(a[6], *v, {r.H}, at::kFloat, r.D) ||
      !optional(a[7], *v, {r.H}, at::kFloat, r.dt_bias) || !optional(a[9], *v, {r.B, r.H, r.n, r.d_v}, at::kFloat, r.s_init) ||
      !optional(a[10], *v, {r.B, r.H, r.n, r.d_v}, at::kFloat, r.s_final) || !optional(a[11], *v, {r.B}, at::kInt, r.lengths) || !given_fits(a[12], *v))
    return not_implemented();
  int overflow = 0;
  const long impl = PyLong_AsLongAndOverflow(a[13], &overflow);
  if (!truth(a[8], r.dt_softplus) || overflow != 0 || impl < INT_MIN || impl > INT_MAX) return not_implemented();
  o.impl = (int)impl;
  PyObject* held = nullptr;
  if (step) o.stream = c10::cuda::getCurrentCUDAStream(v->device().index()).stream();
  else if (!stream_and_scratch(a[0], *v, KATA_FN_SSM_SCAN, r.B, r.H, r.T, r.n, r.d_v, 0, o, held)) return not_implemented();
  const Held hold{held};
  const at::Tensor out = make_output(a[12], *v, true);
  r.q = q->data_ptr(); r.k = k->data_ptr(); r.v = v->data_ptr(); r.dt = dt->data_ptr(); r.out = out.data_ptr();
  const int axes = (int)dim - 1;
  strides(*q, r.q_stride, axes);
  strides(*k, r.k_stride, axes);
  strides(*v, r.v_stride, axes);
  strides(*dt, r.dt_stride, axes);
  strides(out, r.out_stride, axes);
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = step ? kata_decode_ssm_step(&r, &o) : kata_fwd_ssm_scan(&r, &o);
  Py_END_ALLOW_THREADS
  return result(st, {&out});
  END_HANDLE_TH_ERRORS
}

#define KATA_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {KATA_METHOD(forward),        KATA_METHOD(decode),         KATA_METHOD(backward), KATA_METHOD(norm_rope), KATA_METHOD(norm_rope_bwd),
                          KATA_METHOD(short_conv),     KATA_METHOD(short_conv_bwd), KATA_METHOD(ssm),      {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_kata_torch", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The torch and the Python that this was compiled against; the binding looks for it in the file and loads no other.
extern "C" __attribute__((visibility("default"), used)) const char kata_host_tag[] = KATA_HOST_TAG;

PyMODINIT_FUNC PyInit__kata_torch(void) { return PyModule_Create(&kModule); }
