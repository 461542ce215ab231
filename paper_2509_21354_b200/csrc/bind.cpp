// The calls of a decode loop for Python callers that issue them token by token (kvE_decode_step; kvE_append_rope, kvE_append_rope_next and
// kvE_decode_attn_q4; kvE_set_len, kvE_pack_chunks and kvE_unpack_chunks beside them): argument checks and the call without the interpreter in between.  (One robot's decode loop is bound by the host: a token of a small cache takes the GPU 7 us.  Checks in Python and the
// conversion of ten arguments by ctypes took 2.9 us of the 6.3 us that a call took, 1.0 here; 7 tokens call by call 95 -> 82 us.)
#include <Python.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/kve.h"

namespace {

using DecodeStep = int (*)(void*, int, const void*, const void*, const void*, void*, float*, float, int, void*);

// address of a contiguous device tensor; rows > 0: of bf16 [rows, 128]
bool address(PyObject* o, int64_t rows, void** p) {
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, "a tensor is wanted");
    return false;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || !t.is_contiguous() ||
      (rows > 0 && (t.scalar_type() != at::kBFloat16 || t.dim() != 2 || t.size(0) != rows || t.size(1) != 128))) {
    PyErr_SetNone(PyExc_AssertionError);
    return false;
  }
  *p = t.data_ptr();
  return true;
}

// int(o): a float or any other number is taken too
long whole_number(PyObject* o) {
  if (PyLong_Check(o)) return PyLong_AsLong(o);
  PyObject* n = PyNumber_Long(o);
  if (!n) return -1;
  const long x = PyLong_AsLong(n);
  Py_DECREF(n);
  return x;
}

// decode_step(function address, handle, S, device, layer, k_new, v_new, q, out, lse or None, scale, n_reserve, stream or None) -> status
PyObject* decode_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 13) {
    PyErr_SetString(PyExc_TypeError, "13 arguments are wanted");
    return nullptr;
  }
  try {
    const auto fn = reinterpret_cast<DecodeStep>(PyLong_AsVoidPtr(a[0]));
    void* handle = a[1] == Py_None ? nullptr : PyLong_AsVoidPtr(a[1]);
    const long rows = PyLong_AsLong(a[2]), device = PyLong_AsLong(a[3]), layer = PyLong_AsLong(a[4]);
    const double scale = PyFloat_AsDouble(a[10]);
    const long n_reserve = whole_number(a[11]);
    void* stream = a[12] == Py_None ? nullptr : PyLong_AsVoidPtr(a[12]);
    if (PyErr_Occurred()) return nullptr;
    if (layer != (int)layer || n_reserve != (int)n_reserve) {
      PyErr_SetString(PyExc_OverflowError, "layer or n_reserve");
      return nullptr;
    }
    if (a[12] == Py_None) stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    void *k, *v, *q, *out, *lse = nullptr;
    if (!address(a[5], rows, &k) || !address(a[6], rows, &v) || !address(a[7], rows, &q) || !address(a[8], 0, &out)) return nullptr;
    if (a[9] != Py_None && !address(a[9], 0, &lse)) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS      // a launch may wait for room in the queue
    rc = fn(handle, (int)layer, k, v, q, out, static_cast<float*>(lse), (float)scale, (int)n_reserve, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

bool failed_assertion() {
  PyErr_SetNone(PyExc_AssertionError);
  return false;
}

bool tensor(PyObject* o, const at::Tensor** t) {
  if (!THPVariable_Check(o)) {
    PyErr_SetString(PyExc_TypeError, "a tensor is wanted");
    return false;
  }
  *t = &THPVariable_Unpack(o);
  return true;
}

// bf16 [B, n, heads, 128] on the device with contiguous rows, of any strides
bool strided_rows(PyObject* o, int64_t B, int64_t n, int64_t heads, long device, kvE_rows* rows) {
  const at::Tensor* t;
  if (!tensor(o, &t)) return false;
  if (t->scalar_type() != at::kBFloat16 || t->dim() != 4 || t->size(0) != B || t->size(1) != n || t->size(2) != heads || t->size(3) != 128 || t->stride(3) != 1 ||
      !t->is_cuda() || t->device().index() != device)
    return failed_assertion();
  rows->data = t->data_ptr();
  rows->stride_b = B > 1 ? t->stride(0) : 0;
  rows->stride_t = n > 1 ? t->stride(1) : 0;
  rows->stride_h = heads > 1 ? t->stride(2) : 0;
  return true;
}

// a contiguous device tensor of the given type and shape
bool shaped(PyObject* o, at::ScalarType type, at::IntArrayRef shape, long device, void** p) {
  const at::Tensor* t;
  if (!tensor(o, &t)) return false;
  if (t->scalar_type() != type || t->sizes() != shape || !t->is_cuda() || t->device().index() != device || !t->is_contiguous()) return failed_assertion();
  *p = t->data_ptr();
  return true;
}

// (handle, device and stream of the calls below)
struct Call { void* handle; long device; void* stream; bool own_stream; };
bool call_of(PyObject* handle, PyObject* device, PyObject* stream, Call* c) {
  c->handle = handle == Py_None ? nullptr : PyLong_AsVoidPtr(handle);
  c->device = PyLong_AsLong(device);
  c->stream = stream == Py_None ? nullptr : PyLong_AsVoidPtr(stream);
  c->own_stream = stream != Py_None;
  if (PyErr_Occurred()) return false;
  if (stream == Py_None) c->stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)c->device).stream();
  return true;
}
// A bf16 tensor for a result.  Of a call on a stream of its own it is that stream's: a block that the current stream has given back may still be in use there.
// (And the current stream will read it: it is not given out again before that has run.)
at::Tensor result_of(const Call& c, at::IntArrayRef shape) {
  const auto options = at::TensorOptions().dtype(at::kBFloat16).device(at::kCUDA, (c10::DeviceIndex)c.device);
  if (!c.own_stream) return at::empty(shape, options);
  const auto current = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)c.device);
  if (current.stream() == c.stream) return at::empty(shape, options);
  const c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(c.stream), (c10::DeviceIndex)c.device));
  at::Tensor t = at::empty(shape, options);
  if (t.numel() > 0) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), current);
  return t;
}
bool whole_numbers(PyObject* const* a, int n, int* x) {
  for (int i = 0; i < n; ++i) {
    const long y = whole_number(a[i]);
    if (PyErr_Occurred()) return false;
    if (y != (int)y) {
      PyErr_SetString(PyExc_OverflowError, "a whole number of 32 bits is wanted");
      return false;
    }
    x[i] = (int)y;
  }
  return true;
}

using AppendRope = int (*)(void*, int, const kvE_rows*, const kvE_rows*, const kvE_rows*, const int32_t*, int, const kvE_rope*, void*, int*, void*);
using AppendRopeNext = int (*)(void*, int, const kvE_rows*, const kvE_rows*, const kvE_rows*, const int32_t*, int, int, const kvE_rope*, void*, void*);

// append_rope(function address, handle, device, stream or None, next, layer, B, Hq, Hkv, n_reserve, q or None, k_new, v_new, address of the kvE_rope, positions or None,
// q_out or None) -> (status, q_out, chunks ready)
PyObject* append_rope(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 16) {
    PyErr_SetString(PyExc_TypeError, "16 arguments are wanted");
    return nullptr;
  }
  try {
    Call c;
    int x[6];      // next, layer, B, Hq, Hkv, n_reserve
    if (!call_of(a[1], a[2], a[3], &c) || !whole_numbers(a + 4, 6, x)) return nullptr;
    void* fn = PyLong_AsVoidPtr(a[0]);
    const auto* rope = static_cast<const kvE_rope*>(PyLong_AsVoidPtr(a[13]));
    if (PyErr_Occurred()) return nullptr;
    if (!rope) return failed_assertion(), nullptr;
    const at::Tensor* kt;
    if (!tensor(a[11], &kt)) return nullptr;
    const int64_t B = x[2], Hq = x[3], Hkv = x[4], n = kt->dim() > 1 ? kt->size(1) : 0;
    kvE_rows q, k, v;
    if (!strided_rows(a[11], B, n, Hkv, c.device, &k) || !strided_rows(a[12], B, n, Hkv, c.device, &v)) return nullptr;
    void *positions = nullptr, *out = nullptr;
    if (a[14] != Py_None && !shaped(a[14], at::kInt, {B, n, rope->n_axes}, c.device, &positions)) return nullptr;
    PyObject* result = a[15];
    if (a[10] == Py_None) {
      if (a[15] != Py_None) return failed_assertion(), nullptr;
      Py_INCREF(result);
    } else {
      if (!strided_rows(a[10], B, n, Hq, c.device, &q)) return nullptr;
      if (a[15] == Py_None) {
        at::Tensor t = result_of(c, {B, n, Hq, 128});
        out = t.data_ptr();
        result = THPVariable_Wrap(std::move(t));
        if (!result) return nullptr;
      } else {
        if (!shaped(a[15], at::kBFloat16, {B, n, Hq, 128}, c.device, &out)) return nullptr;
        Py_INCREF(result);
      }
    }
    int rc, ready = 0;
    const kvE_rows* pq = a[10] == Py_None ? nullptr : &q;
    Py_BEGIN_ALLOW_THREADS
    if (x[0])
      rc = reinterpret_cast<AppendRopeNext>(fn)(c.handle, x[1], pq, &k, &v, static_cast<const int32_t*>(positions), (int)n, x[5], rope, out, c.stream);
    else
      rc = reinterpret_cast<AppendRope>(fn)(c.handle, x[1], pq, &k, &v, static_cast<const int32_t*>(positions), (int)n, rope, out, &ready, c.stream);
    Py_END_ALLOW_THREADS
    PyObject* answer = Py_BuildValue("(iNi)", rc, result, ready);
    return answer;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

using AttnQ4 = int (*)(void*, int, const void*, int, int, int, void*, float*, float, void*);

// decode_attn_q4(function address, handle, device, stream or None, layer, B, Hq, dense, causal, scale, q, out or None, lse or None) -> (status, out)
PyObject* decode_attn_q4(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 13) {
    PyErr_SetString(PyExc_TypeError, "13 arguments are wanted");
    return nullptr;
  }
  try {
    Call c;
    int x[3];      // layer, B, Hq
    if (!call_of(a[1], a[2], a[3], &c) || !whole_numbers(a + 4, 3, x)) return nullptr;
    void* fn = PyLong_AsVoidPtr(a[0]);
    const int dense = PyObject_IsTrue(a[7]), causal = PyObject_IsTrue(a[8]);
    const double scale = PyFloat_AsDouble(a[9]);
    if (PyErr_Occurred() || dense < 0 || causal < 0) return nullptr;
    const at::Tensor* qt;
    if (!tensor(a[10], &qt)) return nullptr;
    const int64_t B = x[1], Hq = x[2], T = qt->dim() > 1 ? qt->size(1) : 0;
    void *q, *out, *lse = nullptr;
    if (!shaped(a[10], at::kBFloat16, {B, T, Hq, 128}, c.device, &q)) return nullptr;
    if (a[12] != Py_None && !shaped(a[12], at::kFloat, {B, T, Hq}, c.device, &lse)) return nullptr;
    PyObject* result = a[11];
    if (a[11] == Py_None) {
      at::Tensor t = result_of(c, {B, T, Hq, 128});
      out = t.data_ptr();
      result = THPVariable_Wrap(std::move(t));
      if (!result) return nullptr;
    } else {
      if (!shaped(a[11], at::kBFloat16, {B, T, Hq, 128}, c.device, &out)) return nullptr;
      Py_INCREF(result);
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = reinterpret_cast<AttnQ4>(fn)(c.handle, x[0], q, (int)T, dense, causal, out, static_cast<float*>(lse), (float)scale, c.stream);
    Py_END_ALLOW_THREADS
    return Py_BuildValue("(iN)", rc, result);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// chunks(function address, handle, device, stream or None, layer, chunk_begin, chunk_end) -> status (kvE_pack_chunks)
PyObject* chunks(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 7) {
    PyErr_SetString(PyExc_TypeError, "7 arguments are wanted");
    return nullptr;
  }
  try {
    Call c;
    int x[3];
    if (!call_of(a[1], a[2], a[3], &c) || !whole_numbers(a + 4, 3, x)) return nullptr;
    const auto fn = reinterpret_cast<int (*)(void*, int, int, int, void*)>(PyLong_AsVoidPtr(a[0]));
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(c.handle, x[0], x[1], x[2], c.stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// unpack_chunks(function address, handle, device, stream or None, layer, chunk_begin, chunk_end, S, C, k_out or None, v_out or None) -> (status, k_out, v_out)
PyObject* unpack_chunks(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 11) {
    PyErr_SetString(PyExc_TypeError, "11 arguments are wanted");
    return nullptr;
  }
  try {
    Call c;
    int x[5];      // layer, chunk_begin, chunk_end, S, C
    if (!call_of(a[1], a[2], a[3], &c) || !whole_numbers(a + 4, 5, x)) return nullptr;
    const auto fn = reinterpret_cast<int (*)(void*, int, int, int, void*, void*, void*)>(PyLong_AsVoidPtr(a[0]));
    const int64_t S = x[3], rows = (int64_t)(x[2] > x[1] ? x[2] - x[1] : 0) * x[4];
    PyObject* out[2] = {a[9], a[10]};
    void* p[2] = {};
    at::Tensor made[2];
    for (int i = 0; i < 2; ++i) {
      if (out[i] != Py_None) {
        if (!shaped(out[i], at::kBFloat16, {S, rows, 128}, c.device, &p[i])) return nullptr;
      } else {
        made[i] = result_of(c, {S, rows, 128});
        p[i] = made[i].data_ptr();
      }
    }
    int rc = 0;
    if (rows > 0) {      // (an empty tensor has no address)
      Py_BEGIN_ALLOW_THREADS
      rc = fn(c.handle, x[0], x[1], x[2], p[0], p[1], c.stream);
      Py_END_ALLOW_THREADS
    }
    for (int i = 0; i < 2; ++i) {
      if (made[i].defined()) out[i] = THPVariable_Wrap(std::move(made[i]));
      else Py_INCREF(out[i]);
    }
    return Py_BuildValue("(iNN)", rc, out[0], out[1]);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// set_len(function address, handle, device, stream or None, layer, n) -> status
PyObject* set_len(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 6) {
    PyErr_SetString(PyExc_TypeError, "6 arguments are wanted");
    return nullptr;
  }
  try {
    Call c;
    int x[2];
    if (!call_of(a[1], a[2], a[3], &c) || !whole_numbers(a + 4, 2, x)) return nullptr;
    const auto fn = reinterpret_cast<int (*)(void*, int, int, void*)>(PyLong_AsVoidPtr(a[0]));
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(c.handle, x[0], x[1], c.stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

#define KVE_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {KVE_METHOD(append_rope), KVE_METHOD(decode_attn_q4), KVE_METHOD(chunks), KVE_METHOD(unpack_chunks), KVE_METHOD(set_len), {"decode_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode_step)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kve_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kve_bind() { return PyModule_Create(&module); }
