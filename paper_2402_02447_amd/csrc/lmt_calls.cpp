// The calls of lmt.h for Python, part of the extension module _calls: takes tensors apart (address, shape, strides, type,
// device), checks that they fit together, and calls the function whose address lmt_connect() was given, without the
// interpreter's lock.  The smallest calls take the GPU a few microseconds; done in Python and ctypes, this alone takes longer.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "lmt.h"

namespace {

struct Functions {
  decltype(&lmt_embed) embed;
  decltype(&lmt_embed_grad) embed_grad;
  decltype(&lmt_quantize) quantize;
  decltype(&lmt_matmul) matmul;
  decltype(&lmt_cross_entropy) cross_entropy;
  PyObject *types, *current_device;  // {dtype: LMT_* or kBytes}; the device that is current, as a callable
};
constexpr int kBytes = 7;  // 8-bit whole numbers: scales, workspaces

PyObject *s_data_ptr, *s_shape, *s_stride, *s_dtype, *s_get_device, *s_cuda_stream;

struct Tensor {
  const char* name;
  void* at = nullptr;
  int type = -1;
  int dims = 0;
  int64_t size[2] = {1, 1}, stride[2] = {1, 1};
  uint64_t rows() const { return (uint64_t)size[0]; }
  uint64_t cols() const { return (uint64_t)size[1]; }
  uint64_t ld() const { return (uint64_t)stride[0]; }
};

// Arguments in turn; the first one that is wrong sets an exception and makes ok false.
struct Args {
  PyObject* const* a;
  Py_ssize_t i = 0;
  bool ok;
  Functions* f = nullptr;
  long device = -1;  // of the tensors so far

  Args(PyObject* const* args, Py_ssize_t given, Py_ssize_t want) : a(args), ok(given == want) {
    if (!ok) PyErr_Format(PyExc_TypeError, "%zd arguments given, %zd wanted", given, want);
    else ok = (f = static_cast<Functions*>(PyCapsule_GetPointer(a[i++], "lmt.functions"))) != nullptr;
  }
  void refuse(const char* name, const char* what) {
    if (ok) PyErr_Format(PyExc_ValueError, "%s: %s", name, what);
    ok = false;
  }
  void need(bool fits, const char* name, const char* what) {
    if (ok && !fits) refuse(name, what);
  }
  static bool numbers(PyObject* tuple, int n, int64_t* to) {
    for (int d = 0; d < n; ++d) {
      to[d] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, d));
      if (to[d] == -1 && PyErr_Occurred()) return false;
    }
    return true;
  }
  // A tensor of `dims` dimensions whose elements lie one behind the other along the last one.
  bool tensor(const char* name, int dims, Tensor* t, bool may_be_none = false) {
    t->name = name;
    if (!ok) return false;
    PyObject* x = a[i++];
    if (x == Py_None) {
      if (!may_be_none) refuse(name, "a tensor is wanted, not None");
      return false;
    }
    PyObject* shape = PyObject_GetAttr(x, s_shape);
    PyObject* stride = shape ? PyObject_CallMethodNoArgs(x, s_stride) : nullptr;
    PyObject* dtype = stride ? PyObject_GetAttr(x, s_dtype) : nullptr;
    PyObject* where = dtype ? PyObject_CallMethodNoArgs(x, s_get_device) : nullptr;
    PyObject* at = where ? PyObject_CallMethodNoArgs(x, s_data_ptr) : nullptr;
    ok = at != nullptr;
    if (ok) {
      PyObject* type = PyDict_GetItemWithError(f->types, dtype);
      const long place = PyLong_AsLong(where);
      t->at = (void*)(uintptr_t)PyLong_AsUnsignedLongLongMask(at);
      if (PyErr_Occurred()) {
        ok = false;
      } else if (!PyTuple_Check(shape) || !PyTuple_Check(stride) || PyTuple_GET_SIZE(shape) != dims || PyTuple_GET_SIZE(stride) != dims) {
        refuse(name, dims == 1 ? "one dimension is wanted" : "two dimensions are wanted");
      } else if (!type) {
        refuse(name, "not a type that is taken");
      } else if (place < 0) {
        refuse(name, "not on a GPU");
      } else if (device >= 0 && place != device) {
        refuse(name, "not on the device that the others are on");
      } else {
        device = place;
        t->type = (int)PyLong_AsLong(type);
        t->dims = dims;
        int64_t* size = t->size + (2 - dims);
        int64_t* step = t->stride + (2 - dims);
        ok = numbers(shape, dims, size) && numbers(stride, dims, step);
        if (ok && t->size[1] > 1 && t->stride[1] != 1) refuse(name, "elements of a row have to lie one behind the other");
        if (ok && t->size[0] > 1 && t->size[1] > 0 && t->stride[0] < t->size[1] && dims == 2) refuse(name, "rows overlap");
        if (t->size[0] <= 1 || t->size[1] == 0 || dims == 1) t->stride[0] = t->size[1];  // one row, or empty ones: the stride says nothing
      }
    }
    Py_XDECREF(shape), Py_XDECREF(stride), Py_XDECREF(dtype), Py_XDECREF(where), Py_XDECREF(at);
    return ok;
  }
  void matrix(const char* name, Tensor* t) {
    if (tensor(name, 2, t)) need(t->type == LMT_F32 || t->type == LMT_F16 || t->type == LMT_BF16, name, "fp32, fp16 or bf16 is wanted");
  }
  void ids(const char* name, Tensor* t) {
    if (tensor(name, 1, t)) need(t->type == LMT_I32 || t->type == LMT_I64, name, "32- or 64-bit whole numbers are wanted");
  }
  // One dimension of `type` with n elements, or None (nullptr).
  void* vector(const char* name, int type, uint64_t n) {
    Tensor t;
    if (!tensor(name, 1, &t, true)) return nullptr;
    need(t.type == type, name, type == LMT_F32 ? "fp32 is wanted" : "32-bit whole numbers are wanted");
    need(type == LMT_I32 ? t.cols() >= n : t.cols() == n, name, "has another number of elements");
    return t.at;
  }
  void* workspace(uint64_t* bytes) {
    Tensor t;
    *bytes = 0;
    if (!tensor("workspace", 1, &t, true)) return nullptr;
    need(t.type == kBytes, "workspace", "8-bit whole numbers are wanted");
    *bytes = t.cols();
    return t.at;
  }
  // A matrix in the 8-bit form and its scales; both None (false) if that is allowed.
  bool fp8(const char* name, const char* scales_name, Tensor* q, Tensor* s, bool may_be_none) {
    const bool there = tensor(name, 2, q, may_be_none);
    const bool scaled = tensor(scales_name, 2, s, may_be_none);
    if (!ok) return false;
    if (there != scaled) refuse(name, "a matrix and its scales go together");
    if (!there || !ok) return false;
    need(q->type == LMT_E4M3 || q->type == LMT_E5M2, name, "8-bit floating point is wanted");
    need(s->type == kBytes, scales_name, "8-bit whole numbers are wanted");
    need(q->cols() % 128 == 0 && q->ld() == q->cols(), name, "rows of whole blocks of 128 without gaps are wanted");
    need(s->rows() == q->rows() && s->cols() == 4 * ((q->cols() + 511) / 512) && s->ld() == s->cols(), scales_name, "rows of 4 bytes for every 512 elements are wanted");
    return ok;
  }
  double real() {
    double x = 0;
    if (ok) ok = !((x = PyFloat_AsDouble(a[i++])) == -1.0 && PyErr_Occurred());
    return x;
  }
  int64_t number() {
    int64_t x = 0;
    if (ok) ok = !((x = PyLong_AsLongLong(a[i++])) == -1 && PyErr_Occurred());
    return x;
  }
  bool truth() {
    int x = 0;
    if (ok) ok = (x = PyObject_IsTrue(a[i++])) >= 0;
    return x == 1;
  }
  // A stream: None, an object with cuda_stream (torch's), or a whole number.
  void* stream() {
    if (!ok) return nullptr;
    PyObject* x = a[i++];
    if (x == Py_None) return nullptr;
    PyObject* number = PyObject_GetAttr(x, s_cuda_stream);
    if (!number && PyErr_ExceptionMatches(PyExc_AttributeError)) {
      PyErr_Clear();
      Py_INCREF(number = x);
    }
    void* s = number ? (void*)(uintptr_t)PyLong_AsUnsignedLongLongMask(number) : nullptr;
    Py_XDECREF(number);
    ok = !PyErr_Occurred();
    return s;
  }
  template <typename F>
  PyObject* call(F go) {
    if (ok) {
      PyObject* now = PyObject_CallNoArgs(f->current_device);
      ok = now != nullptr;
      if (ok) need(PyLong_AsLong(now) == device, "the tensors", "not on the device that is current");
      Py_XDECREF(now);
    }
    if (!ok) return nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = go();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  }
};

// lmt_embed(functions, table, tokens, out, scale, status, stream)
PyObject* call_embed(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 7);
  Tensor table, tokens, out;
  a.matrix("table", &table), a.ids("tokens", &tokens), a.matrix("out", &out);
  const double scale = a.real();
  int32_t* status = static_cast<int32_t*>(a.vector("status", LMT_I32, 1));
  void* s = a.stream();
  a.need(out.rows() == tokens.cols() && out.cols() == table.cols(), "out", "a row for every token, as long as the table's, is wanted");
  return a.call([&] {
    return a.f->embed(table.at, table.type, table.rows(), table.cols(), table.ld(), tokens.at, tokens.type, tokens.cols(), scale, out.at, out.type, out.ld(), status, s);
  });
}

// lmt_embed_grad(functions, grad_out, tokens, grad, workspace, scale, skip_token, accumulate, status, stream)
PyObject* call_embed_grad(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 10);
  Tensor from, tokens, grad;
  uint64_t bytes;
  a.matrix("grad_out", &from), a.ids("tokens", &tokens), a.matrix("grad", &grad);
  void* workspace = a.workspace(&bytes);
  const double scale = a.real();
  const int64_t skip = a.number();
  const uint32_t flags = a.truth() ? LMT_ACCUMULATE : 0u;
  int32_t* status = static_cast<int32_t*>(a.vector("status", LMT_I32, 1));
  void* s = a.stream();
  a.need(from.rows() == tokens.cols() && from.cols() == grad.cols(), "grad_out", "a row for every token, as long as the table's, is wanted");
  return a.call([&] {
    return a.f->embed_grad(from.at, from.type, from.ld(), tokens.at, tokens.type, tokens.cols(), scale, skip, grad.at, grad.type, grad.rows(), grad.cols(), grad.ld(), flags,
                           status, workspace, bytes, s);
  });
}

// lmt_quantize(functions, x, q, scales, qt, scales_t, tile, stream)
PyObject* call_quantize(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 8);
  Tensor x, q, qs, t, ts;
  a.matrix("x", &x);
  const bool rows = a.fp8("q", "scales", &q, &qs, true), cols = a.fp8("qt", "scales_t", &t, &ts, true);
  const uint32_t flags = a.truth() ? LMT_TILE_SCALES : 0u;
  void* s = a.stream();
  a.need(rows || cols, "q", "neither q nor qt is given");
  a.need(!rows || (q.rows() == x.rows() && q.cols() == (x.cols() + 127) / 128 * 128), "q", "x's rows, in whole blocks of 128, are wanted");
  a.need(!cols || (t.rows() == x.cols() && t.cols() == (x.rows() + 127) / 128 * 128), "qt", "x's columns, in whole blocks of 128, are wanted");
  a.need(!rows || !cols || q.type == t.type, "qt", "q's type is wanted");
  return a.call([&] {
    return a.f->quantize(x.at, x.type, x.rows(), x.cols(), x.ld(), rows ? q.type : t.type, flags, q.at, static_cast<uint8_t*>(qs.at), t.at, static_cast<uint8_t*>(ts.at), s);
  });
}

// lmt_matmul(functions, a, a_scales, b, b_scales, c, workspace, accumulate, stream[, fp32_sums])
PyObject* call_matmul(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, n == 10 ? 10 : 9);
  Tensor x, xs, y, ys, c;
  uint64_t bytes;
  a.fp8("a", "a_scales", &x, &xs, false), a.fp8("b", "b_scales", &y, &ys, false);
  a.matrix("c", &c);
  void* workspace = a.workspace(&bytes);
  uint32_t flags = a.truth() ? LMT_ACCUMULATE : 0u;
  void* s = a.stream();
  if (n == 10 && a.truth()) flags |= LMT_FP32_SUMS;
  a.need(x.cols() == y.cols(), "b", "rows as long as a's are wanted");
  a.need(c.rows() == x.rows() && c.cols() == y.rows(), "c", "a's rows times b's rows are wanted");
  return a.call([&] {
    return a.f->matmul(x.at, x.type, static_cast<uint8_t*>(xs.at), y.at, y.type, static_cast<uint8_t*>(ys.at), x.rows(), y.rows(), x.cols(), c.at, c.type, c.ld(), flags, workspace, bytes, s);
  });
}

// lmt_cross_entropy(functions, logits, targets, loss, lse, grad, weights, ignore, status, stream)
PyObject* call_cross_entropy(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 10);
  Tensor x, targets, grad;
  a.matrix("logits", &x), a.ids("targets", &targets);
  float* loss = static_cast<float*>(a.vector("loss", LMT_F32, x.rows()));
  float* lse = static_cast<float*>(a.vector("lse", LMT_F32, x.rows()));
  const bool has_grad = a.tensor("grad", 2, &grad, true);
  const float* weights = static_cast<float*>(a.vector("weights", LMT_F32, x.rows()));
  const int64_t ignore = a.number();
  int32_t* status = static_cast<int32_t*>(a.vector("status", LMT_I32, 1));
  void* s = a.stream();
  a.need(targets.cols() == x.rows(), "targets", "one for every row is wanted");
  a.need(!has_grad || (grad.type == x.type && grad.rows() == x.rows() && grad.cols() == x.cols()), "grad", "the logits' type and shape are wanted");
  return a.call([&] {
    return a.f->cross_entropy(x.at, x.type, x.rows(), x.cols(), x.ld(), targets.at, targets.type, ignore, weights, loss, lse, has_grad ? grad.at : nullptr, has_grad ? grad.ld() : 0, status, s);
  });
}

void release(PyObject* capsule) {
  Functions* f = static_cast<Functions*>(PyCapsule_GetPointer(capsule, "lmt.functions"));
  Py_XDECREF(f->types), Py_XDECREF(f->current_device);
  PyMem_Free(f);
}

// lmt_connect(addresses of the five functions in the order of Functions, types, current_device) -> what every call takes first
PyObject* connect(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 7 || !PyDict_Check(args[5]) || !PyCallable_Check(args[6])) {
    PyErr_SetString(PyExc_TypeError, "five addresses, a dict and a callable are wanted");
    return nullptr;
  }
  void* at[5];
  for (int i = 0; i < 5; ++i) {
    at[i] = (void*)(uintptr_t)PyLong_AsUnsignedLongLong(args[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  Functions* f = static_cast<Functions*>(PyMem_Malloc(sizeof(Functions)));
  if (!f) return PyErr_NoMemory();
  f->embed = (decltype(f->embed))at[0], f->embed_grad = (decltype(f->embed_grad))at[1];
  f->quantize = (decltype(f->quantize))at[2], f->matmul = (decltype(f->matmul))at[3];
  f->cross_entropy = (decltype(f->cross_entropy))at[4];
  f->types = args[5], f->current_device = args[6];
  PyObject* capsule = PyCapsule_New(f, "lmt.functions", release);
  if (!capsule) {
    PyMem_Free(f);
    return nullptr;
  }
  Py_INCREF(f->types), Py_INCREF(f->current_device);
  return capsule;
}

#define METHOD(name, function) {name, (PyCFunction)(void (*)(void))function, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD("lmt_connect", connect), METHOD("lmt_embed", call_embed), METHOD("lmt_embed_grad", call_embed_grad), METHOD("lmt_quantize", call_quantize),
                         METHOD("lmt_matmul", call_matmul), METHOD("lmt_cross_entropy", call_cross_entropy), {nullptr, nullptr, 0, nullptr}};

}  // namespace

// The functions above; nullptr with an exception set.
PyMethodDef* lmt_methods() {
  s_data_ptr = PyUnicode_InternFromString("data_ptr"), s_shape = PyUnicode_InternFromString("shape"), s_stride = PyUnicode_InternFromString("stride");
  s_dtype = PyUnicode_InternFromString("dtype"), s_get_device = PyUnicode_InternFromString("get_device"), s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  return s_data_ptr && s_shape && s_stride && s_dtype && s_get_device && s_cuda_stream ? methods : nullptr;
}
