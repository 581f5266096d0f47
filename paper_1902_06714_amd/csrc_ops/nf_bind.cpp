// The tensors' side of the operators' binding: checks torch tensors, takes their
// pointers, sizes and pitches, and calls include/nf.h.  A small operator takes 3 to
// 4 us on the GPU, and marshalling its dozen arguments one by one from Python took
// longer than that (4 us of a call's 6 to 7); here it takes about one.
//
// Each function returns the call's nf_status; what is no fitting tensor raises
// TypeError or ValueError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <initializer_list>

#include "nf.h"

namespace {

PyObject *get_device = nullptr, *get_stream = nullptr;     // of torch._C

struct Raised {};                                          // a Python error is set

[[noreturn]] void refuse(PyObject* kind, const char* fmt, ...) {
  va_list a;
  va_start(a, fmt);
  PyErr_FormatV(kind, fmt, a);
  va_end(a);
  throw Raised();
}

// Others may run Python meanwhile: a launch waits where the queue is full, and so may
// an allocation.
struct Unlocked {
  PyThreadState* s = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(s); }
};
template <class F, class... A>
int call(F f, A... a) {
  Unlocked u;
  return (int)f(a...);
}

long as_long(PyObject* o) {
  const long v = o ? PyLong_AsLong(o) : -1;
  Py_XDECREF(o);
  if (PyErr_Occurred()) throw Raised();
  return v;
}
long current_device() { return as_long(PyObject_CallNoArgs(get_device)); }

// -1: the current stream; else a hipStream_t, 0 the default stream
void* queue(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  if (v != -1) return reinterpret_cast<void*>(v);
  PyObject* d = PyLong_FromLong(current_device());
  PyObject* r = d ? PyObject_CallOneArg(get_stream, d) : nullptr;
  Py_XDECREF(d);
  const unsigned long long s = r ? PyLong_AsUnsignedLongLong(r) : 0;
  Py_XDECREF(r);
  if (PyErr_Occurred()) throw Raised();
  return reinterpret_cast<void*>(s);
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a torch tensor on the GPU", name);
  return THPVariable_Unpack(o);
}

int elem_code(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return NF_F32;
    case at::kBFloat16: return NF_BF16;
    case at::kHalf: return NF_F16;
    default: return -1;
  }
}

// The current device, asked once a call, which all of a call's tensors lie on.
struct Device {
  long at = -1;
  void holds(const at::Tensor& t, const char* name) {
    if (at < 0) at = current_device();
    if (t.get_device() != at) refuse(PyExc_ValueError, "%s is not on the current device", name);
  }
};

// nf_dtype of a tensor on the device
int elem(Device& dev, const at::Tensor& t, const char* name) {
  const int code = elem_code(t);
  if (code < 0 || !t.is_cuda()) refuse(PyExc_ValueError, "%s must be an fp32, bf16 or fp16 GPU tensor", name);
  dev.holds(t, name);
  return code;
}

struct Matrix {
  void* p;
  int64_t rows, cols, ld;
};
Matrix matrix(const at::Tensor& t, const char* name) {
  if (t.dim() != 2) refuse(PyExc_ValueError, "%s must be 2-D", name);
  Matrix m{t.data_ptr(), t.size(0), t.size(1), t.stride(0)};
  if (m.rows <= 1) m.ld = m.cols;
  if ((t.stride(1) != 1 && m.cols > 1) || m.ld < m.cols)
    refuse(PyExc_ValueError, "%s's rows must be contiguous and apart", name);
  return m;
}
Matrix matrix(const at::Tensor& t, const char* name, int64_t rows, int64_t cols) {
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols)
    refuse(PyExc_ValueError, "%s must be 2-D of shape (%lld, %lld)", name, (long long)rows, (long long)cols);
  return matrix(t, name);
}
Matrix bytes_matrix(Device& dev, PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != at::kChar || !t.is_cuda()) refuse(PyExc_ValueError, "%s must be an int8 GPU tensor", name);
  dev.holds(t, name);
  return matrix(t, name);
}

// pointer of a contiguous GPU tensor of this type and shape (of any with the sizes of
// `like`), NULL for None
void* whole(Device& dev, const at::Tensor& t, const char* name, at::ScalarType type, at::IntArrayRef shape) {
  if (t.scalar_type() != type || !t.is_cuda() || t.sizes() != shape || !t.is_contiguous())
    refuse(PyExc_ValueError, "%s must be a contiguous GPU tensor of the type and shape that go with the others", name);
  dev.holds(t, name);
  return t.data_ptr();
}
void* vector(Device& dev, PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape) {
  return o == Py_None ? nullptr : whole(dev, tensor(o, name), name, type, shape);
}

// the caller's workspace, or one from torch's allocator, which hands it on only
// behind this call on the current stream
struct Work {
  at::Tensor keep;
  void* p = nullptr;
  int64_t bytes = 0;
  // need: below 0 for sizes that the call refuses, which tells why
  void take(Device& dev, PyObject* o, int64_t need, const at::Tensor& like) {
    if (o == Py_None) {
      if (need <= 0) return;
      Unlocked u;
      keep = at::empty({need}, like.options().dtype(at::kByte));
    } else {
      keep = tensor(o, "work");
      if (!keep.is_cuda() || !keep.is_contiguous()) refuse(PyExc_ValueError, "work must be a contiguous GPU tensor");
      dev.holds(keep, "work");
    }
    p = keep.data_ptr();
    bytes = keep.numel() * keep.element_size();
  }
};

// A call's status, once the tensors that it wrote have a new version: what autograd kept of
// their values before is no longer there.
int wrote(std::initializer_list<PyObject*> outs, int st) {
  if (st == NF_OK)
    for (PyObject* o : outs)
      if (o != Py_None) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
      }
  return st;
}

double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return v;
}
int64_t whole_number(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}

// f's status, or the Python error that it set; n arguments are wanted
template <class F>
PyObject* guarded(Py_ssize_t have, Py_ssize_t want, F&& f) {
  try {
    if (have != want) refuse(PyExc_TypeError, "%zd arguments, %zd are wanted", have, want);
    return PyLong_FromLong(f());
  } catch (const Raised&) {
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());
  }
  return nullptr;
}

// logits, targets, logp, entropy, stat, top_ids, top_logp, scale, work, stream
PyObject* logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    Device dev;
    const at::Tensor& x = tensor(a[0], "logits");
    const int code = elem(dev, x, "logits");
    const Matrix m = matrix(x, "logits");
    int64_t top = 0;
    for (int k : {6, 5})
      if (a[k] != Py_None) top = tensor(a[k], "top").dim() ? THPVariable_Unpack(a[k]).size(-1) : 0;
    if (top > NF_TOP_MAX) top = NF_TOP_MAX + 1;            // refused below
    Work w;
    w.take(dev, a[8], nf_logprobs_work(code, m.rows, m.cols < 1 ? 1 : m.cols, (int)(top > NF_TOP_MAX ? 0 : top), 0), x);
    return wrote({a[2], a[3], a[4], a[5], a[6]},
                 call(nf_logprobs, m.p, code, m.rows, m.cols, m.ld, (float)number(a[7]),
                      (const int64_t*)vector(dev, a[1], "targets", at::kLong, {m.rows}), (int)top,
                      (float*)vector(dev, a[2], "logp", at::kFloat, {m.rows}),
                      (float*)vector(dev, a[3], "entropy", at::kFloat, {m.rows}),
                      (float*)vector(dev, a[4], "stat", at::kFloat, {m.rows, 2}),
                      (int32_t*)vector(dev, a[5], "top_ids", at::kInt, {m.rows, top}),
                      (float*)vector(dev, a[6], "top_logp", at::kFloat, {m.rows, top}), w.p, w.bytes, queue(a[9])));
  });
}

Matrix gradient(Device& dev, PyObject* o, int code, const Matrix& like) {
  const at::Tensor& t = tensor(o, "dlogits");
  if (elem(dev, t, "dlogits") != code) refuse(PyExc_ValueError, "dlogits must have the type of the logits");
  return matrix(t, "dlogits", like.rows, like.cols);
}

// logits, targets, g_logp, g_entropy, dlogits, logp, entropy, stat, scale, work, stream
PyObject* logprobs_train(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&] {
    Device dev;
    const at::Tensor& x = tensor(a[0], "logits");
    const int code = elem(dev, x, "logits");
    const Matrix m = matrix(x, "logits"), d = gradient(dev, a[4], code, m);
    Work w;
    w.take(dev, a[9], nf_logprobs_work(code, m.rows, m.cols < 1 ? 1 : m.cols, 0, 1), x);
    return wrote({a[4], a[5], a[6], a[7]},
                 call(nf_logprobs_train, m.p, code, m.rows, m.cols, m.ld, (float)number(a[8]),
                      (const int64_t*)vector(dev, a[1], "targets", at::kLong, {m.rows}),
                      (const float*)vector(dev, a[2], "g_logp", at::kFloat, {m.rows}),
                      (const float*)vector(dev, a[3], "g_entropy", at::kFloat, {m.rows}),
                      (float*)vector(dev, a[5], "logp", at::kFloat, {m.rows}),
                      (float*)vector(dev, a[6], "entropy", at::kFloat, {m.rows}),
                      (float*)vector(dev, a[7], "stat", at::kFloat, {m.rows, 2}), d.p, d.ld, w.p, w.bytes, queue(a[10])));
  });
}

// logits, targets, stat, entropy, g_logp, g_entropy, dlogits, scale, stream
PyObject* logprobs_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    Device dev;
    const at::Tensor& x = tensor(a[0], "logits");
    const int code = elem(dev, x, "logits");
    const Matrix m = matrix(x, "logits"), d = gradient(dev, a[6], code, m);
    return wrote({a[6]},
                 call(nf_logprobs_grad, m.p, code, m.rows, m.cols, m.ld, (float)number(a[7]),
                      (const int64_t*)vector(dev, a[1], "targets", at::kLong, {m.rows}),
                      (const float*)vector(dev, a[2], "stat", at::kFloat, {m.rows, 2}),
                      (const float*)vector(dev, a[3], "entropy", at::kFloat, {m.rows}),
                      (const float*)vector(dev, a[4], "g_logp", at::kFloat, {m.rows}),
                      (const float*)vector(dev, a[5], "g_entropy", at::kFloat, {m.rows}), d.p, d.ld, queue(a[8])));
  });
}

struct Stack {
  void* p;
  int64_t count, rows, cols, ld, stride;
};
Stack stack(const at::Tensor& t, const char* name) {
  const int64_t d = t.dim();
  if (d != 2 && d != 3) refuse(PyExc_ValueError, "%s must be a matrix or a stack of matrices", name);
  Stack s{t.data_ptr(), d == 3 ? t.size(0) : 1, t.size(-2), t.size(-1), t.stride(-2), 0};
  if (s.count > 1) s.stride = t.stride(0);
  if (s.rows <= 1) s.ld = s.cols;
  if ((t.stride(-1) != 1 && s.cols > 1) || s.ld < s.cols)
    refuse(PyExc_ValueError, "%s's rows must be contiguous and apart", name);
  return s;
}

// x, out, work, stream
PyObject* orthogonalize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 4, [&] {
    Device dev;
    const at::Tensor &x = tensor(a[0], "x"), &out = tensor(a[1], "out");
    const int code = elem(dev, x, "x");
    if (elem(dev, out, "out") != code || out.sizes() != x.sizes()) refuse(PyExc_ValueError, "out must have x's type and shape");
    const Stack s = stack(x, "x"), o = stack(out, "out");
    Work w;
    w.take(dev, a[2], nf_orthogonalize_work(code, s.count, s.rows, s.cols), x);
    return wrote({a[1]},
                 call(nf_orthogonalize, s.p, code, s.count, s.rows, s.cols, s.ld, s.stride, o.p, o.ld, o.stride, w.p, w.bytes,
                      queue(a[3])));
  });
}

// w, m, g, w_out, m_out, eta, momentum, nesterov, decay, work, stream
PyObject* muon_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&] {
    Device dev;
    const at::Tensor &w = tensor(a[0], "w"), &g = tensor(a[2], "g");
    const int wc = elem(dev, w, "w"), gc = elem(dev, g, "g");
    const auto shape = w.sizes();
    const Stack s = stack(w, "w");
    void* const wp = whole(dev, w, "w", w.scalar_type(), shape);
    void* const gp = whole(dev, g, "g", g.scalar_type(), shape);
    void* const mp = whole(dev, tensor(a[1], "m"), "m", at::kFloat, shape);
    void* const wo = whole(dev, tensor(a[3], "w_out"), "w_out", w.scalar_type(), shape);
    void* const mo = whole(dev, tensor(a[4], "m_out"), "m_out", at::kFloat, shape);
    Work k;
    k.take(dev, a[9], nf_orthogonalize_work(wc, s.count, s.rows, s.cols), w);
    return wrote({a[3], a[4]},
                 call(nf_muon_step, wp, wc, (const float*)mp, gp, gc, s.count, s.rows, s.cols, (float)number(a[5]),
                      (float)number(a[6]), (int)whole_number(a[7]), (float)number(a[8]), wo, (float*)mo, k.p,
                      k.bytes, queue(a[10])));
  });
}

int64_t whole16(int64_t v) { return (v + 15) / 16 * 16; }

// x, q, scale, stream
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 4, [&] {
    Device dev;
    const at::Tensor& x = tensor(a[0], "x");
    const int code = elem(dev, x, "x");
    const Matrix m = matrix(x, "x"), q = bytes_matrix(dev, a[1], "q");
    if (q.rows != m.rows || q.cols < whole16(m.cols))
      refuse(PyExc_ValueError, "q must have x's rows and columns, these up to a multiple of 16");
    return wrote({a[1], a[2]},
                 call(nf_quantize_rows, m.p, code, m.rows, m.cols, m.ld, (int8_t*)q.p, q.ld,
                      (float*)vector(dev, a[2], "scale", at::kFloat, {m.rows}), queue(a[3])));
  });
}

// xq, x_scale, wq, w_scale, y, inputs, bias, act, stream
PyObject* linear_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    Device dev;
    const Matrix x = bytes_matrix(dev, a[0], "xq"), w = bytes_matrix(dev, a[2], "wq");
    const int64_t inputs = whole_number(a[5]);
    if (x.cols < whole16(inputs) || w.cols < whole16(inputs))
      refuse(PyExc_ValueError, "xq and wq must hold the inputs, up to a multiple of 16");
    const at::Tensor& yt = tensor(a[4], "y");
    const int yc = elem(dev, yt, "y");
    const Matrix y = matrix(yt, "y", x.rows, w.rows);
    return wrote({a[4]},
                 call(nf_linear_i8, (const int8_t*)x.p, x.ld, (const float*)vector(dev, a[1], "x_scale", at::kFloat, {x.rows}),
                      (const int8_t*)w.p, w.ld, (const float*)vector(dev, a[3], "w_scale", at::kFloat, {w.rows}),
                      (const float*)vector(dev, a[6], "bias", at::kFloat, {w.rows}), (int)whole_number(a[7]), x.rows, inputs,
                      w.rows, y.p, yc, y.ld, queue(a[8])));
  });
}

// x, wq, w_scale, y, bias, act, work, stream
PyObject* linear_i8_dynamic(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    Device dev;
    const at::Tensor &xt = tensor(a[0], "x"), &yt = tensor(a[3], "y");
    const int xc = elem(dev, xt, "x"), yc = elem(dev, yt, "y");
    const Matrix x = matrix(xt, "x"), w = bytes_matrix(dev, a[1], "wq");
    if (w.cols < whole16(x.cols)) refuse(PyExc_ValueError, "wq must hold x's columns, up to a multiple of 16");
    const Matrix y = matrix(yt, "y", x.rows, w.rows);
    const auto* ws = (const float*)vector(dev, a[2], "w_scale", at::kFloat, {w.rows});
    const auto* bs = (const float*)vector(dev, a[4], "bias", at::kFloat, {w.rows});
    Work k;
    k.take(dev, a[6], nf_linear_i8_work(x.rows, x.cols), xt);
    return wrote({a[3]},
                 call(nf_linear_i8_dynamic, x.p, xc, x.ld, (const int8_t*)w.p, w.ld, ws, bs, (int)whole_number(a[5]), x.rows,
                      x.cols, w.rows, y.p, yc, y.ld, k.p, k.bytes, queue(a[7])));
  });
}

#define NF_ENTRY(name) {#name, (PyCFunction)(void (*)())name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {NF_ENTRY(logprobs), NF_ENTRY(logprobs_train), NF_ENTRY(logprobs_grad), NF_ENTRY(orthogonalize),
                         NF_ENTRY(muon_step), NF_ENTRY(quantize_rows), NF_ENTRY(linear_i8), NF_ENTRY(linear_i8_dynamic),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_nfbind", "Calls of the operators with torch tensors.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__nfbind() {
  PyObject* c = PyImport_ImportModule("torch._C");
  if (!c) return nullptr;
  get_device = PyObject_GetAttrString(c, "_cuda_getDevice");
  get_stream = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
  Py_DECREF(c);
  PyErr_Clear();                                           // a torch without GPUs: no tensor passes elem()
  return PyModule_Create(&module);
}
