// The Python calls of the microscaled 4-bit operators, without the interpreter's part of them: checks of the tensors,
// outputs from torch's allocator, the current stream and the C entry point.  A decode call's kernels take a few
// microseconds, so the host's time counts: a product took 10.8 us through ctypes and torch's Python, 3.7 here.
//
// A function takes what the Python function of the same operator takes, outputs excepted, and returns its result, or the
// status of a call that the library refused, or None where the arguments are not the ordinary ones (other types, shapes,
// strides, a device that is not the current one): the Python function then says what is wrong with them.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/cat_w4a4.h"

namespace {

// A tensor argument on a GPU, dense, of `dims` dimensions; else null.
const at::Tensor* dense(PyObject* o, int64_t dims) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() && t.layout() == at::kStrided && t.dim() == dims && t.is_contiguous() ? &t : nullptr;
}
// The library launches on the current device, whatever its pointers are of.
bool current(const at::Tensor& t) { return t.get_device() == c10::cuda::current_device(); }
bool real(const at::Tensor& t) { return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16; }
cat_dtype code(const at::Tensor& t) { return t.scalar_type() == at::kFloat ? CAT_F32 : CAT_BF16; }

// The type of a product's output: float32 for None.  False: some other type.
bool out_type(PyObject* o, at::ScalarType* t) {
  *t = at::kFloat;
  if (o == Py_None) return true;
  if (!THPDtype_Check(o)) return false;
  *t = reinterpret_cast<THPDtype*>(o)->scalar_type;
  return *t == at::kFloat || *t == at::kBFloat16;
}

cat_stream_t stream_of(const at::Tensor& t) {
  return reinterpret_cast<cat_stream_t>(c10::cuda::getCurrentCUDAStream(t.get_device()).stream());
}
// A new tensor on the current device, from torch's allocator without its dispatcher (0.44 us, 0.81 with it).
at::Tensor make(int64_t rows, int64_t cols, at::ScalarType type) {
  return at::detail::empty_generic({rows, cols}, c10::cuda::CUDACachingAllocator::get(),
                                   c10::DispatchKeySet(c10::DispatchKey::CUDA), type, c10::nullopt);
}
at::Tensor bytes(int64_t rows, int64_t cols) { return make(rows, cols, at::kByte); }
uint8_t* u8(const at::Tensor& t) { return static_cast<uint8_t*>(t.data_ptr()); }

// Codes [.., half] and scales [.., pitch] of one device; the rows' shapes are the caller's to compare.
bool form(const at::Tensor* q, const at::Tensor* s, int64_t device) {
  if (!q || !s || q->scalar_type() != at::kByte || s->scalar_type() != at::kByte) return false;
  const int64_t dims = q->dim();
  for (int64_t i = 0; i + 1 < dims; ++i)
    if (q->size(i) != s->size(i)) return false;
  return s->size(dims - 1) == (q->size(dims - 1) + 255) / 256 * 16 && q->get_device() == device && s->get_device() == device;
}

PyObject* wrap(std::initializer_list<at::Tensor> out) {
  PyObject* tuple = PyTuple_New((Py_ssize_t)out.size());
  if (!tuple) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor& t : out) {
    PyObject* o = THPVariable_Wrap(t);
    if (!o) {
      Py_DECREF(tuple);
      return nullptr;
    }
    PyTuple_SET_ITEM(tuple, i++, o);
  }
  return tuple;
}

// What a call does behind its checks -- its outputs' allocation and the launch -- goes without the interpreter's lock: a thread
// that waits for memory, or for room in the launch queue, does not stop the others.
class Unlocked {
 public:
  Unlocked() : state_(PyEval_SaveThread()) {}
  ~Unlocked() { PyEval_RestoreThread(state_); }
  Unlocked(const Unlocked&) = delete;

 private:
  PyThreadState* state_;
};
template <typename F>
cat_status unlocked(F&& call) {
  const Unlocked here;
  return call();
}

bool count(Py_ssize_t got, Py_ssize_t want) {
  if (got == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
  return false;
}

// (x, rows)
PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (!count(nargs, 2)) return nullptr;
  const at::Tensor* x = dense(args[0], 2);
  if (!x || !real(*x) || !current(*x)) Py_RETURN_NONE;
  const at::Tensor* rows = nullptr;
  const int64_t n = x->size(0), d = x->size(1);
  if (args[1] != Py_None && (!(rows = dense(args[1], 1)) || rows->scalar_type() != at::kInt || rows->get_device() != x->get_device()))
    Py_RETURN_NONE;
  const int64_t m = rows ? rows->size(0) : n;
  at::Tensor xq, xs;
  const cat_status st = unlocked([&] {
    xq = bytes(m, d / 2), xs = bytes(m, (d + 511) / 512 * 16);
    return cat_mx_quantize(x->data_ptr(), code(*x), n, d, rows ? static_cast<const int32_t*>(rows->data_ptr()) : nullptr, m, u8(xq),
                           u8(xs), stream_of(*x));
  });
  return st == CAT_OK ? wrap({xq, xs}) : PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

// (gu)
PyObject* swiglu_quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (!count(nargs, 1)) return nullptr;
  const at::Tensor* gu = dense(args[0], 2);
  if (!gu || !real(*gu) || gu->size(1) % 2 || !current(*gu)) Py_RETURN_NONE;
  const int64_t n = gu->size(0), d = gu->size(1) / 2;
  at::Tensor xq, xs;
  const cat_status st = unlocked([&] {
    xq = bytes(n, d / 2), xs = bytes(n, (d + 511) / 512 * 16);
    return cat_mx_swiglu_quantize(gu->data_ptr(), code(*gu), n, d, u8(xq), u8(xs), stream_of(*gu));
  });
  return st == CAT_OK ? wrap({xq, xs}) : PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

// (x, weight, eps, residual): without a residual, h is x
PyObject* rmsnorm_quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (!count(nargs, 4)) return nullptr;
  const at::Tensor *x = dense(args[0], 2), *w = dense(args[1], 1), *r = nullptr;
  if (!x || !w || !real(*x) || !real(*w) || w->size(0) != x->size(1) || w->get_device() != x->get_device() || !current(*x))
    Py_RETURN_NONE;
  const double eps = PyFloat_AsDouble(args[2]);
  if (eps == -1.0 && PyErr_Occurred()) return nullptr;
  const int64_t n = x->size(0), d = x->size(1);
  if (args[3] != Py_None && (!(r = dense(args[3], 2)) || r->scalar_type() != x->scalar_type() || r->size(0) != n || r->size(1) != d ||
                             r->get_device() != x->get_device()))
    Py_RETURN_NONE;
  at::Tensor h = *x, xq, xs;
  const cat_status st = unlocked([&] {
    if (r) h = make(n, d, x->scalar_type());
    xq = bytes(n, d / 2), xs = bytes(n, (d + 511) / 512 * 16);
    return cat_mx_rmsnorm_quantize(x->data_ptr(), r ? r->data_ptr() : nullptr, code(*x), w->data_ptr(), code(*w), n, d, (float)eps,
                                   r ? h.data_ptr() : nullptr, u8(xq), u8(xs), stream_of(*x));
  });
  return st == CAT_OK ? wrap({xq, xs, h}) : PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

// (xq, xs, out_dtype)
PyObject* dequantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (!count(nargs, 3)) return nullptr;
  const at::Tensor *q = dense(args[0], 2), *s = dense(args[1], 2);
  at::ScalarType type;
  if (!form(q, s, q ? q->get_device() : -1) || !out_type(args[2], &type) || !current(*q)) Py_RETURN_NONE;
  const int64_t n = q->size(0), d = 2 * q->size(1);
  at::Tensor out;
  const cat_status st = unlocked([&] {
    out = make(n, d, type);
    return cat_mx_dequantize(u8(*q), u8(*s), n, d, code(out), out.data_ptr(), stream_of(*q));
  });
  return st == CAT_OK ? THPVariable_Wrap(out) : PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

// (xq, xs, Wq, ws, out_dtype)
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (!count(nargs, 5)) return nullptr;
  const at::Tensor *q = dense(args[0], 2), *s = dense(args[1], 2), *wq = dense(args[2], 2), *ws = dense(args[3], 2);
  at::ScalarType type;
  const int64_t device = q ? q->get_device() : -1;
  if (!form(q, s, device) || !form(wq, ws, device) || wq->size(1) != q->size(1) || !out_type(args[4], &type) || !current(*q))
    Py_RETURN_NONE;
  const int64_t n = q->size(0), d_out = wq->size(0);
  at::Tensor y;
  const cat_status st = unlocked([&] {
    y = make(n, d_out, type);
    return cat_mx_linear(u8(*q), u8(*s), u8(*wq), u8(*ws), n, 2 * q->size(1), d_out, code(y), y.data_ptr(), stream_of(*q));
  });
  return st == CAT_OK ? THPVariable_Wrap(y) : PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

// (xq, xs, Wq, ws, offsets, out_dtype)
PyObject* linear_grouped(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (!count(nargs, 6)) return nullptr;
  const at::Tensor *q = dense(args[0], 2), *s = dense(args[1], 2), *wq = dense(args[2], 3), *ws = dense(args[3], 3),
                   *o = dense(args[4], 1);
  at::ScalarType type;
  const int64_t device = q ? q->get_device() : -1;
  if (!form(q, s, device) || !form(wq, ws, device) || wq->size(2) != q->size(1) || !o || o->scalar_type() != at::kInt ||
      o->size(0) != wq->size(0) + 1 || o->get_device() != device || !out_type(args[5], &type) || !current(*q))
    Py_RETURN_NONE;
  const int64_t m = q->size(0), d_out = wq->size(1);
  at::Tensor y;
  const cat_status st = unlocked([&] {
    y = make(m, d_out, type);
    return cat_mx_linear_grouped(u8(*q), u8(*s), u8(*wq), u8(*ws), static_cast<const int32_t*>(o->data_ptr()), wq->size(0), m,
                                 2 * q->size(1), d_out, code(y), y.data_ptr(), stream_of(*q));
  });
  return st == CAT_OK ? THPVariable_Wrap(y) : PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

#define CAT_CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef calls[] = {CAT_CALL(quantize), CAT_CALL(swiglu_quantize), CAT_CALL(rmsnorm_quantize), CAT_CALL(dequantize),
                       CAT_CALL(linear), CAT_CALL(linear_grouped), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mx_calls", nullptr, -1, calls, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mx_calls(void) { return PyModule_Create(&module); }
