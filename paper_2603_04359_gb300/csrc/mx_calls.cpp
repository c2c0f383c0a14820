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

// A cache [pages][2][hkv][bytes of a page] of heads of d channels.
struct Cache {
  const at::Tensor* t;
  int64_t pages, page, hkv;
  Cache(PyObject* o, int64_t d) : t(dense(o, 4)), pages(0), page(0), hkv(0) {
    if (!t) return;
    const int64_t part = t->size(3), token = d / 2 + d / 32;
    if (t->scalar_type() != at::kByte || t->size(1) != 2 || token <= 0 || part % token != 0 ||
        cat_mx_cache_page_bytes(part / token, d) != part) {
      t = nullptr;
      return;
    }
    pages = t->size(0), page = part / token, hkv = t->size(2);
  }
  bool on(int64_t device) const { return t && t->get_device() == device; }
};
// int32 [n] of a device, any n for -1
const at::Tensor* numbers(PyObject* o, int64_t n, int64_t device) {
  const at::Tensor* t = dense(o, 1);
  return t && t->scalar_type() == at::kInt && (n < 0 || t->size(0) == n) && t->get_device() == device ? t : nullptr;
}
// Whether two tensors share memory.
bool shared(const at::Tensor& a, const at::Tensor& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.data_ptr()), y = reinterpret_cast<uintptr_t>(b.data_ptr());
  return x < y + b.nbytes() && y < x + a.nbytes();
}
const int32_t* i32(const at::Tensor* t) { return t ? static_cast<const int32_t*>(t->data_ptr()) : nullptr; }
at::Tensor make3(int64_t a, int64_t b, int64_t c, at::ScalarType type) {
  return at::detail::empty_generic({a, b, c}, c10::cuda::CUDACachingAllocator::get(), c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                   type, c10::nullopt);
}

// (k, v, slots, cache): 0 once done
PyObject* cache_write(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (!count(nargs, 4)) return nullptr;
  const at::Tensor *k = dense(args[0], 3), *v = dense(args[1], 3);
  if (!k || !v || !real(*k) || v->scalar_type() != k->scalar_type() || v->sizes() != k->sizes() || v->get_device() != k->get_device() ||
      !current(*k))
    Py_RETURN_NONE;
  const int64_t n = k->size(0), hkv = k->size(1), d = k->size(2);
  const at::Tensor* slots = numbers(args[2], n, k->get_device());
  const Cache c(args[3], d);
  if (!slots || !c.on(k->get_device()) || c.hkv != hkv || shared(*k, *c.t) || shared(*v, *c.t) || shared(*slots, *c.t)) Py_RETURN_NONE;
  const cat_status st = unlocked([&] {
    return cat_mx_cache_write(k->data_ptr(), v->data_ptr(), code(*k), n, i32(slots), u8(*c.t), c.pages, c.page, hkv, d, stream_of(*k));
  });
  return PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

// An integer argument; false where it is none (or too large).
bool integer(PyObject* o, int64_t* v) {
  if (!PyLong_Check(o)) return false;
  int over = 0;
  *v = PyLong_AsLongLongAndOverflow(o, &over);
  return over == 0;
}

// (cache, slots, d, out_dtype)
PyObject* cache_read(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (!count(nargs, 4)) return nullptr;
  int64_t d;
  at::ScalarType type;
  if (!integer(args[2], &d) || !out_type(args[3], &type)) Py_RETURN_NONE;
  const Cache c(args[0], d);
  if (!c.t || !current(*c.t)) Py_RETURN_NONE;
  const at::Tensor* slots = numbers(args[1], -1, c.t->get_device());
  if (!slots) Py_RETURN_NONE;
  const int64_t m = slots->size(0);
  at::Tensor k, v;
  const cat_status st = unlocked([&] {
    k = make3(m, c.hkv, d, type), v = make3(m, c.hkv, d, type);
    return cat_mx_cache_read(u8(*c.t), c.pages, c.page, c.hkv, d, i32(slots), m, code(k), k.data_ptr(), v.data_ptr(), stream_of(*c.t));
  });
  return st == CAT_OK ? wrap({k, v}) : PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

// (qkv, d, positions, cos, sin, slots, cache, q_weight, k_weight, eps, interleaved)
PyObject* rope_cache_write(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (!count(nargs, 11)) return nullptr;
  const at::Tensor* x = dense(args[0], 2);
  int64_t d;
  if (!x || !real(*x) || !integer(args[1], &d) || d <= 0 || !current(*x)) Py_RETURN_NONE;
  const int64_t device = x->get_device(), n = x->size(0), heads = x->size(1) / d;
  const Cache c(args[6], d);
  const at::Tensor *positions = numbers(args[2], n, device), *cos = dense(args[3], 2), *sin = dense(args[4], 2),
                   *slots = numbers(args[5], n, device);
  if (!c.on(device) || x->size(1) % d != 0 || heads <= 2 * c.hkv || !positions || !slots || !cos || !sin ||
      cos->scalar_type() != at::kFloat || sin->scalar_type() != at::kFloat || cos->sizes() != sin->sizes() ||
      cos->get_device() != device || sin->get_device() != device || shared(*x, *c.t) || shared(*positions, *c.t) || shared(*slots, *c.t) ||
      shared(*cos, *c.t) || shared(*sin, *c.t))
    Py_RETURN_NONE;
  const at::Tensor* w[2] = {nullptr, nullptr};
  for (int i = 0; i < 2; ++i)
    if (args[7 + i] != Py_None &&
        (!(w[i] = dense(args[7 + i], 1)) || !real(*w[i]) || w[i]->size(0) != d || w[i]->get_device() != device))
      Py_RETURN_NONE;
  if (w[0] && w[1] && w[0]->scalar_type() != w[1]->scalar_type()) Py_RETURN_NONE;
  if ((w[0] && shared(*w[0], *c.t)) || (w[1] && shared(*w[1], *c.t))) Py_RETURN_NONE;
  const double eps = PyFloat_AsDouble(args[9]);
  if (eps == -1.0 && PyErr_Occurred()) return nullptr;
  const int interleaved = PyObject_IsTrue(args[10]);
  if (interleaved < 0) return nullptr;
  const at::Tensor* weight = w[0] ? w[0] : w[1];
  const int64_t hq = heads - 2 * c.hkv;
  at::Tensor q;
  const cat_status st = unlocked([&] {
    q = make3(n, hq, d, at::kBFloat16);
    return cat_mx_rope_cache_write(x->data_ptr(), code(*x), n, hq, w[0] ? w[0]->data_ptr() : nullptr,
                                   w[1] ? w[1]->data_ptr() : nullptr, weight ? code(*weight) : CAT_F32, eps, i32(positions),
                                   static_cast<const float*>(cos->data_ptr()), static_cast<const float*>(sin->data_ptr()),
                                   cos->size(0), 2 * cos->size(1), interleaved, i32(slots), u8(*c.t), c.pages, c.page, c.hkv, d,
                                   q.data_ptr(), stream_of(*x));
  });
  return st == CAT_OK ? THPVariable_Wrap(q) : PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

// (q, cache, table, lens, scale, offsets, window, out_dtype)
PyObject* attention(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (!count(nargs, 8)) return nullptr;
  const at::Tensor *q = dense(args[0], 3), *table = dense(args[2], 2), *offsets = nullptr;
  if (!q || q->scalar_type() != at::kBFloat16 || !table || !current(*q)) Py_RETURN_NONE;
  const int64_t device = q->get_device(), n = q->size(0), hq = q->size(1), d = q->size(2), seqs = table->size(0);
  const Cache c(args[1], d);
  const at::Tensor* lens = numbers(args[3], seqs, device);
  at::ScalarType type = at::kBFloat16;
  int64_t window;
  if (!c.on(device) || !lens || table->scalar_type() != at::kInt || table->get_device() != device || !integer(args[6], &window) ||
      (args[5] != Py_None && !(offsets = numbers(args[5], seqs + 1, device))) || (args[7] != Py_None && !out_type(args[7], &type)))
    Py_RETURN_NONE;
  const double scale = PyFloat_AsDouble(args[4]);
  if (scale == -1.0 && PyErr_Occurred()) return nullptr;
  at::Tensor out, ws;
  const cat_status st = unlocked([&] {
    const int64_t need = cat_mx_attention_workspace(n, seqs, hq, c.hkv, d);
    out = make3(n, hq, d, type);
    if (need > 0) ws = bytes(1, need);
    return cat_mx_attention(q->data_ptr(), n, hq, u8(*c.t), c.pages, c.page, c.hkv, d, i32(table), table->size(1), i32(lens), seqs,
                            i32(offsets), (float)scale, window, code(out), out.data_ptr(), need > 0 ? ws.data_ptr() : nullptr,
                            need > 0 ? need : 0, stream_of(*q));
  });
  return st == CAT_OK ? THPVariable_Wrap(out) : PyLong_FromLong(st);
  END_HANDLE_TH_ERRORS
}

#define CAT_CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef calls[] = {CAT_CALL(quantize), CAT_CALL(swiglu_quantize), CAT_CALL(rmsnorm_quantize), CAT_CALL(dequantize),
                       CAT_CALL(linear), CAT_CALL(linear_grouped), CAT_CALL(cache_write), CAT_CALL(cache_read),
                       CAT_CALL(rope_cache_write), CAT_CALL(attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mx_calls", nullptr, -1, calls, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mx_calls(void) { return PyModule_Create(&module); }
