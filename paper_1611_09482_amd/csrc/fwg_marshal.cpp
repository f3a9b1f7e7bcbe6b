// Argument marshalling of ops.py for the calls whose time the host decides: the module _marshal.
//
// A call of 4-bit rows or adjusted logits for few streams takes the device 3 to 7 us and took the host 7 to 9, of which 4 to 5
// were the checks of ops.py, tensor by tensor.  Here the same checks read the tensors directly.  Only the plain case is taken:
// torch.Tensor objects, dense and contiguous, on the current device, of the types and shapes that belong together.
// Everything else is declined (None), and ops.py goes through its own checks, which take more layouts and say what is
// wrong.  No device work happens here but what the C entries of fwg.h enqueue.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include "fwg.h"

namespace {

struct Entries {
  decltype(&fwg_quant_mx) quant;
  decltype(&fwg_norm_mx) norm;
  decltype(&fwg_matmul_mx_workspace) matmul_workspace;
  decltype(&fwg_matmul_mx) matmul;
  decltype(&fwg_adjust_logits) adjust;
} entries;

constexpr int64_t kMost = INT32_MAX;

// The tensor behind an argument, or NULL where it is not a plain one on the device.
const at::Tensor *plain(PyObject *o, int64_t device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor &t = THPVariable_Unpack(o);
  if (t.layout() != c10::kStrided || !t.is_cuda() || t.get_device() != device || !t.is_contiguous()) return nullptr;
  return &t;
}

bool same_lead(const at::Tensor &a, const at::Tensor &b, int64_t last) {
  const auto x = a.sizes(), y = b.sizes();
  return x.size() == y.size() && y.back() == last && std::equal(x.begin(), x.end() - 1, y.begin());
}

// One call's arguments, taken from `at` on; `fits` stays true while they are what the call wants.
struct Taker {
  int64_t device;
  bool fits = true;
  // Rows of float32 or bfloat16.
  const at::Tensor *rows(PyObject *o, int *kind) {
    const at::Tensor *t = plain(o, device);
    if (!t || t->dim() < 1 || t->sizes().back() < 1 || t->sizes().back() > kMost) return no();
    if (t->scalar_type() == at::kFloat) *kind = FWG_F32;
    else if (t->scalar_type() == at::kBFloat16) *kind = FWG_BF16;
    else return no();
    return t;
  }
  // Rows of a type, as many as another tensor's and so wide; None gives NULL where it may.
  void *like(PyObject *o, at::ScalarType type, const at::Tensor *other, int64_t width, bool optional = false) {
    if (optional && o == Py_None) return nullptr;
    const at::Tensor *t = fits ? plain(o, device) : nullptr;
    if (!t || t->scalar_type() != type || !same_lead(*other, *t, width)) return no(), nullptr;
    return t->data_ptr();
  }
  void *vector(PyObject *o, at::ScalarType type, int64_t n, bool optional = false) {
    if (optional && o == Py_None) return nullptr;
    const at::Tensor *t = fits ? plain(o, device) : nullptr;
    if (!t || t->scalar_type() != type || t->numel() != n) return no(), nullptr;
    return t->data_ptr();
  }
  // One row for all (stride 0), or a row for each.
  void *one_or_each(PyObject *o, at::ScalarType type, const at::Tensor *other, int64_t width, int64_t *stride) {
    *stride = 0;
    if (o == Py_None) return nullptr;
    const at::Tensor *t = fits ? plain(o, device) : nullptr;
    if (!t || t->scalar_type() != type) return no(), nullptr;
    if (t->dim() == 1) {
      if (t->numel() != width) return no(), nullptr;
      return t->data_ptr();
    }
    if (!same_lead(*other, *t, width)) return no(), nullptr;
    *stride = width;
    return t->data_ptr();
  }
  const at::Tensor *no() {
    fits = false;
    return nullptr;
  }
};

template <typename F> PyObject *enqueue(F call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

bool begin(PyObject *const *a, Py_ssize_t have, Py_ssize_t want, Taker *take, void **stream) {
  if (have != want) return false;
  take->device = PyLong_AsLongLong(a[0]);
  *stream = PyLong_AsVoidPtr(a[1]);
  if (!PyErr_Occurred()) return true;
  PyErr_Clear();
  return false;
}

// (device, stream, x, q, scale, values)
PyObject *quant_mx(PyObject *, PyObject *const *a, Py_ssize_t n) try {
  Taker take;
  void *stream;
  int kind;
  if (!begin(a, n, 6, &take, &stream)) Py_RETURN_NONE;
  const at::Tensor *x = take.rows(a[2], &kind);
  if (!x) Py_RETURN_NONE;
  const int64_t width = x->sizes().back(), rows = x->numel() / width, blocks = (width + 31) / 32;
  auto *q = (uint8_t *)take.like(a[3], at::kByte, x, 16 * blocks), *scale = (uint8_t *)take.like(a[4], at::kByte, x, blocks);
  auto *values = (uint16_t *)take.like(a[5], at::kBFloat16, x, width, true);
  if (!take.fits) Py_RETURN_NONE;
  const void *xp = x->data_ptr();
  return enqueue([&] {
    return entries.quant(kind, rows, (int32_t)width, xp, width, q, 16 * blocks, scale, blocks, values, width, stream);
  });
} catch (...) {
  Py_RETURN_NONE;
}

// (device, stream, x, gain, residual, eps, q, scale, row_scale, summed, values)
PyObject *norm_mx(PyObject *, PyObject *const *a, Py_ssize_t n) try {
  Taker take;
  void *stream;
  int kind;
  if (!begin(a, n, 11, &take, &stream) || !PyFloat_CheckExact(a[5])) Py_RETURN_NONE;
  const at::Tensor *x = take.rows(a[2], &kind);
  if (!x) Py_RETURN_NONE;
  const int64_t width = x->sizes().back(), rows = x->numel() / width, blocks = (width + 31) / 32;
  const at::ScalarType type = x->scalar_type();
  auto *gain = (const float *)take.vector(a[3], at::kFloat, width, true);
  const void *residual = take.like(a[4], type, x, width, true);
  auto *q = (uint8_t *)take.like(a[6], at::kByte, x, 16 * blocks), *scale = (uint8_t *)take.like(a[7], at::kByte, x, blocks);
  auto *row_scale = (float *)take.vector(a[8], at::kFloat, rows);
  void *summed = take.like(a[9], type, x, width, true);
  auto *values = (uint16_t *)take.like(a[10], at::kBFloat16, x, width, true);
  if (!take.fits) Py_RETURN_NONE;
  const float eps = (float)PyFloat_AS_DOUBLE(a[5]);
  const void *xp = x->data_ptr();
  return enqueue([&] {
    return entries.norm(kind, rows, (int32_t)width, xp, width, residual, width, gain, eps, summed, width, q, 16 * blocks, scale,
                        blocks, row_scale, values, width, stream);
  });
} catch (...) {
  Py_RETURN_NONE;
}

// (device, stream, x, x_scale, w, w_scale, row_scale, bias, out)
PyObject *matmul_mx(PyObject *, PyObject *const *a, Py_ssize_t n) try {
  Taker take;
  void *stream;
  int kind;
  if (!begin(a, n, 9, &take, &stream)) Py_RETURN_NONE;
  const at::Tensor *x = plain(a[2], take.device), *w = plain(a[4], take.device), *out = take.rows(a[8], &kind);
  if (!x || !w || !out || x->scalar_type() != at::kByte || w->scalar_type() != at::kByte || x->dim() < 1 || w->dim() != 2) Py_RETURN_NONE;
  const int64_t bytes = x->sizes().back(), outputs = w->size(0), blocks = bytes / 16;
  if (bytes < 16 || bytes > kMost || bytes % 16 || w->size(1) != bytes || outputs > kMost || !same_lead(*x, *out, outputs)) Py_RETURN_NONE;
  const int64_t rows = x->numel() / bytes;
  auto *xs = (const uint8_t *)take.like(a[3], at::kByte, x, blocks), *ws = (const uint8_t *)take.like(a[5], at::kByte, w, blocks);
  auto *row_scale = (const float *)take.vector(a[6], at::kFloat, rows, true);
  auto *bias = (const float *)take.vector(a[7], at::kFloat, outputs, true);
  size_t need = 0;
  if (!take.fits || entries.matmul_workspace(rows, (int32_t)outputs, (int32_t)blocks, &need) != FWG_OK) Py_RETURN_NONE;
  at::Tensor workspace;  // torch's allocator keeps it for this stream, as ops.py's
  if (need) workspace = at::empty({(int64_t)need}, x->options());
  void *const space = need ? workspace.data_ptr() : nullptr;
  auto *xp = (const uint8_t *)x->data_ptr(), *wp = (const uint8_t *)w->data_ptr();
  void *op = out->data_ptr();
  return enqueue([&] {
    return entries.matmul(kind, rows, (int32_t)outputs, (int32_t)blocks, xp, bytes, xs, blocks, wp, bytes, ws, blocks, row_scale,
                          bias, op, outputs, space, need, stream);
  });
} catch (...) {
  Py_RETURN_NONE;
}

// (device, stream, logits, tokens, lengths, prompts, repetition, presence, frequency, bias, allowed, out)
PyObject *adjust_logits(PyObject *, PyObject *const *a, Py_ssize_t n) try {
  Taker take;
  void *stream;
  int kind;
  if (!begin(a, n, 12, &take, &stream)) Py_RETURN_NONE;
  const at::Tensor *z = take.rows(a[2], &kind);
  if (!z) Py_RETURN_NONE;
  const int64_t vocab = z->sizes().back(), rows = z->numel() / vocab;
  int64_t history = 0, bias_stride, allowed_stride;
  const int32_t *tokens = nullptr;
  if (a[3] == Py_None) {
    for (int i = 4; i < 9; ++i)
      if (a[i] != Py_None) Py_RETURN_NONE;
  } else {
    const at::Tensor *t = plain(a[3], take.device);
    if (!t || t->scalar_type() != at::kInt || t->dim() < 1 || t->sizes().back() > kMost) Py_RETURN_NONE;
    history = t->sizes().back();
    if (!same_lead(*z, *t, history)) Py_RETURN_NONE;
    tokens = (const int32_t *)t->data_ptr();
  }
  auto *lengths = (const int32_t *)take.vector(a[4], at::kInt, rows, true);
  auto *prompts = (const int32_t *)take.vector(a[5], at::kInt, rows, true);
  auto *repetition = (const float *)take.vector(a[6], at::kFloat, rows, true);
  auto *presence = (const float *)take.vector(a[7], at::kFloat, rows, true);
  auto *frequency = (const float *)take.vector(a[8], at::kFloat, rows, true);
  auto *bias = (const float *)take.one_or_each(a[9], at::kFloat, z, vocab, &bias_stride);
  auto *allowed = (const uint32_t *)take.one_or_each(a[10], at::kInt, z, (vocab + 31) / 32, &allowed_stride);
  void *out = take.like(a[11], z->scalar_type(), z, vocab);
  if (!take.fits) Py_RETURN_NONE;
  const void *zp = z->data_ptr();
  return enqueue([&] {
    return entries.adjust(kind, rows, (int32_t)vocab, zp, vocab, (int32_t)history, tokens, history, lengths, prompts, repetition,
                          presence, frequency, bias, bias_stride, allowed, allowed_stride, out, vocab, stream);
  });
} catch (...) {
  Py_RETURN_NONE;
}

// The addresses of the entries, in the order of Entries.
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
  void *at[5];
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "five addresses are wanted");
    return nullptr;
  }
  for (int i = 0; i < 5; ++i) {
    at[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  entries = {(decltype(entries.quant))at[0], (decltype(entries.norm))at[1], (decltype(entries.matmul_workspace))at[2],
             (decltype(entries.matmul))at[3], (decltype(entries.adjust))at[4]};
  Py_RETURN_NONE;
}

#define ENTRY(name) {#name, (PyCFunction)(void *)name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(bind), ENTRY(quant_mx), ENTRY(norm_mx), ENTRY(matmul_mx), ENTRY(adjust_logits),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef definition = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&definition); }
