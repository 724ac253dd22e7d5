// Marshalling of the block-scaled layers' calls for Python: torch tensors in, torch tensors out, the C ABI of
// include/stamp.h in between.  The kernels of a decode step take one to ten microseconds; checking arguments, allocating
// outputs and converting them through ctypes takes ten.  Here the same takes about two.  Nothing is computed.
//
// Every function returns its outputs, or the stamp_status of the call as an int where it is not STAMP_OK (binding.py
// raises it); wrong shapes, types and places raise ValueError, and what torch throws becomes the Python exception it is.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdio>

#include "stamp.h"

namespace {

constexpr int64_t BLOCK = 128;   // features per scale
constexpr auto CODES = at::kFloat8_e4m3fn;
constexpr auto SCALE = at::kFloat8_e8m0fnu;

int64_t blocks(int64_t n) { return (n + BLOCK - 1) / BLOCK; }

// A Python exception is set: unwinds to the entry point.
struct Refused {};
[[noreturn]] void refuse(const char* text) {
  PyErr_SetString(PyExc_ValueError, text);
  throw Refused();
}

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (THPVariable_Check(o)) return THPVariable_Unpack(o);
  char text[80];
  snprintf(text, sizeof text, "%s: expected a tensor", what);
  refuse(text);
}

// A dense tensor of this shape and type on x's device.
void* dense(const at::Tensor& t, const char* what, at::IntArrayRef shape, at::ScalarType type, const at::Device& device) {
  if (t.scalar_type() != type || t.sizes() != shape || t.device() != device || !t.is_contiguous()) {
    std::string text = std::string(what) + ": expected a contiguous tensor of shape (";
    for (size_t i = 0; i < shape.size(); ++i) text += (i ? ", " : "") + std::to_string(shape[i]);
    text += std::string(") and type ") + c10::toString(type) + " on " + device.str() + ", got " + c10::toString(t.scalar_type()) + " of shape (";
    for (int64_t i = 0; i < t.dim(); ++i) text += (i ? ", " : "") + std::to_string(t.size(i));
    text += ") on " + t.device().str();
    refuse(text.c_str());
  }
  return t.data_ptr();
}

int dtype_code(at::ScalarType t) {
  if (t == at::kFloat) return STAMP_F32;
  if (t == at::kBFloat16) return STAMP_BF16;
  refuse("unsupported dtype: float32 and bfloat16 are taken");
}

int as_int(int64_t v) {
  if (v > INT32_MAX) refuse("a size does not fit 32 bits");
  return static_cast<int>(v);
}

// A matrix whose rows are dense; its rows may be any distance apart (a slice of columns of a wider one).
struct Rows {
  const at::Tensor& t;
  int64_t rows, features, ld;
};
Rows rows_of(PyObject* o) {
  const at::Tensor& t = tensor(o, "X");
  if (!t.is_cuda() || t.dim() != 2) refuse("X: expected a two-dimensional CUDA tensor");
  const int64_t rows = t.size(0), features = t.size(1);
  if (features > 1 && t.stride(1) != 1) refuse("X: expected dense rows");
  return Rows{t, rows, features, rows > 1 ? t.stride(0) : features};
}

// Output `o` if it is given (then it has to fit), else a new one.
at::Tensor output(PyObject* o, const char* what, at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) {
  if (o == Py_None) return at::empty(shape, like.options().dtype(type));
  const at::Tensor& t = tensor(o, what);
  dense(t, what, shape, type, like.device());
  return t;
}

PyObject* status_or(int status, const at::Tensor& a) { return status != STAMP_OK ? PyLong_FromLong(status) : THPVariable_Wrap(a); }
PyObject* status_or(int status, const at::Tensor& a, const at::Tensor& b) {
  if (status != STAMP_OK) return PyLong_FromLong(status);
  PyObject* pair = PyTuple_New(2);
  if (!pair) return nullptr;
  PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(a));
  PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(b));
  return pair;
}

void* stream_of(const at::Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.get_device()).stream(); }

void expect(Py_ssize_t got, Py_ssize_t want) {
  if (got != want) refuse("wrong number of arguments");
}

#define STAMP_ENTRY \
  HANDLE_TH_ERRORS  \
  try {
#define STAMP_ENTRY_END       \
  }                           \
  catch (const Refused&) {    \
    return nullptr;           \
  }                           \
  END_HANDLE_TH_ERRORS

// (X, rows | None, codes | None, scale | None) -> (codes, scale)
PyObject* fp8_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  STAMP_ENTRY
  expect(n, 4);
  const Rows x = rows_of(a[0]);
  const c10::cuda::CUDAGuard guard(x.t.device());
  int64_t M = x.rows;
  const void* rows = nullptr;
  if (a[1] != Py_None) {
    const at::Tensor& r = tensor(a[1], "rows");
    M = r.numel();
    rows = dense(r, "rows", {M}, at::kInt, x.t.device());
  }
  const int type = dtype_code(x.t.scalar_type());
  const at::Tensor codes = output(a[2], "codes", {M, x.features}, CODES, x.t);
  const at::Tensor scale = output(a[3], "scale", {M, blocks(x.features)}, SCALE, x.t);
  return status_or(stamp_fp8_quantize(x.t.data_ptr(), type, x.ld, static_cast<const int32_t*>(rows), as_int(x.rows), as_int(M),
                                      as_int(x.features), codes.data_ptr(), scale.data_ptr(), stream_of(x.t)),
                   codes, scale);
  STAMP_ENTRY_END
}

// (X, codes | None, scale | None) -> (codes, scale)
PyObject* fp8_gated_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  STAMP_ENTRY
  expect(n, 3);
  const Rows x = rows_of(a[0]);
  const c10::cuda::CUDAGuard guard(x.t.device());
  if (x.features % 2 != 0) refuse("X: expected as many gates as ups");
  const int64_t F = x.features / 2;
  const int type = dtype_code(x.t.scalar_type());
  const at::Tensor codes = output(a[1], "codes", {x.rows, F}, CODES, x.t);
  const at::Tensor scale = output(a[2], "scale", {x.rows, blocks(F)}, SCALE, x.t);
  return status_or(stamp_fp8_gated_quantize(x.t.data_ptr(), type, x.ld, as_int(x.rows), as_int(F), codes.data_ptr(), scale.data_ptr(),
                                            stream_of(x.t)),
                   codes, scale);
  STAMP_ENTRY_END
}

// The operands of a product, checked: x [M, K], x_scale, offsets [E + 1] (grouped), w [(E,) N, K], w_scale, bias [(E,) N].
PyObject* product(PyObject* const* a, bool grouped) {
  PyObject* const* const rest = a + (grouped ? 3 : 2);   // w, w_scale, bias | None, out_dtype, out | None
  const at::Tensor &x = tensor(a[0], "x"), &x_scale = tensor(a[1], "x_scale"), &w = tensor(rest[0], "w"), &w_scale = tensor(rest[1], "w_scale");
  if (!x.is_cuda() || x.dim() != 2) refuse("x: expected a two-dimensional CUDA tensor");
  if (w.dim() != (grouped ? 3 : 2)) refuse(grouped ? "w: expected a matrix for each expert" : "w: expected a matrix");
  const at::Device device = x.device();
  const c10::cuda::CUDAGuard guard(device);
  const int64_t M = x.size(0), K = x.size(1), N = w.size(-2), E = grouped ? w.size(0) : 1;
  const int64_t w_shape[3] = {E, N, K}, s_shape[3] = {E, blocks(N), blocks(K)}, b_shape[2] = {E, N};
  const size_t skip = grouped ? 0 : 1;
  const void* xp = dense(x, "x", {M, K}, CODES, device);
  const void* xs = dense(x_scale, "x_scale", {M, blocks(K)}, SCALE, device);
  const void* offsets = grouped ? dense(tensor(a[2], "offsets"), "offsets", {E + 1}, at::kInt, device) : nullptr;
  const void* wp = dense(w, "w", at::IntArrayRef(w_shape + skip, 3 - skip), CODES, device);
  const void* ws = dense(w_scale, "w_scale", at::IntArrayRef(s_shape + skip, 3 - skip), SCALE, device);
  const void* bias = rest[2] == Py_None ? nullptr : dense(tensor(rest[2], "bias"), "bias", at::IntArrayRef(b_shape + skip, 2 - skip), at::kFloat, device);
  at::ScalarType type;
  if (rest[4] != Py_None) {
    type = tensor(rest[4], "out").scalar_type();
  } else {
    if (!THPDtype_Check(rest[3])) refuse("out_dtype: expected a torch.dtype");
    type = reinterpret_cast<THPDtype*>(rest[3])->scalar_type;
  }
  const int code = dtype_code(type);
  const at::Tensor y = output(rest[4], "out", {M, N}, type, x);
  const int status =
      grouped ? stamp_fp8_linear_grouped(xp, xs, static_cast<const int32_t*>(offsets), wp, ws, static_cast<const float*>(bias), as_int(M),
                                         as_int(E), as_int(N), as_int(K), y.data_ptr(), code, stream_of(x))
              : stamp_fp8_linear(xp, xs, wp, ws, static_cast<const float*>(bias), as_int(M), as_int(N), as_int(K), y.data_ptr(), code,
                                 stream_of(x));
  return status_or(status, y);
}

// (x, x_scale, w, w_scale, bias | None, out_dtype, out | None) -> out
PyObject* fp8_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  STAMP_ENTRY
  expect(n, 7);
  return product(a, false);
  STAMP_ENTRY_END
}

// (x, x_scale, offsets, w, w_scale, bias | None, out_dtype, out | None) -> out
PyObject* fp8_linear_grouped(PyObject*, PyObject* const* a, Py_ssize_t n) {
  STAMP_ENTRY
  expect(n, 8);
  return product(a, true);
  STAMP_ENTRY_END
}

#define STAMP_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {STAMP_METHOD(fp8_quantize), STAMP_METHOD(fp8_gated_quantize), STAMP_METHOD(fp8_linear),
                         STAMP_METHOD(fp8_linear_grouped), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls() { return PyModule_Create(&module); }
