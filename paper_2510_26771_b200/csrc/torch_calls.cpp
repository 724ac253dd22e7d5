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

// One matrix and its operands, checked.
struct Product {
  const at::Tensor& x;
  const void *xp, *xs, *wp, *ws;
  const float* bias;
  int64_t M, N, K;
};
Product product_of(PyObject* const* a) {   // x, x_scale, w, w_scale, bias | None
  const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[2], "w");
  if (!x.is_cuda() || x.dim() != 2) refuse("x: expected a two-dimensional CUDA tensor");
  if (w.dim() != 2) refuse("w: expected a matrix");
  const at::Device device = x.device();
  const int64_t M = x.size(0), K = x.size(1), N = w.size(0);
  return Product{x,
                 dense(x, "x", {M, K}, CODES, device),
                 dense(tensor(a[1], "x_scale"), "x_scale", {M, blocks(K)}, SCALE, device),
                 dense(w, "w", {N, K}, CODES, device),
                 dense(tensor(a[3], "w_scale"), "w_scale", {blocks(N), blocks(K)}, SCALE, device),
                 a[4] == Py_None ? nullptr : static_cast<const float*>(dense(tensor(a[4], "bias"), "bias", {N}, at::kFloat, device)),
                 M, N, K};
}

int as_int(PyObject* o, const char* what) {
  const long v = PyLong_Check(o) ? PyLong_AsLong(o) : -1;
  if (v < 0 || v > INT32_MAX) {
    PyErr_Clear();
    char text[80];
    snprintf(text, sizeof text, "%s: expected a small non-negative number", what);
    refuse(text);
  }
  return static_cast<int>(v);
}

// A residual [rows, features]: dense rows any distance apart.
struct Residual {
  const void* p = nullptr;
  int type = STAMP_F32;
  int64_t ld = 0;
};
Residual residual_of(PyObject* o, int64_t rows, int64_t features, const at::Device& device) {
  Residual r;
  if (o == Py_None) return r;
  const at::Tensor& t = tensor(o, "residual");
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != features || t.device() != device) refuse("residual: expected the output's shape and device");
  if (features > 1 && t.stride(1) != 1) refuse("residual: expected dense rows");
  if (rows > 1 && t.stride(0) < features) refuse("residual: expected rows that do not overlap");
  r.p = t.data_ptr();
  r.type = dtype_code(t.scalar_type());
  r.ld = rows > 1 ? t.stride(0) : features;
  return r;
}

at::ScalarType out_type(PyObject* dtype, PyObject* out) {
  if (out != Py_None) return tensor(out, "out").scalar_type();
  if (!THPDtype_Check(dtype)) refuse("out_dtype: expected a torch.dtype");
  return reinterpret_cast<THPDtype*>(dtype)->scalar_type;
}

// (x, x_scale, w, w_scale, bias | None, activation, residual | None, out_dtype, out | None) -> out
PyObject* fp8_linear_fused(PyObject*, PyObject* const* a, Py_ssize_t n) {
  STAMP_ENTRY
  expect(n, 9);
  const Product p = product_of(a);
  const c10::cuda::CUDAGuard guard(p.x.device());
  const int act = as_int(a[5], "activation");
  const Residual r = residual_of(a[6], p.M, p.N, p.x.device());
  const at::ScalarType type = out_type(a[7], a[8]);
  const int code = dtype_code(type);
  const at::Tensor y = output(a[8], "out", {p.M, p.N}, type, p.x);
  return status_or(stamp_fp8_linear_fused(p.xp, p.xs, p.wp, p.ws, p.bias, act, r.p, r.type, r.ld, as_int(p.M), as_int(p.N), as_int(p.K),
                                          y.data_ptr(), code, stream_of(p.x)),
                   y);
  STAMP_ENTRY_END
}

// (x, x_scale, w, w_scale, bias | None, activation, codes | None, scale | None) -> (codes, scale)
PyObject* fp8_linear_quantized(PyObject*, PyObject* const* a, Py_ssize_t n) {
  STAMP_ENTRY
  expect(n, 8);
  const Product p = product_of(a);
  const c10::cuda::CUDAGuard guard(p.x.device());
  const int act = as_int(a[5], "activation");
  const at::Tensor codes = output(a[6], "codes", {p.M, p.N}, CODES, p.x);
  const at::Tensor scale = output(a[7], "scale", {p.M, blocks(p.N)}, SCALE, p.x);
  return status_or(stamp_fp8_linear_quantized(p.xp, p.xs, p.wp, p.ws, p.bias, act, as_int(p.M), as_int(p.N), as_int(p.K), codes.data_ptr(),
                                              scale.data_ptr(), stream_of(p.x)),
                   codes, scale);
  STAMP_ENTRY_END
}

// Scratch of at least `bytes`: `o` if it is given, else new memory of x's device (ordered, like the outputs, by its stream).
at::Tensor scratch(PyObject* o, size_t bytes, const at::Tensor& x) {
  if (o == Py_None) return at::empty({static_cast<int64_t>(bytes)}, x.options().dtype(at::kByte));
  const at::Tensor& t = tensor(o, "ws");
  if (t.device() != x.device() || !t.is_contiguous()) refuse("ws: expected a contiguous tensor on the inputs' device");
  return t;
}

// A contiguous tensor of this shape and type (four bytes wide) in `room`'s memory, `first` words in.
at::Tensor part_of(const at::Tensor& room, int64_t first, at::IntArrayRef shape, at::ScalarType type) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(room.storage()), room.key_set(), c10::scalarTypeToTypeMeta(type));
  t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
  t.unsafeGetTensorImpl()->set_storage_offset(first);
  return t;
}

// (logits, top, normalize, out | None) -> (chosen, share, rows, place, offsets, row_share)
PyObject* expert_route(PyObject*, PyObject* const* a, Py_ssize_t n) {
  STAMP_ENTRY
  expect(n, 4);
  const Rows l = rows_of(a[0]);
  const c10::cuda::CUDAGuard guard(l.t.device());
  const int64_t T = l.rows, E = l.features;
  const int top = as_int(a[1], "top"), type = dtype_code(l.t.scalar_type());
  PyObject* given[6] = {Py_None, Py_None, Py_None, Py_None, Py_None, Py_None};
  if (a[3] != Py_None) {
    if (!PyTuple_Check(a[3]) || PyTuple_GET_SIZE(a[3]) != 6) refuse("out: expected a tuple of six tensors");
    for (int i = 0; i < 6; ++i) given[i] = PyTuple_GET_ITEM(a[3], i);
  }
  size_t bytes = 0;
  if (const int rc = stamp_expert_route_workspace_bytes(as_int(T), as_int(E), top, &bytes)) return PyLong_FromLong(rc);
  // Six buffers of one allocation, with room for the counts: allocating each would take longer than the kernels do.
  const int64_t rows = T * top, sizes[6] = {rows, rows, rows, rows, E + 1, rows};
  const int64_t two[2] = {T, top}, one[1] = {rows}, ends[1] = {E + 1};
  const at::IntArrayRef shapes[6] = {two, two, one, two, ends, one};
  constexpr at::ScalarType types[6] = {at::kInt, at::kFloat, at::kInt, at::kInt, at::kInt, at::kFloat};
  constexpr const char* names[6] = {"chosen", "share", "rows", "place", "offsets", "row_share"};
  at::Tensor t[6], room;
  if (a[3] == Py_None) {
    int64_t at = 0, words = 0;
    for (int64_t s : sizes) words += (s + 63) / 64 * 64;
    room = at::empty({words}, l.t.options().dtype(at::kInt));
    for (int i = 0; i < 6; ++i) {
      t[i] = part_of(room, at, shapes[i], types[i]);
      at += (sizes[i] + 63) / 64 * 64;
    }
  } else {
    for (int i = 0; i < 6; ++i) t[i] = output(given[i], names[i], shapes[i], types[i], l.t);
  }
  at::Tensor ws;
  if (bytes > 0) ws = scratch(Py_None, bytes, l.t);
  const int status = stamp_expert_route(l.t.data_ptr(), type, l.ld, as_int(T), as_int(E), top, a[2] == Py_True, static_cast<int32_t*>(t[0].data_ptr()),
                                        static_cast<float*>(t[1].data_ptr()), static_cast<int32_t*>(t[2].data_ptr()),
                                        static_cast<int32_t*>(t[3].data_ptr()), static_cast<int32_t*>(t[4].data_ptr()),
                                        static_cast<float*>(t[5].data_ptr()), bytes > 0 ? ws.data_ptr() : nullptr, bytes, stream_of(l.t));
  if (status != STAMP_OK) return PyLong_FromLong(status);
  PyObject* all = PyTuple_New(6);
  if (!all) return nullptr;
  for (int i = 0; i < 6; ++i) PyTuple_SET_ITEM(all, i, THPVariable_Wrap(t[i]));
  return all;
  STAMP_ENTRY_END
}

// (y, place, share, residual | None, out_dtype, out | None) -> out
PyObject* expert_combine(PyObject*, PyObject* const* a, Py_ssize_t n) {
  STAMP_ENTRY
  expect(n, 6);
  const at::Tensor &y = tensor(a[0], "y"), &place = tensor(a[1], "place"), &share = tensor(a[2], "share");
  if (!y.is_cuda() || y.dim() != 2 || !y.is_contiguous()) refuse("y: expected a contiguous two-dimensional CUDA tensor");
  if (place.dim() != 2) refuse("place: expected a matrix");
  const c10::cuda::CUDAGuard guard(y.device());
  const int64_t M = y.size(0), N = y.size(1), T = place.size(0), top = place.size(1);
  const void* pp = dense(place, "place", {T, top}, at::kInt, y.device());
  const void* sp = dense(share, "share", {T, top}, at::kFloat, y.device());
  const Residual r = residual_of(a[3], T, N, y.device());
  const at::ScalarType type = out_type(a[4], a[5]);
  const int code = dtype_code(type), y_code = dtype_code(y.scalar_type());
  const at::Tensor out = output(a[5], "out", {T, N}, type, y);
  return status_or(stamp_expert_combine(y.data_ptr(), y_code, static_cast<const int32_t*>(pp), static_cast<const float*>(sp), r.p, r.type, r.ld,
                                        as_int(T), as_int(top), as_int(M), as_int(N), out.data_ptr(), code, stream_of(y)),
                   out);
  STAMP_ENTRY_END
}

// (x, rows, share, offsets, up, up_scale, up_bias | None, down, down_scale, down_bias | None, residual | None, out_dtype, out | None,
//  ws | None) -> out
PyObject* fp8_expert_layer(PyObject*, PyObject* const* a, Py_ssize_t n) {
  STAMP_ENTRY
  expect(n, 14);
  const Rows x = rows_of(a[0]);
  const at::Device device = x.t.device();
  const c10::cuda::CUDAGuard guard(device);
  const at::Tensor &rows = tensor(a[1], "rows"), &up = tensor(a[4], "up"), &down = tensor(a[7], "down");
  if (up.dim() != 3 || down.dim() != 3) refuse("up, down: expected a matrix for each expert");
  const int64_t T = x.rows, K = x.features, M = rows.numel(), E = up.size(0), F = down.size(2), N = down.size(1);
  const void* rp = dense(rows, "rows", {M}, at::kInt, device);
  const void* sp = dense(tensor(a[2], "row_share"), "row_share", {M}, at::kFloat, device);
  const void* op = dense(tensor(a[3], "offsets"), "offsets", {E + 1}, at::kInt, device);
  const void* wu = dense(up, "up", {E, 2 * F, K}, CODES, device);
  const void* su = dense(tensor(a[5], "up_scale"), "up_scale", {E, blocks(2 * F), blocks(K)}, SCALE, device);
  const void* bu = a[6] == Py_None ? nullptr : dense(tensor(a[6], "up_bias"), "up_bias", {E, 2 * F}, at::kFloat, device);
  const void* wd = dense(down, "down", {E, N, F}, CODES, device);
  const void* sd = dense(tensor(a[8], "down_scale"), "down_scale", {E, blocks(N), blocks(F)}, SCALE, device);
  const void* bd = a[9] == Py_None ? nullptr : dense(tensor(a[9], "down_bias"), "down_bias", {E, N}, at::kFloat, device);
  const Residual r = residual_of(a[10], T, N, device);
  const at::ScalarType type = out_type(a[11], a[12]);
  const int code = dtype_code(type), x_code = dtype_code(x.t.scalar_type());
  size_t bytes = 0;
  if (const int rc = stamp_fp8_expert_workspace_bytes(as_int(M), as_int(F), &bytes)) return PyLong_FromLong(rc);
  const at::Tensor y = output(a[12], "out", {T, N}, type, x.t);
  const at::Tensor ws = scratch(a[13], bytes, x.t);
  return status_or(stamp_fp8_expert_layer(x.t.data_ptr(), x_code, x.ld, static_cast<const int32_t*>(rp), static_cast<const float*>(sp),
                                          static_cast<const int32_t*>(op), wu, su, static_cast<const float*>(bu), wd, sd,
                                          static_cast<const float*>(bd), r.p, r.type, r.ld, as_int(T), as_int(M), as_int(E), as_int(K), as_int(F),
                                          as_int(N), y.data_ptr(), code, ws.data_ptr(), static_cast<size_t>(ws.numel() * ws.element_size()),
                                          stream_of(x.t)),
                   y);
  STAMP_ENTRY_END
}

#define STAMP_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {STAMP_METHOD(fp8_quantize), STAMP_METHOD(fp8_gated_quantize), STAMP_METHOD(fp8_linear),
                         STAMP_METHOD(fp8_linear_grouped), STAMP_METHOD(fp8_linear_fused), STAMP_METHOD(fp8_linear_quantized),
                         STAMP_METHOD(expert_route), STAMP_METHOD(expert_combine), STAMP_METHOD(fp8_expert_layer), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls() { return PyModule_Create(&module); }
