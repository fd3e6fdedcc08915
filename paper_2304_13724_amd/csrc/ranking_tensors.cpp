// The ranking calls of include/bgmf.h on PyTorch tensors: a CPython module
// (paper_2304_13724_amd._ranking) that checks the tensors, allocates results
// and workspaces with PyTorch, and calls the library.  In Python these steps
// took longer than the smallest calls' kernels (a log_probs call 13 us, a
// clip of 211 gradients 140 us), which is why they are here; ranking.py has
// the documentation and the rest of the interface.
//
// A call that the library refuses returns its status code (an int) in place of
// tensors; arguments that do not fit raise ValueError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/util/Exception.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/forward_grad.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <cstdio>
#include <new>
#include <optional>
#include <stdexcept>
#include <string>
#include <vector>

#include "../../include/bgmf.h"

namespace {

struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};
// What the library refused, with its message.
struct Failed : std::runtime_error {
  int code;
  explicit Failed(int rc) : std::runtime_error(bgmf_last_error(nullptr)), code(rc) {}
};
void check(int rc) {
  if (rc != BGMF_OK) throw Failed(rc);
}

[[noreturn]] void refuse(const char *fmt, ...) __attribute__((format(printf, 1, 2)));
void refuse(const char *fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  throw Refused(buf);
}

constexpr unsigned kFloats =
    1u << BGMF_TYPE_F32 | 1u << BGMF_TYPE_BF16 | 1u << BGMF_TYPE_F16;
constexpr unsigned kBytes = 1u << BGMF_TYPE_I8;

int type_of(const at::Tensor &t) {
  switch (t.scalar_type()) {
    case at::kFloat: return BGMF_TYPE_F32;
    case at::kBFloat16: return BGMF_TYPE_BF16;
    case at::kHalf: return BGMF_TYPE_F16;
    case at::kChar: return BGMF_TYPE_I8;
    default: return -1;
  }
}

at::ScalarType dtype_of(int type) {
  return type == BGMF_TYPE_F32 ? at::kFloat : type == BGMF_TYPE_BF16 ? at::kBFloat16 : at::kHalf;
}

// Whether forward-mode derivatives are being computed: tensors have tangents at
// no other time, and looking for one takes 10 ns a tensor.
thread_local bool t_forward_mode = false;

// The tensor behind a Python object, which keeps it alive during the call.  No
// call has a forward-mode derivative, and none drops a tangent silently.
const at::Tensor &tensor(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) refuse("%s must be a tensor", name);
  const at::Tensor &t = THPVariable_Unpack(o);
  if (t_forward_mode && t._fw_grad(0).defined())
    refuse("%s has a tangent: forward-mode derivatives are not supported", name);
  if (t.is_neg() || t._is_zerotensor())
    refuse("%s: its memory does not hold its values (call .resolve_neg() or .clone())", name);
  return t;
}

// A 2-D tensor on the GPU of one of the types, the elements of a row adjacent.
const at::Tensor &matrix(PyObject *o, const char *name, unsigned types, int *type) {
  const at::Tensor &t = tensor(o, name);
  if (t.dim() != 2) refuse("%s must be a 2-D tensor", name);
  *type = type_of(t);
  if (*type < 0 || !(types >> *type & 1))
    refuse("%s must be %s%s%s, not %s", name, types & kFloats ? "float32, bfloat16 or float16" : "",
           types == (kFloats | kBytes) ? " or " : "", types & kBytes ? "int8" : "",
           c10::toString(t.scalar_type()));
  if (!t.is_cuda()) refuse("%s must be on the GPU", name);
  if (t.size(1) > 1 && t.stride(1) != 1)
    refuse("%s: the elements of a row must be adjacent (call .contiguous())", name);
  return t;
}

// A contiguous vector on the device of `like`; null for None.
const void *vector(PyObject *o, const char *name, const at::Tensor &like, int64_t count,
                   at::ScalarType dtype, bool optional) {
  if (optional && o == Py_None) return nullptr;
  const at::Tensor &t = tensor(o, name);
  if (t.dim() != 1 || t.size(0) != count)
    refuse("%s must be a 1-D tensor of length %lld", name, (long long)count);
  if (t.scalar_type() != dtype || t.device() != like.device())
    refuse("%s must be %s on the same GPU", name, c10::toString(dtype));
  if (count > 1 && t.stride(0) != 1) refuse("%s must be contiguous", name);
  return t.const_data_ptr();
}

const uint8_t *excluded_items(PyObject *o, const at::Tensor &scores, int64_t *stride) {
  *stride = 0;
  if (o == Py_None) return nullptr;
  const at::Tensor &t = tensor(o, "excluded");
  if (t.scalar_type() != at::kBool && t.scalar_type() != at::kByte)
    refuse("excluded must be a bool or uint8 tensor");
  if (t.sizes() != scores.sizes() || t.device() != scores.device())
    refuse("excluded must have the shape and the device of the scores");
  if (t.size(1) > 1 && t.stride(1) != 1)
    refuse("excluded: the elements of a row must be adjacent (call .contiguous())");
  *stride = t.stride(0);
  return static_cast<const uint8_t *>(t.const_data_ptr());
}

at::Tensor make(at::IntArrayRef sizes, const at::Tensor &like, at::ScalarType dtype) {
  return at::empty(sizes, like.options().dtype(dtype).layout(at::kStrided).requires_grad(false));
}

// Whether autograd records what is done with a tensor.
bool in_graph(const at::Tensor &t) {
  return at::GradMode::is_enabled() && t.defined() && t.requires_grad();
}
// What a call writes into has no derivative: a tensor with a history would keep one
// that is no longer its own.
void not_in_graph(const at::Tensor &t, const char *name) {
  if (in_graph(t)) refuse("%s takes no part in a graph, and it requires grad", name);
}

// An output given by the caller, or a new one for None.  `part`: a tensor of the call
// that may be the output though it is part of a graph.
at::Tensor output(PyObject *o, const char *name, const at::Tensor &like, int64_t rows,
                  int64_t cols, at::ScalarType dtype, PyObject *part = nullptr) {
  if (o == Py_None) return make({rows, cols}, like, dtype);
  const at::Tensor &t = tensor(o, name);
  if (o != part) not_in_graph(t, name);
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols || t.scalar_type() != dtype ||
      t.device() != like.device())
    refuse("%s must be %s of shape (%lld, %lld) on the same GPU", name, c10::toString(dtype),
           (long long)rows, (long long)cols);
  if ((cols > 1 && t.stride(1) != 1) || (rows > 1 && t.stride(0) < cols))
    refuse("%s: rows must not overlap and their elements must be adjacent", name);
  return t;
}

// A tensor of the caller's has been written: graphs that hold it from before
// notice at their backward pass, as after PyTorch's in-place functions.
void written(const at::Tensor &t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void written(PyObject *o, const at::Tensor &t) {
  if (o != Py_None) written(t);
}

double number(PyObject *o, const char *name) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    refuse("%s must be a number", name);
  }
  return v;
}
int64_t integer(PyObject *o, const char *name) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    refuse("%s must be an integer", name);
  }
  return v;
}
void *stream_of(PyObject *o) { return reinterpret_cast<void *>(integer(o, "stream")); }

template <class T>
T *at_(const at::Tensor &t) {
  return static_cast<T *>(t.mutable_data_ptr());
}

// (scores, given, top, temperature, excluded, stream) -> (log_prob, entropy,
// top_item, top_log_prob, row_max, row_sum)
PyObject *log_probs(PyObject *const *a) {
  int type;
  const at::Tensor &x = matrix(a[0], "scores", kFloats, &type);
  const int64_t rows = x.size(0), cols = x.size(1), top = integer(a[2], "top");
  const void *given = vector(a[1], "given", x, rows, at::kInt, true);
  if (top < 0 || top > BGMF_TOP_MAX) refuse("top must be in [0, %d]", BGMF_TOP_MAX);
  int64_t ex_stride;
  const uint8_t *ex = excluded_items(a[4], x, &ex_stride);
  const c10::DeviceGuard guard(x.device());
  const int64_t ws_bytes = bgmf_log_probs_workspace(rows, cols, (int32_t)top);
  at::Tensor ws;
  if (ws_bytes) ws = make({ws_bytes}, x, at::kByte);
  const at::Tensor log_prob = make({rows}, x, at::kFloat), entropy = make({rows}, x, at::kFloat),
                   row_max = make({rows}, x, at::kFloat), row_sum = make({rows}, x, at::kFloat),
                   item = make({rows, top}, x, at::kInt), top_lp = make({rows, top}, x, at::kFloat);
  // without given items every log probability is 0, as for given = -1
  const int rc = bgmf_log_probs(
      x.const_data_ptr(), type, rows, cols, x.stride(0), ex, ex_stride,
      static_cast<const int32_t *>(given), (float)number(a[3], "temperature"), (int32_t)top,
      given ? at_<float>(log_prob) : nullptr, at_<float>(entropy), at_<float>(row_max),
      at_<float>(row_sum), at_<int32_t>(item), at_<float>(top_lp),
      ws_bytes ? ws.mutable_data_ptr() : nullptr, ws_bytes, stream_of(a[5]));
  if (rc != BGMF_OK) return PyLong_FromLong(rc);
  if (!given) log_prob.zero_();
  return Py_BuildValue("(NNNNNN)", THPVariable_Wrap(log_prob), THPVariable_Wrap(entropy),
                       THPVariable_Wrap(item), THPVariable_Wrap(top_lp), THPVariable_Wrap(row_max),
                       THPVariable_Wrap(row_sum));
}

// (scores, given, row_max, row_sum, entropy, grad_log_prob, grad_entropy,
// temperature, excluded, out, stream) -> out
PyObject *log_probs_backward(PyObject *const *a) {
  int type;
  const at::Tensor &x = matrix(a[0], "scores", kFloats, &type);
  const int64_t rows = x.size(0), cols = x.size(1);
  const auto floats = [&](PyObject *o, const char *name, bool optional) {
    return static_cast<const float *>(vector(o, name, x, rows, at::kFloat, optional));
  };
  const float *row_max = floats(a[2], "row_max", false), *row_sum = floats(a[3], "row_sum", false),
              *entropy = floats(a[4], "entropy", true),
              *g_log_prob = floats(a[5], "grad_log_prob", true),
              *g_entropy = floats(a[6], "grad_entropy", true);
  const void *given = vector(a[1], "given", x, rows, at::kInt, true);
  int64_t ex_stride;
  const uint8_t *ex = excluded_items(a[8], x, &ex_stride);
  const c10::DeviceGuard guard(x.device());
  const at::Tensor out = output(a[9], "out", x, rows, cols, x.scalar_type());
  const int rc = bgmf_log_probs_grad(
      x.const_data_ptr(), type, rows, cols, x.stride(0), ex, ex_stride,
      static_cast<const int32_t *>(given), (float)number(a[7], "temperature"), row_max, row_sum,
      entropy, g_log_prob, g_entropy, out.mutable_data_ptr(), out.stride(0), stream_of(a[10]));
  if (rc != BGMF_OK) return PyLong_FromLong(rc);
  written(a[9], out);
  return THPVariable_Wrap(out);
}

// (x, stream) -> (q, scale); the rows of q start on 16-byte boundaries
PyObject *quantize_rows(PyObject *const *a) {
  int type;
  const at::Tensor &x = matrix(a[0], "x", kFloats, &type);
  const int64_t rows = x.size(0), k = x.size(1);
  if (k < 1) refuse("x has rows of no elements");
  const c10::DeviceGuard guard(x.device());
  const at::Tensor wide = make({rows, (k + 15) / 16 * 16}, x, at::kChar);
  const at::Tensor q = wide.narrow(1, 0, k), scale = make({rows}, x, at::kFloat);
  const int rc = bgmf_quantize_rows(x.const_data_ptr(), type, rows, k, x.stride(0),
                                    at_<int8_t>(q), q.stride(0), at_<float>(scale),
                                    stream_of(a[1]));
  if (rc != BGMF_OK) return PyLong_FromLong(rc);
  return Py_BuildValue("(NN)", THPVariable_Wrap(q), THPVariable_Wrap(scale));
}

// (rows, items, item_scale, row_scale, out type, out, stream) -> out
PyObject *quantized_scores(PyObject *const *a) {
  int type, item_type;
  const at::Tensor &x = matrix(a[0], "rows", kFloats | kBytes, &type);
  const at::Tensor &items = matrix(a[1], "items", kBytes, &item_type);
  const int64_t n = x.size(0), k = x.size(1), m = items.size(0);
  if (items.size(1) != k || items.device() != x.device())
    refuse("rows and items must have equally many columns, on one device");
  const void *item_scale = vector(a[2], "item_scale", x, m, at::kFloat, false);
  const void *row_scale = vector(a[3], "row_scale", x, n, at::kFloat, true);
  if ((a[3] != Py_None) != (type == BGMF_TYPE_I8))
    refuse("row_scale goes with int8 rows and with no others");
  const int out_type = (int)integer(a[4], "out type");
  const c10::DeviceGuard guard(x.device());
  const at::Tensor out = output(a[5], "out", x, n, m, dtype_of(out_type));
  const int64_t ws_bytes = bgmf_quantized_scores_workspace(n, m, k, type);
  at::Tensor ws;
  if (ws_bytes) ws = make({ws_bytes}, x, at::kByte);
  const int rc = bgmf_quantized_scores(
      x.const_data_ptr(), type, n, k, x.stride(0), static_cast<const float *>(row_scale),
      static_cast<const int8_t *>(items.const_data_ptr()), m, items.stride(0),
      static_cast<const float *>(item_scale), out.mutable_data_ptr(), out_type, out.stride(0),
      ws_bytes ? ws.mutable_data_ptr() : nullptr, ws_bytes, stream_of(a[6]));
  if (rc != BGMF_OK) return PyLong_FromLong(rc);
  written(a[5], out);
  return THPVariable_Wrap(out);
}

// rows x cols with a row stride that cover a gradient's elements.
void layout(const at::Tensor &t, bool as_matrix, int64_t *rows, int64_t *cols, int64_t *stride) {
  if (!as_matrix) {
    *rows = 1, *cols = *stride = t.numel();
    return;
  }
  if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1) ||
      (t.size(0) > 1 && t.stride(0) < t.size(1)))
    refuse("a gradient is neither contiguous nor 2-D with adjacent row elements");
  *rows = t.size(0), *cols = t.size(1), *stride = t.stride(0);
}

// (grads, max_norm, out or None, stream) -> norm; grads and out: lists
PyObject *clip_grad_norm(PyObject *const *a) {
  if (!PyList_Check(a[0]) || (a[2] != Py_None && !PyList_Check(a[2])))
    refuse("gradients come as a list");
  const bool in_place = a[2] == Py_None;
  const Py_ssize_t count = PyList_GET_SIZE(a[0]);
  if (count == 0) refuse("clip_grad_norm needs at least one gradient");
  if (!in_place && PyList_GET_SIZE(a[2]) != count) refuse("out must have a tensor for each gradient");
  std::vector<bgmf_grad_t> table((size_t)count);
  const at::Tensor &first = tensor(PyList_GET_ITEM(a[0], 0), "a gradient");
  for (Py_ssize_t i = 0; i < count; ++i) {
    const at::Tensor &g = tensor(PyList_GET_ITEM(a[0], i), "a gradient");
    const at::Tensor &o = in_place ? g : tensor(PyList_GET_ITEM(a[2], i), "out");
    bgmf_grad_t &e = table[(size_t)i];
    e.type = type_of(g);
    if (e.type < 0 || e.type == BGMF_TYPE_I8)
      refuse("gradients must be float32, bfloat16 or float16");
    if (!g.is_cuda() || g.device() != first.device() || o.device() != first.device())
      refuse("gradients and out must be on one GPU");
    if (o.scalar_type() != g.scalar_type() || o.sizes() != g.sizes())
      refuse("out must have the gradients' types and shapes");
    const bool as_matrix = !g.is_contiguous() || !o.is_contiguous();
    layout(g, as_matrix, &e.rows, &e.cols, &e.in_stride);
    layout(o, as_matrix, &e.rows, &e.cols, &e.out_stride);
    e.in = g.const_data_ptr();
    e.out = o.mutable_data_ptr();
  }
  const c10::DeviceGuard guard(first.device());
  const at::Tensor norm = make({}, first, at::kFloat);
  const int64_t ws_bytes = bgmf_clip_grad_norm_workspace(count);
  const at::Tensor ws = make({ws_bytes}, first, at::kByte);
  const int rc = bgmf_clip_grad_norm(table.data(), count, (float)number(a[1], "max_norm"),
                                     at_<float>(norm), ws.mutable_data_ptr(), ws_bytes,
                                     stream_of(a[3]));
  if (rc != BGMF_OK) return PyLong_FromLong(rc);
  PyObject *outs = in_place ? a[0] : a[2];
  for (Py_ssize_t i = 0; i < count; ++i) written(THPVariable_Unpack(PyList_GET_ITEM(outs, i)));
  return THPVariable_Wrap(norm);
}

// A 2-D tensor of bytes on the GPU, the bytes of a row adjacent.
const at::Tensor &byte_rows(PyObject *o, const char *name) {
  const at::Tensor &t = tensor(o, name);
  if (t.dim() != 2 || t.scalar_type() != at::kByte) refuse("%s must be a 2-D tensor of uint8", name);
  if (!t.is_cuda()) refuse("%s must be on the GPU", name);
  if (t.size(1) > 1 && t.stride(1) != 1)
    refuse("%s: the bytes of a row must be adjacent (call .contiguous())", name);
  return t;
}
// Rows in 4 bits with their scales: 16 bytes and one byte for each of their blocks.
const at::Tensor &blocks_of(PyObject *o, const char *name, PyObject *scales,
                            const char *scales_name, const at::Tensor **scale) {
  const at::Tensor &q = byte_rows(o, name), &s = byte_rows(scales, scales_name);
  if (s.size(0) != q.size(0) || q.size(1) != 16 * s.size(1) || s.device() != q.device())
    refuse("%s (rows of 16 bytes a block) and %s (rows of one) do not go together", name,
           scales_name);
  if (s.size(1) < 1) refuse("%s has rows of no elements", name);
  *scale = &s;
  return q;
}
const uint8_t *bytes(const at::Tensor &t) {
  return static_cast<const uint8_t *>(t.const_data_ptr());
}

// (x, stream) -> (q, scale)
PyObject *quantize_rows_mx(PyObject *const *a) {
  int type;
  const at::Tensor &x = matrix(a[0], "x", kFloats, &type);
  const int64_t rows = x.size(0), k = x.size(1), blocks = (k + 31) / 32;
  if (k < 1) refuse("x has rows of no elements");
  const c10::DeviceGuard guard(x.device());
  const at::Tensor q = make({rows, blocks * 16}, x, at::kByte),
                   scale = make({rows, blocks}, x, at::kByte);
  const int rc = bgmf_quantize_rows_mx(x.const_data_ptr(), type, rows, k, x.stride(0),
                                       at_<uint8_t>(q), blocks * 16, at_<uint8_t>(scale), blocks,
                                       stream_of(a[1]));
  if (rc != BGMF_OK) return PyLong_FromLong(rc);
  return Py_BuildValue("(NN)", THPVariable_Wrap(q), THPVariable_Wrap(scale));
}

// (q, scale, k or None, out type, out, stream) -> out
PyObject *dequantize_rows_mx(PyObject *const *a) {
  const at::Tensor *scale;
  const at::Tensor &q = blocks_of(a[0], "q", a[1], "scale", &scale);
  const int64_t rows = q.size(0), blocks = scale->size(1);
  const int64_t k = a[2] == Py_None ? blocks * 32 : integer(a[2], "k");
  if (k <= (blocks - 1) * 32 || k > blocks * 32)
    refuse("k must be in (%lld, %lld] for rows of %lld blocks", (long long)(blocks - 1) * 32,
           (long long)blocks * 32, (long long)blocks);
  const int out_type = (int)integer(a[3], "out type");
  const c10::DeviceGuard guard(q.device());
  const at::Tensor out = output(a[4], "out", q, rows, k, dtype_of(out_type));
  const int rc = bgmf_dequantize_rows_mx(bytes(q), q.stride(0), bytes(*scale), scale->stride(0),
                                         rows, k, out.mutable_data_ptr(), out_type, out.stride(0),
                                         stream_of(a[5]));
  if (rc != BGMF_OK) return PyLong_FromLong(rc);
  written(a[4], out);
  return THPVariable_Wrap(out);
}

// (rows, items, item_scale, row_scale, out type, out, stream) -> out
PyObject *mx_scores(PyObject *const *a) {
  const at::Tensor *item_scale, *row_scale = nullptr;
  const at::Tensor &items = blocks_of(a[1], "items", a[2], "item_scale", &item_scale);
  const int64_t blocks = item_scale->size(1), m = items.size(0);
  int type = BGMF_TYPE_MX4;
  int64_t k = blocks * 32;
  const at::Tensor *rows;
  if (a[3] != Py_None) {
    rows = &blocks_of(a[0], "rows", a[3], "row_scale", &row_scale);
    if (row_scale->size(1) != blocks) refuse("rows and items must have equally many blocks");
  } else {
    if (THPVariable_Check(a[0]) && THPVariable_Unpack(a[0]).scalar_type() == at::kByte)
      refuse("row_scale goes with uint8 rows and with no others");
    rows = &matrix(a[0], "rows", kFloats, &type);
    k = rows->size(1);
    if (k < 1 || (k + 31) / 32 != blocks)
      refuse("rows of %lld columns have %lld blocks, those of items %lld", (long long)k,
             (long long)(k + 31) / 32, (long long)blocks);
  }
  if (rows->device() != items.device()) refuse("rows and items must be on one device");
  const int64_t n = rows->size(0);
  const int out_type = (int)integer(a[4], "out type");
  const c10::DeviceGuard guard(items.device());
  const at::Tensor out = output(a[5], "out", items, n, m, dtype_of(out_type));
  const int64_t ws_bytes = bgmf_mx_scores_workspace(n, m, k, type);
  at::Tensor ws;
  if (ws_bytes) ws = make({ws_bytes}, items, at::kByte);
  const int rc = bgmf_mx_scores(
      rows->const_data_ptr(), type, n, k, rows->stride(0), row_scale ? bytes(*row_scale) : nullptr,
      row_scale ? row_scale->stride(0) : 0, bytes(items), m, items.stride(0), bytes(*item_scale),
      item_scale->stride(0), out.mutable_data_ptr(), out_type, out.stride(0),
      ws_bytes ? ws.mutable_data_ptr() : nullptr, ws_bytes, stream_of(a[6]));
  if (rc != BGMF_OK) return PyLong_FromLong(rc);
  written(a[5], out);
  return THPVariable_Wrap(out);
}

// The reference's scores, laid out as the policy's are.
const void *reference_scores(PyObject *o, const at::Tensor &x, int64_t *stride) {
  *stride = 0;
  if (o == Py_None) return nullptr;
  int type;
  const at::Tensor &t = matrix(o, "reference", kFloats, &type);
  if (t.sizes() != x.sizes() || t.scalar_type() != x.scalar_type() || t.device() != x.device())
    refuse("reference must have the shape, the type and the device of the scores");
  *stride = t.stride(0);
  return t.const_data_ptr();
}

// The current stream of a device, from the function that ranking.py gave
// (set_stream_function): a backward pass runs on a thread and, it may be, on a
// stream of PyTorch's choice.
PyObject *g_stream_function = nullptr;
void *current_stream(const at::Device &device) {
  const PyGILState_STATE gil = PyGILState_Ensure();
  PyObject *r = PyObject_CallFunction(g_stream_function, "i", (int)device.index());
  void *stream = r ? PyLong_AsVoidPtr(r) : nullptr;
  const bool failed = !r || PyErr_Occurred();
  PyErr_Clear();
  Py_XDECREF(r);
  PyGILState_Release(gil);
  if (failed) throw std::runtime_error("no current stream");
  return stream;
}
PyObject *set_stream_function(PyObject *const *a) {
  Py_XDECREF(g_stream_function);
  Py_INCREF(a[0]);
  g_stream_function = a[0];
  Py_INCREF(Py_None);
  return Py_None;
}

using torch::autograd::AutogradContext;
using torch::autograd::Variable;
using torch::autograd::variable_list;

// Results that have no derivative: a backward pass that reaches them raises.
struct NoDerivative : torch::autograd::Function<NoDerivative> {
  static Variable forward(AutogradContext *ctx, const Variable &result, const Variable &of,
                          const Variable &and_of, std::string name) {
    ctx->saved_data["name"] = name;
    return result.view(result.sizes());
  }
  static variable_list backward(AutogradContext *ctx, variable_list) {
    throw std::runtime_error(ctx->saved_data["name"].toStringRef() +
                             " has no derivative: call it under torch.no_grad(), or on detached "
                             "tensors");
  }
};

// A gradient as autograd passes it, in memory of its own kind: a view that negates
// is resolved, a tensor of zeros without memory gets some.  One whose derivative
// would be lost is refused.
at::Tensor passed(const Variable &g) {
  if (g._fw_grad(0).defined())
    throw Refused("a gradient has a tangent: forward-mode derivatives are not supported");
  if (!g.has_storage()) throw Refused("a gradient has no memory of its own (vmap?)");
  return (g._is_zerotensor() ? make(g.sizes(), g, g.scalar_type()).zero_() : g.resolve_neg())
      .contiguous();
}

// Saved tensors come back as they were, unless a hook of the caller's changes them.
void same_as(bool same, const char *name) {
  if (!same) throw Refused(std::string("the saved ") + name + " came back changed");
}

// The gradient from what the forward pass saved.
at::Tensor policy_gradient(const variable_list &saved, const at::Tensor &weight, double kl_weight,
                           double temperature) {
  const at::Tensor &x = saved[0], &given = saved[1], &ref = saved[2], &ex = saved[3],
                   &state = saved[4];
  const int64_t rows = x.size(0), cols = x.size(1);
  const auto adjacent = [&](const at::Tensor &t) {
    return t.is_cuda() && t.device() == x.device() && t.sizes() == x.sizes() &&
           (cols < 2 || t.stride(1) == 1);
  };
  const auto dense = [&](const at::Tensor &t, at::ScalarType type, int64_t count) {
    return t.device() == x.device() && t.scalar_type() == type && t.numel() == count &&
           t.is_contiguous();
  };
  same_as(adjacent(x), "scores");
  same_as(dense(given, at::kInt, rows), "given");
  same_as(!ref.defined() || (adjacent(ref) && ref.scalar_type() == x.scalar_type()), "reference");
  same_as(!ex.defined() || (adjacent(ex) && ex.element_size() == 1), "excluded");
  same_as(dense(state, at::kFloat, 5 * rows) && dense(weight, at::kFloat, rows), "state");
  const c10::DeviceGuard guard(x.device());
  const at::Tensor out = make(x.sizes(), x, x.scalar_type());
  check(bgmf_policy_loss_grad(
      x.const_data_ptr(), type_of(x), rows, cols, x.stride(0),
      ref.defined() ? ref.const_data_ptr() : nullptr, ref.defined() ? ref.stride(0) : 0,
      ex.defined() ? static_cast<const uint8_t *>(ex.const_data_ptr()) : nullptr,
      ex.defined() ? ex.stride(0) : 0, static_cast<const int32_t *>(given.const_data_ptr()),
      (float)temperature, (float)kl_weight, static_cast<const float *>(state.const_data_ptr()),
      static_cast<const float *>(weight.const_data_ptr()), out.mutable_data_ptr(), out.stride(0),
      current_stream(x.device())));
  return out;
}

// (scores, given, advantage, old_log_prob, reference, reference_log_prob,
// kl_weight, clip_low, clip_high, temperature, excluded, weight, out, stream),
// checked; the three results, with row_state or the gradient where wanted.
struct PolicyCall {
  const at::Tensor &x;
  int type;
  int64_t rows, cols, ex_stride, ref_stride;
  const void *given, *ref;
  const float *advantage, *old_log_prob, *ref_log_prob, *weight;
  const uint8_t *ex;
  double kl_weight, clip_low, clip_high, temperature;
  void *stream;
  at::Tensor loss, log_prob, kl, state, grad;

  explicit PolicyCall(PyObject *const *a) : x(matrix(a[0], "scores", kFloats, &type)) {
    rows = x.size(0), cols = x.size(1);
    const auto floats = [&](PyObject *o, const char *name, bool optional) {
      return static_cast<const float *>(vector(o, name, x, rows, at::kFloat, optional));
    };
    given = vector(a[1], "given", x, rows, at::kInt, false);
    advantage = floats(a[2], "advantage", false);
    old_log_prob = floats(a[3], "old_log_prob", false);
    ref_log_prob = floats(a[5], "reference_log_prob", true);
    weight = floats(a[11], "weight", true);
    ref = reference_scores(a[4], x, &ref_stride);
    if (a[4] != Py_None && a[5] != Py_None)
      refuse("reference or reference_log_prob, not both");
    ex = excluded_items(a[10], x, &ex_stride);
    kl_weight = number(a[6], "kl_weight"), clip_low = number(a[7], "clip_low");
    clip_high = number(a[8], "clip_high"), temperature = number(a[9], "temperature");
    stream = stream_of(a[13]);
  }
  // out: null for no gradient
  void run(bool want_state, PyObject *out, PyObject *scores = nullptr) {
    const c10::DeviceGuard guard(x.device());
    loss = make({rows}, x, at::kFloat), log_prob = make({rows}, x, at::kFloat);
    kl = make({rows}, x, at::kFloat);
    if (want_state) state = make({5, rows}, x, at::kFloat);
    if (out) grad = output(out, "out", x, rows, cols, x.scalar_type(), scores);
    at::Tensor ws;
    const int64_t ws_bytes = bgmf_policy_loss_workspace(rows, cols);
    if (ws_bytes) ws = make({ws_bytes}, x, at::kByte);
    check(bgmf_policy_loss(
        x.const_data_ptr(), type, rows, cols, x.stride(0), ref, ref_stride, ex, ex_stride,
        static_cast<const int32_t *>(given), advantage, old_log_prob, ref_log_prob,
        (float)temperature, (float)clip_low, (float)clip_high, (float)kl_weight, at_<float>(loss),
        at_<float>(log_prob), at_<float>(kl), want_state ? at_<float>(state) : nullptr, weight,
        out ? grad.mutable_data_ptr() : nullptr, out ? grad.stride(0) : 0,
        ws_bytes ? ws.mutable_data_ptr() : nullptr, ws_bytes, stream));
    if (out) written(out, grad);
  }
};

at::Tensor or_undefined(PyObject *o) {
  return o == Py_None ? at::Tensor() : THPVariable_Unpack(o);
}

// The loss in a graph: its derivative with respect to the scores.
struct PolicyLoss : torch::autograd::Function<PolicyLoss> {
  static variable_list forward(AutogradContext *ctx, const Variable &scores, PolicyCall *call,
                               PyObject *const *a) {
    call->run(true, nullptr);
    ctx->save_for_backward({scores, THPVariable_Unpack(a[1]), or_undefined(a[4]),
                            or_undefined(a[10]), call->state});
    ctx->saved_data["kl_weight"] = call->kl_weight;
    ctx->saved_data["temperature"] = call->temperature;
    ctx->mark_non_differentiable({call->log_prob, call->kl});
    return {call->loss, call->log_prob, call->kl};
  }
  static variable_list backward(AutogradContext *ctx, variable_list grads) {
    const variable_list saved = ctx->get_saved_variables();
    const Variable &x = saved[0];
    Variable grad;
    {
      const at::NoGradGuard no_grad;
      grad = policy_gradient(saved, passed(grads[0]), ctx->saved_data["kl_weight"].toDouble(),
                             ctx->saved_data["temperature"].toDouble());
    }
    if (in_graph(x) || in_graph(grads[0]))
      grad = NoDerivative::apply(grad, x, grads[0], std::string("the gradient of policy_loss"));
    return {grad, Variable(), Variable()};
  }
};

// PolicyCall's arguments -> (loss, log_prob, kl)
PyObject *policy_loss(PyObject *const *a) {
  PolicyCall call(a);
  if (in_graph(call.x)) {
    const variable_list r = PolicyLoss::apply(call.x, &call, a);
    return Py_BuildValue("(NNN)", THPVariable_Wrap(r[0]), THPVariable_Wrap(r[1]),
                         THPVariable_Wrap(r[2]));
  }
  call.run(false, nullptr);
  return Py_BuildValue("(NNN)", THPVariable_Wrap(call.loss), THPVariable_Wrap(call.log_prob),
                       THPVariable_Wrap(call.kl));
}

// The same -> (loss, log_prob, kl, the gradient of the losses times weight)
PyObject *policy_loss_and_grad(PyObject *const *a) {
  PolicyCall call(a);
  call.run(false, a[12], a[0]);
  return Py_BuildValue("(NNNN)", THPVariable_Wrap(call.loss), THPVariable_Wrap(call.log_prob),
                       THPVariable_Wrap(call.kl), THPVariable_Wrap(call.grad));
}

// A Python (or numpy) integer in [0, 2^64).
uint64_t word(PyObject *o, const char *name) {
  PyObject *i = THPVariable_Check(o) ? nullptr : PyNumber_Index(o);
  const unsigned long long v = i ? PyLong_AsUnsignedLongLong(i) : 0;
  Py_XDECREF(i);
  if (!i || PyErr_Occurred()) {
    PyErr_Clear();
    refuse("%s must be an integer in [0, 2^64)", name);
  }
  return v;
}

// x dropped into out (undefined: a new tensor).
at::Tensor dropped(const at::Tensor &x, double p, uint64_t seed, uint64_t offset,
                   const at::Tensor &on_device, at::Tensor out, void *stream) {
  int64_t rows = 1, cols = x.numel(), stride = cols, out_stride = cols;
  const bool as_matrix = !x.is_contiguous() || (out.defined() && !out.is_contiguous());
  const c10::DeviceGuard guard(x.device());
  if (!out.defined()) {
    out = make(x.sizes(), x, x.scalar_type());
  } else if (out.sizes() != x.sizes() || out.scalar_type() != x.scalar_type() ||
             out.device() != x.device()) {
    refuse("out must have the shape, the type and the device of x");
  }
  if (as_matrix) {
    if (x.dim() != 2 || (x.size(1) > 1 && (x.stride(1) != 1 || out.stride(1) != 1)))
      refuse("x and out must be contiguous, or 2-D with adjacent row elements");
    rows = x.size(0), cols = x.size(1), stride = x.stride(0), out_stride = out.stride(0);
  }
  check(bgmf_dropout(
      x.const_data_ptr(), type_of(x), rows, cols, stride, p, seed, offset,
      on_device.defined() ? static_cast<const uint64_t *>(on_device.const_data_ptr()) : nullptr,
      out.mutable_data_ptr(), out_stride, stream));
  return out;
}

// Dropout in a graph.  Its derivative drops the gradient alike, and has the same
// derivative itself.
struct Dropout : torch::autograd::Function<Dropout> {
  static std::optional<at::Tensor> optional(const at::Tensor &t) {
    return t.defined() ? std::optional<at::Tensor>(t) : std::nullopt;
  }
  static Variable forward(AutogradContext *ctx, const Variable &x, double p, int64_t seed,
                          int64_t offset, const std::optional<at::Tensor> &more, void *stream) {
    const Variable on_device = more ? *more : Variable();
    ctx->save_for_backward({on_device});
    ctx->saved_data["p"] = p, ctx->saved_data["seed"] = seed, ctx->saved_data["offset"] = offset;
    return dropped(x, p, (uint64_t)seed, (uint64_t)offset, on_device, at::Tensor(), stream);
  }
  static variable_list backward(AutogradContext *ctx, variable_list grads) {
    const Variable on_device = ctx->get_saved_variables()[0], g = passed(grads[0]);
    same_as(!on_device.defined() || (on_device.numel() == 1 && on_device.device() == g.device() &&
                                     on_device.scalar_type() == at::kLong),
            "offset");
    const double p = ctx->saved_data["p"].toDouble();
    const int64_t seed = ctx->saved_data["seed"].toInt(), offset = ctx->saved_data["offset"].toInt();
    void *stream = current_stream(g.device());
    const Variable grad = in_graph(g) ? apply(g, p, seed, offset, optional(on_device), stream)
                                      : dropped(g, p, (uint64_t)seed, (uint64_t)offset, on_device,
                                                at::Tensor(), stream);
    return {grad, Variable(), Variable(), Variable(), Variable(), Variable()};
  }
};

// (x, p, seed, offset, out, stream) -> out
PyObject *dropout(PyObject *const *a) {
  const at::Tensor &x = tensor(a[0], "x");
  const int type = type_of(x);
  if (type < 0 || !(kFloats >> type & 1)) refuse("x must be float32, bfloat16 or float16");
  if (!x.is_cuda()) refuse("x must be on the GPU");
  if (x.layout() != at::kStrided) refuse("x must be a dense tensor");
  const double p = number(a[1], "p");
  const uint64_t seed = word(a[2], "seed");
  uint64_t offset = 0;
  at::Tensor on_device;
  if (THPVariable_Check(a[3])) {
    on_device = tensor(a[3], "offset");
    if (on_device.numel() != 1 || on_device.scalar_type() != at::kLong ||
        on_device.device() != x.device())
      refuse("offset must be an integer or an int64 tensor of one element on the same GPU");
  } else {
    offset = word(a[3], "offset");
  }
  if (in_graph(x)) {
    if (a[4] != Py_None) refuse("dropout: out takes no part in a graph, and x requires grad");
    return THPVariable_Wrap(
        Dropout::apply(x, p, (int64_t)seed, (int64_t)offset, Dropout::optional(on_device),
                       stream_of(a[5])));
  }
  at::Tensor to;
  if (a[4] != Py_None) to = tensor(a[4], "out"), not_in_graph(to, "out");
  const at::Tensor out = dropped(x, p, seed, offset, on_device, to, stream_of(a[5]));
  written(a[4], out);
  return THPVariable_Wrap(out);
}

// PyTorch's exception for a full device, which callers catch by its type.
void set_out_of_memory(const c10::Error &e) {
  PyObject *torch = PyImport_ImportModule("torch");
  PyObject *type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
  if (type) PyErr_SetString(type, e.what_without_backtrace());
  Py_XDECREF(type);
  Py_XDECREF(torch);
}

// Argument count, and C++ exceptions as Python's.
template <PyObject *(*F)(PyObject *const *), Py_ssize_t N>
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n) {
  try {
    if (n != N) refuse("%lld arguments are needed", (long long)N);
    t_forward_mode = torch::autograd::ForwardADLevel::try_get_by_idx(0) != nullptr;
    return F(args);
  } catch (const Refused &e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const Failed &e) {
    return PyLong_FromLong(e.code);
  } catch (const c10::OutOfMemoryError &e) {
    set_out_of_memory(e);
  } catch (const std::bad_alloc &) {
    PyErr_NoMemory();
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

template <PyObject *(*F)(PyObject *const *), Py_ssize_t N>
PyMethodDef method(const char *name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&call<F, N>)),
          METH_FASTCALL, nullptr};
}

PyMethodDef g_methods[] = {
    method<log_probs, 6>("log_probs"),
    method<log_probs_backward, 11>("log_probs_backward"),
    method<quantize_rows, 2>("quantize_rows"),
    method<quantized_scores, 7>("quantized_scores"),
    method<clip_grad_norm, 4>("clip_grad_norm"),
    method<quantize_rows_mx, 2>("quantize_rows_mx"),
    method<dequantize_rows_mx, 6>("dequantize_rows_mx"),
    method<mx_scores, 7>("mx_scores"),
    method<policy_loss, 14>("policy_loss"),
    method<policy_loss_and_grad, 14>("policy_loss_and_grad"),
    method<set_stream_function, 1>("set_stream_function"),
    method<dropout, 6>("dropout"),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_ranking", nullptr, -1, g_methods,
                        nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ranking(void) { return PyModule_Create(&g_module); }
