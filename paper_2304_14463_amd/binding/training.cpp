// What the Python binding does before and behind the training operators' calls, natively: tensors and checkpoints
// checked and turned into descriptors, results and workspaces made.  Small calls are bound by the host: a row of 1000
// written as a checkpoint and read back takes the GPU 3 us.
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <stdint.h>
#include <algorithm>
#include <string>

#include "moccasin_training.h"

namespace {

// What bind() was given: the class of checkpoints, what says the current stream of a device, and the library's calls.
PyObject *checkpoint_class = nullptr, *current_stream = nullptr;
struct Calls {
  decltype(&moc_checkpoint_write) checkpoint_write;
  decltype(&moc_checkpoint_read) checkpoint_read;
  decltype(&moc_norm_forward) norm_forward;
  decltype(&moc_norm_backward) norm_backward;
  decltype(&moc_norm_backward_work) norm_backward_work;
  decltype(&moc_linear_forward) linear_forward;
  decltype(&moc_linear_backward_input) linear_backward_input;
  decltype(&moc_linear_backward_weight) linear_backward_weight;
  decltype(&moc_linear_work) linear_work;
} calls;
PyObject *name_codes, *name_scales, *name_fmt;   // interned

[[noreturn]] void refuse(PyObject* type, const std::string& what) {
  PyErr_SetString(type, what.c_str());
  throw python_error();
}
[[noreturn]] void bad(const char* what, const std::string& why) { refuse(PyExc_ValueError, std::string(what) + ": " + why); }

std::string sizes(int64_t rows, int64_t cols) { return std::to_string(rows) + " x " + std::to_string(cols); }

uintptr_t address(PyObject* x) {   // a Python int, or None: 0
  if (x == Py_None) return 0;
  const unsigned long long v = PyLong_AsUnsignedLongLong(x);
  if (v == (unsigned long long)-1 && PyErr_Occurred()) throw python_error();
  return (uintptr_t)v;
}

int32_t act_of(PyObject* x) {
  const long v = PyLong_AsLong(x);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return (int32_t)v;
}

bool truth(PyObject* x) {
  const int v = PyObject_IsTrue(x);
  if (v < 0) throw python_error();
  return v != 0;
}

int32_t type_of(at::ScalarType t, const char* what) {
  switch (t) {
    case at::kFloat: return MOC_F32;
    case at::kHalf: return MOC_F16;
    case at::kBFloat16: return MOC_BF16;
    default: bad(what, std::string("float32, float16 or bfloat16 expected, got ") + c10::toString(t));
  }
}

at::ScalarType dtype_of(PyObject* x, at::ScalarType otherwise) {
  if (x == Py_None) return otherwise;
  if (!THPDtype_Check(x)) refuse(PyExc_TypeError, "dtype: a torch.dtype expected");
  return reinterpret_cast<THPDtype*>(x)->scalar_type;
}

bool is_checkpoint(PyObject* x) { return (PyObject*)Py_TYPE(x) == checkpoint_class; }

// Elements from one row to the next.
int64_t stride_of(const at::Tensor& x, const char* what) {
  const int64_t rows = x.size(0), cols = x.size(1);
  if (cols > 1 && x.stride(1) != 1) bad(what, "the values of a row must lie next to each other");
  if (rows <= 1) return cols > 1 ? cols : 1;
  if (x.stride(0) < cols) bad(what, "rows must not overlap");
  return x.stride(0) > 1 ? x.stride(0) : 1;
}

// ---- memory that an output shares with an input -------------------------------------------------

// `rows` of `bytes`, `step` apart.
struct Span {
  uintptr_t at = 0;
  int64_t rows = 0, bytes = 0, step = 1;
};

// Of matrices with one step: whether a row of b begins before the end of a row of a and ends behind its start, d rows further on
// than it; the smallest d that is far enough is looked at.
bool shared_at_one_step(const Span& a, const Span& b, int64_t step) {
  const int64_t gap = (int64_t)(b.at - a.at), least = -b.bytes - gap;   // d * step > least
  const int64_t below = least / step - (least % step < 0 ? 1 : 0), d = std::max(below + 1, 1 - a.rows);
  return d < b.rows && gap + d * step < a.bytes;
}

bool shared(const Span& a, const Span& b) {
  if (a.rows < 1 || a.bytes < 1 || b.rows < 1 || b.bytes < 1) return false;
  if (b.at >= a.at + (a.rows - 1) * a.step + a.bytes || a.at >= b.at + (b.rows - 1) * b.step + b.bytes) return false;
  if (a.rows == 1) return shared_at_one_step(a, b, b.step);
  if (b.rows == 1 || a.step == b.step) return shared_at_one_step(a, b, a.step);
  const Span &few = a.rows < b.rows ? a : b, &many = a.rows < b.rows ? b : a;
  for (int64_t i = 0; i < few.rows; ++i)
    if (shared_at_one_step(Span{few.at + i * few.step, 1, few.bytes, 1}, many, many.step)) return true;
  return false;
}

// A tensor or a checkpoint, or nothing (None where that is allowed), as the library takes it.
struct Held {
  moc_matrix m = {};
  int64_t rows = 0, cols = 0;
  at::Tensor values;   // or the codes
  bool there = false, kept = false;
  const moc_matrix* get() const { return there ? &m : nullptr; }
  Span span() const {
    if (!there) return Span{};
    const int64_t each = values.element_size();
    return Span{reinterpret_cast<uintptr_t>(m.data), rows, cols * each, m.stride * each};
  }
  Span scale_span() const { return kept ? Span{reinterpret_cast<uintptr_t>(m.scales), rows, (cols + MOC_BLOCK - 1) / MOC_BLOCK, m.scale_stride} : Span{}; }
  // the very matrix
  bool is(const Held& o) const { return there && o.there && !kept && !o.kept && m.data == o.m.data && m.stride == o.m.stride && m.type == o.m.type; }
};

// Results are computed in any order: an output that shares memory with an input is refused, unless it is the input and each of
// its values is read before it is written (`in_place`).
void apart(const Held& out, const char* name, const Held& in, const char* what, bool in_place = false) {
  if (!out.there || !in.there || (in_place && out.is(in))) return;
  for (const Span& o : {out.span(), out.scale_span()})
    if (shared(o, in.span()) || shared(o, in.scale_span())) bad(name, std::string("shares memory with ") + what);
}

at::Tensor attribute(PyObject* x, PyObject* name, const char* what) {
  THPObjectPtr got(PyObject_GetAttr(x, name));
  if (!got) throw python_error();
  if (!THPVariable_Check(got.get())) bad(what, "a checkpoint's codes and scales must be two-dimensional CUDA tensors on one device");
  return THPVariable_Unpack(got.get());
}

Held held(PyObject* x, const char* what, int64_t rows = -1, int64_t cols = -1, bool optional = false) {
  Held h;
  if (optional && x == Py_None) return h;
  h.there = true;
  if (is_checkpoint(x)) {
    h.kept = true;
    h.values = attribute(x, name_codes, what);
    const at::Tensor scales = attribute(x, name_scales, what);
    if (!h.values.is_cuda() || !scales.is_cuda() || h.values.device() != scales.device() || h.values.dim() != 2 || scales.dim() != 2)
      bad(what, "a checkpoint's codes and scales must be two-dimensional CUDA tensors on one device");
    h.rows = h.values.size(0);
    h.cols = h.values.size(1);
    const int64_t blocks = (h.cols + MOC_BLOCK - 1) / MOC_BLOCK;
    if (h.values.element_size() != 1 || scales.element_size() != 1 || scales.size(0) != h.rows || scales.size(1) != blocks)
      bad(what, "a checkpoint of " + sizes(h.rows, h.cols) + " has bytes as codes and " + sizes(h.rows, blocks) + " bytes as scales");
    THPObjectPtr fmt(PyObject_GetAttr(x, name_fmt));
    if (!fmt) throw python_error();
    const bool text = PyUnicode_Check(fmt.get());
    h.m.type = text && PyUnicode_CompareWithASCIIString(fmt.get(), "e4m3") == 0   ? MOC_E4M3
               : text && PyUnicode_CompareWithASCIIString(fmt.get(), "int8") == 0 ? MOC_I8
                                                                                  : -1;
    if (h.m.type < 0) bad(what, "a checkpoint's format is \"e4m3\" or \"int8\"");
    h.m.scales = static_cast<uint8_t*>(scales.data_ptr());
    h.m.stride = stride_of(h.values, what);
    h.m.scale_stride = stride_of(scales, what);
  } else {
    if (!THPVariable_Check(x)) refuse(PyExc_TypeError, std::string(what) + ": a two-dimensional CUDA tensor or a Checkpoint expected");
    h.values = THPVariable_Unpack(x);
    if (!h.values.is_cuda() || h.values.dim() != 2) bad(what, "a two-dimensional CUDA tensor or a Checkpoint expected");
    h.rows = h.values.size(0);
    h.cols = h.values.size(1);
    h.m.stride = stride_of(h.values, what);
    h.m.type = type_of(h.values.scalar_type(), what);
  }
  h.m.data = h.values.data_ptr();
  if ((rows >= 0 && h.rows != rows) || (cols >= 0 && h.cols != cols))
    bad(what, sizes(rows >= 0 ? rows : h.rows, cols >= 0 ? cols : h.cols) + " expected, got " + sizes(h.rows, h.cols));
  return h;
}

void same_device(const at::Tensor& a, const at::Tensor& b) {
  if (b.defined() && a.device() != b.device()) refuse(PyExc_ValueError, "all arguments must be on one device");
}

// A vector of n values of float32, float16 or bfloat16 (`floats`: float32), or none.
struct Vector {
  at::Tensor x;
  void* data = nullptr;
  int32_t type = 0;
};
Vector vector(PyObject* p, int64_t n, const char* what, const at::Tensor& beside, bool floats = false) {
  Vector v;
  if (p == Py_None && !floats) return v;
  if (THPVariable_Check(p)) v.x = THPVariable_Unpack(p);
  if (!v.x.defined() || !v.x.is_cuda() || !v.x.is_contiguous() || v.x.numel() != n || (floats && v.x.scalar_type() != at::kFloat))
    bad(what, std::string("a contiguous ") + (floats ? "float32 " : "") + "CUDA tensor of " + std::to_string(n) + " values expected");
  same_device(beside, v.x);
  v.type = type_of(v.x.scalar_type(), what);
  v.data = v.x.data_ptr();
  return v;
}

// ---- results ------------------------------------------------------------------------------------

THPObjectPtr wrapped(at::Tensor x) {
  THPObjectPtr p(THPVariable_Wrap(std::move(x)));
  if (!p) throw python_error();
  return p;
}

at::Tensor room_for(const at::Tensor& like, at::ScalarType type, at::IntArrayRef dims) { return at::empty(dims, at::TensorOptions().dtype(type).device(like.device())); }

// The caller's tensor, or a new one.
THPObjectPtr result(PyObject* out, const at::Tensor& like, at::ScalarType type, int64_t rows, int64_t cols) {
  if (out == Py_None) return wrapped(room_for(like, type, {rows, cols}));
  Py_INCREF(out);
  return THPObjectPtr(out);
}

THPObjectPtr new_checkpoint(const at::Tensor& like, int64_t rows, int64_t cols, PyObject* fmt) {
  THPObjectPtr codes = wrapped(room_for(like, at::kByte, {rows, cols})), scales = wrapped(room_for(like, at::kByte, {rows, (cols + MOC_BLOCK - 1) / MOC_BLOCK}));
  PyObject* const args[3] = {codes.get(), scales.get(), fmt};
  THPObjectPtr made(PyObject_Vectorcall(checkpoint_class, args, 3, nullptr));
  if (!made) throw python_error();
  return made;
}

// None, the caller's checkpoint, or a new one of the format.
THPObjectPtr room_kept(PyObject* keep, const at::Tensor& like, int64_t rows, int64_t cols) {
  if (keep != Py_None && !is_checkpoint(keep)) return new_checkpoint(like, rows, cols, keep);
  Py_INCREF(keep);
  return THPObjectPtr(keep);
}

// The caller's workspace, or one of `need` bytes (negative: the library's refusal, which its call repeats).
struct Work {
  at::Tensor room;
  void* data = nullptr;
  int64_t bytes = 0;
};
Work workspace(PyObject* work, int64_t need, const at::Tensor& like) {
  Work w;
  if (work != Py_None) {
    if (!THPVariable_Check(work)) refuse(PyExc_TypeError, "work: a CUDA tensor expected");
    w.room = THPVariable_Unpack(work);
    if (!w.room.is_cuda() || !w.room.is_contiguous()) bad("work", "a contiguous CUDA tensor expected");
    same_device(like, w.room);
  } else if (need > 0) {
    w.room = room_for(like, at::kByte, {need});
  }
  if (w.room.defined()) {
    w.data = w.room.data_ptr();
    w.bytes = (int64_t)w.room.nbytes();
  }
  return w;
}

void arguments(Py_ssize_t count, Py_ssize_t wanted, const char* name) {
  if (count != wanted) refuse(PyExc_TypeError, std::string(name) + ": " + std::to_string(wanted) + " arguments");
  if (!checkpoint_class) refuse(PyExc_RuntimeError, "bind() comes first");
}
// The handle of the current stream, asked for when the arguments have been checked; refused where these are not on the current
// device, on which the kernels would run.
void* stream_for(const at::Tensor& x) {
  THPObjectPtr device(PyLong_FromLong(x.device().index()));
  if (!device) throw python_error();
  PyObject* const args[1] = {device.get()};
  THPObjectPtr handle(PyObject_Vectorcall(current_stream, args, 1, nullptr));
  if (!handle) throw python_error();
  return reinterpret_cast<void*>(address(handle));
}

template <class F>
int released(const F& f) {
  int code;
  Py_BEGIN_ALLOW_THREADS
  code = f();
  Py_END_ALLOW_THREADS
  return code;
}

// ---- the calls: each returns (code, results..) --------------------------------------------------

// checkpoint_write(x, fmt, out) -> (code, out)
PyObject* checkpoint_write(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 3, "checkpoint_write");
  const Held x = held(a[0], "x");
  THPObjectPtr out = room_kept(a[2] == Py_None ? a[1] : a[2], x.values, x.rows, x.cols);
  const Held k = held(out, "out", x.rows, x.cols);
  same_device(x.values, k.values);
  apart(k, "out", x, "x");
  void* const stream = stream_for(x.values);
  const int code = released([&] { return calls.checkpoint_write(x.rows, x.cols, x.get(), k.get(), stream); });
  return Py_BuildValue("iN", code, out.release());
  END_HANDLE_TH_ERRORS
}

// checkpoint_read(kept, dtype, act, out) -> (code, out)
PyObject* checkpoint_read(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 4, "checkpoint_read");
  const Held k = held(a[0], "kept");
  if (!k.kept) bad("kept", "a Checkpoint expected");
  const int32_t act = act_of(a[2]);
  THPObjectPtr out = result(a[3], k.values, dtype_of(a[1], at::kFloat), k.rows, k.cols);
  const Held y = held(out, "out", k.rows, k.cols);
  same_device(k.values, y.values);
  apart(y, "out", k, "kept");
  void* const stream = stream_for(k.values);
  const int code = released([&] { return calls.checkpoint_read(k.rows, k.cols, k.get(), act, y.get(), stream); });
  return Py_BuildValue("iN", code, out.release());
  END_HANDLE_TH_ERRORS
}

// norm_forward(x, gamma, beta, eps, keep, dtype, out) -> (code, y, mean, rstd, kept)
PyObject* norm_forward(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 7, "norm_forward");
  const Held x = held(a[0], "x");
  const Vector gamma = vector(a[1], x.cols, "gamma", x.values), beta = vector(a[2], x.cols, "beta", x.values);
  if (gamma.data && beta.data && gamma.type != beta.type) refuse(PyExc_ValueError, "gamma and beta must have one type");
  const double eps = PyFloat_AsDouble(a[3]);
  if (eps == -1.0 && PyErr_Occurred()) throw python_error();
  THPObjectPtr out = result(a[6], x.values, dtype_of(a[5], x.kept ? at::kFloat : x.values.scalar_type()), x.rows, x.cols), kept = room_kept(a[4], x.values, x.rows, x.cols);
  const Held y = held(out, "out", x.rows, x.cols), k = held(kept, "keep", x.rows, x.cols, true);
  same_device(x.values, y.values);
  same_device(x.values, k.values);
  apart(y, "out", x, "x", true);
  apart(k, "keep", x, "x");
  apart(k, "keep", y, "out");
  at::Tensor mean = room_for(x.values, at::kFloat, {x.rows}), rstd = room_for(x.values, at::kFloat, {x.rows});
  void* const stream = stream_for(x.values);
  const int code = released([&] {
    return calls.norm_forward(x.rows, x.cols, x.get(), gamma.data, beta.data, gamma.data ? gamma.type : beta.type, (float)eps, y.get(), k.get(),
                              static_cast<float*>(mean.data_ptr()), static_cast<float*>(rstd.data_ptr()), stream);
  });
  return Py_BuildValue("iNNNN", code, out.release(), wrapped(std::move(mean)).release(), wrapped(std::move(rstd)).release(), kept.release());
  END_HANDLE_TH_ERRORS
}

// norm_backward(dy, x, gamma, mean, rstd, residual, want_params, out, work) -> (code, dx, dgamma, dbeta)
PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 9, "norm_backward");
  const Held d = held(a[0], "dy"), x = held(a[1], "x", d.rows, d.cols), r = held(a[5], "residual", d.rows, d.cols, true);
  const Vector gamma = vector(a[2], d.cols, "gamma", d.values), mean = vector(a[3], d.rows, "mean", d.values, true), rstd = vector(a[4], d.rows, "rstd", d.values, true);
  same_device(d.values, x.values);
  same_device(d.values, r.values);
  THPObjectPtr out = result(a[7], d.values, d.values.scalar_type(), d.rows, d.cols);
  const Held dx = held(out, "out", d.rows, d.cols);
  same_device(d.values, dx.values);
  apart(dx, "out", d, "dy", true);
  apart(dx, "out", x, "x", true);
  apart(dx, "out", r, "residual", true);
  const bool params = truth(a[6]);
  Work work;
  THPObjectPtr dgamma, dbeta;
  float *pg = nullptr, *pb = nullptr;
  if (params) {
    at::Tensor grads = room_for(d.values, at::kFloat, {2, d.cols});   // next to each other: one launch adds both up
    work = workspace(a[8], a[8] == Py_None ? calls.norm_backward_work(d.rows, d.cols) : 0, d.values);
    pg = static_cast<float*>(grads.data_ptr());
    pb = pg + d.cols;
    dgamma = wrapped(grads.select(0, 0));
    dbeta = wrapped(grads.select(0, 1));
  } else {
    Py_INCREF(Py_None);
    Py_INCREF(Py_None);
    dgamma = Py_None;
    dbeta = Py_None;
  }
  void* const stream = stream_for(d.values);
  const int code = released([&] {
    return calls.norm_backward(d.rows, d.cols, d.get(), x.get(), gamma.data, gamma.type, static_cast<const float*>(mean.data), static_cast<const float*>(rstd.data), r.get(), dx.get(),
                               pg, pb, work.data, work.bytes, stream);
  });
  return Py_BuildValue("iNNN", code, out.release(), dgamma.release(), dbeta.release());
  END_HANDLE_TH_ERRORS
}

// linear_forward(x, w, bias, act, residual, keep, dtype, out, work) -> (code, y, kept)
PyObject* linear_forward(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 9, "linear_forward");
  const Held x = held(a[0], "x"), w = held(a[1], "w", -1, x.cols);
  const int64_t rows = x.rows, cin = x.cols, cout = w.rows;
  const Held r = held(a[4], "residual", rows, cout, true);
  const Vector bias = vector(a[2], cout, "bias", x.values);
  same_device(x.values, w.values);
  same_device(x.values, r.values);
  const int32_t act = act_of(a[3]);
  if (x.kept) bad("x", "a tensor expected");
  THPObjectPtr out = result(a[7], x.values, dtype_of(a[6], x.values.scalar_type()), rows, cout), kept = room_kept(a[5], x.values, rows, cout);
  const Held y = held(out, "out", rows, cout), k = held(kept, "keep", rows, cout, true);
  same_device(x.values, y.values);
  same_device(x.values, k.values);
  apart(y, "out", x, "x");
  apart(y, "out", w, "w");
  apart(y, "out", r, "residual", true);
  apart(k, "keep", x, "x");
  apart(k, "keep", w, "w");
  apart(k, "keep", r, "residual");
  apart(k, "keep", y, "out");
  const Work work = workspace(a[8], a[8] == Py_None ? calls.linear_work(rows, cin, cout) : 0, x.values);
  void* const stream = stream_for(x.values);
  const int code =
      released([&] { return calls.linear_forward(rows, cin, cout, x.get(), w.get(), bias.data, bias.type, act, r.get(), y.get(), k.get(), work.data, work.bytes, stream); });
  return Py_BuildValue("iNN", code, out.release(), kept.release());
  END_HANDLE_TH_ERRORS
}

// linear_backward_input(dy, w, act, pre, dtype, out, work) -> (code, dx)
PyObject* linear_backward_input(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 7, "linear_backward_input");
  const Held d = held(a[0], "dy"), w = held(a[1], "w", d.cols);
  const int64_t rows = d.rows, cout = d.cols, cin = w.cols;
  const Held pre = held(a[3], "pre", rows, cin, true);
  same_device(d.values, w.values);
  same_device(d.values, pre.values);
  const int32_t act = act_of(a[2]);
  if (d.kept) bad("dy", "a tensor expected");
  THPObjectPtr out = result(a[5], d.values, dtype_of(a[4], d.values.scalar_type()), rows, cin);
  const Held dx = held(out, "out", rows, cin);
  same_device(d.values, dx.values);
  apart(dx, "out", d, "dy");
  apart(dx, "out", w, "w");
  apart(dx, "out", pre, "pre", true);
  const Work work = workspace(a[6], a[6] == Py_None ? calls.linear_work(rows, cin, cout) : 0, d.values);
  void* const stream = stream_for(d.values);
  const int code = released([&] { return calls.linear_backward_input(rows, cin, cout, d.get(), w.get(), act, pre.get(), dx.get(), work.data, work.bytes, stream); });
  return Py_BuildValue("iN", code, out.release());
  END_HANDLE_TH_ERRORS
}

// linear_backward_weight(dy, x, dtype, want_bias, out, work) -> (code, dw, db)
PyObject* linear_backward_weight(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 6, "linear_backward_weight");
  const Held d = held(a[0], "dy"), x = held(a[1], "x", d.rows);
  const int64_t rows = d.rows, cout = d.cols, cin = x.cols;
  same_device(d.values, x.values);
  THPObjectPtr out = result(a[4], d.values, dtype_of(a[2], at::kFloat), cout, cin);
  const Held dw = held(out, "out", cout, cin);
  same_device(d.values, dw.values);
  apart(dw, "out", d, "dy");
  apart(dw, "out", x, "x");
  THPObjectPtr db;
  float* bias = nullptr;
  if (truth(a[3])) {
    at::Tensor sums = room_for(d.values, at::kFloat, {cout});
    bias = static_cast<float*>(sums.data_ptr());
    db = wrapped(std::move(sums));
  } else {
    Py_INCREF(Py_None);
    db = Py_None;
  }
  const Work work = workspace(a[5], a[5] == Py_None ? calls.linear_work(rows, cin, cout) : 0, d.values);
  void* const stream = stream_for(d.values);
  const int code = released([&] { return calls.linear_backward_weight(rows, cin, cout, d.get(), x.get(), dw.get(), bias, work.data, work.bytes, stream); });
  return Py_BuildValue("iNN", code, out.release(), db.release());
  END_HANDLE_TH_ERRORS
}

// shares((address, rows, bytes of a row, from one row to the next) twice): whether two matrices share memory
PyObject* shares(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  if (count != 8) refuse(PyExc_TypeError, "shares: 8 arguments");
  int64_t v[8];
  for (int i = 0; i < 8; ++i) v[i] = (int64_t)address(a[i]);
  if (v[3] < 1 || v[7] < 1) refuse(PyExc_ValueError, "shares: rows are apart");
  return PyBool_FromLong(shared(Span{(uintptr_t)v[0], v[1], v[2], v[3]}, Span{(uintptr_t)v[4], v[5], v[6], v[7]}));
  END_HANDLE_TH_ERRORS
}

// bind(class of checkpoints, current stream's handle as a function of the operands' device, {name of a call: its address})
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  if (count != 3 || !PyType_Check(a[0]) || !PyCallable_Check(a[1]) || !PyDict_Check(a[2])) refuse(PyExc_TypeError, "bind: a class, a function and a dict");
  Calls c;
  const auto take = [&](auto& call, const char* name) {
    PyObject* const at = PyDict_GetItemString(a[2], name);
    if (!at) refuse(PyExc_KeyError, name);
    call = reinterpret_cast<std::remove_reference_t<decltype(call)>>(address(at));
  };
  take(c.checkpoint_write, "moc_checkpoint_write");
  take(c.checkpoint_read, "moc_checkpoint_read");
  take(c.norm_forward, "moc_norm_forward");
  take(c.norm_backward, "moc_norm_backward");
  take(c.norm_backward_work, "moc_norm_backward_work");
  take(c.linear_forward, "moc_linear_forward");
  take(c.linear_backward_input, "moc_linear_backward_input");
  take(c.linear_backward_weight, "moc_linear_backward_weight");
  take(c.linear_work, "moc_linear_work");
  calls = c;
  Py_INCREF(a[0]);
  Py_INCREF(a[1]);
  Py_XDECREF(checkpoint_class);
  Py_XDECREF(current_stream);
  checkpoint_class = a[0];
  current_stream = a[1];
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

#define MOC_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {MOC_METHOD(bind), MOC_METHOD(checkpoint_write), MOC_METHOD(checkpoint_read), MOC_METHOD(norm_forward), MOC_METHOD(norm_backward), MOC_METHOD(linear_forward),
                         MOC_METHOD(linear_backward_input), MOC_METHOD(linear_backward_weight), MOC_METHOD(shares), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_training", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// training_version: of the header that this was built with.
PyMODINIT_FUNC PyInit__training() {
  name_codes = PyUnicode_InternFromString("codes");
  name_scales = PyUnicode_InternFromString("scales");
  name_fmt = PyUnicode_InternFromString("fmt");
  PyObject* const made = name_codes && name_scales && name_fmt ? PyModule_Create(&module) : nullptr;
  if (made && PyModule_AddIntConstant(made, "training_version", MOC_TRAINING_VERSION) != 0) {
    Py_DECREF(made);
    return nullptr;
  }
  return made;
}
