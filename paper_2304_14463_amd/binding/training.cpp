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
#include <initializer_list>
#include <string>
#include <utility>
#include <vector>

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
  decltype(&moc_residual_forward) residual_forward;
  decltype(&moc_residual_backward) residual_backward;
  decltype(&moc_residual_backward_work) residual_backward_work;
  decltype(&moc_logprob_forward_work) logprob_forward_work;
  decltype(&moc_logprob_forward) logprob_forward;
  decltype(&moc_logprob_backward) logprob_backward;
  decltype(&moc_adamw_step) adamw_step;
  decltype(&moc_moments_read) moments_read;
} calls;
PyObject *name_codes, *name_scales, *name_fmt, *name_m, *name_v, *name_m_scales, *name_v_scales;   // interned

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
  at::Tensor scales;
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
    h.scales = attribute(x, name_scales, what);
    const at::Tensor& scales = h.scales;
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

// A tensor that a call has written to: autograd refuses graphs that have saved it, as after any change in place.
void changed(const at::Tensor& t) {
  if (t.defined() && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// What of these the caller gave (`given`) has been written to, where the call was not refused.
void changed(int code, std::initializer_list<std::pair<const Held*, PyObject*>> outputs) {
  if (code != MOC_OK) return;
  for (const auto& [h, given] : outputs) {
    if (!THPVariable_Check(given) && !is_checkpoint(given)) continue;
    changed(h->values);
    changed(h->scales);
  }
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
  changed(code, {{&k, a[2]}});
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
  changed(code, {{&y, a[3]}});
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
  changed(code, {{&y, a[6]}, {&k, a[4]}});
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
  changed(code, {{&dx, a[7]}});
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
  changed(code, {{&y, a[7]}, {&k, a[5]}});
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
  changed(code, {{&dx, a[5]}});
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
  changed(code, {{&dw, a[4]}});
  return Py_BuildValue("iNN", code, out.release(), db.release());
  END_HANDLE_TH_ERRORS
}

double number(PyObject* x) {
  const double v = PyFloat_AsDouble(x);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return v;
}

// A vector of floats that may be missing.
Vector floats_or_none(PyObject* p, int64_t n, const char* what, const at::Tensor& beside) { return p == Py_None ? Vector{} : vector(p, n, what, beside, true); }

void apart(const Held& out, const char* name, const Vector& in, const char* what) {
  if (!out.there || !in.data || in.x.numel() == 0) return;
  const Span of{reinterpret_cast<uintptr_t>(in.data), 1, (int64_t)in.x.nbytes(), 1};
  if (shared(out.span(), of) || shared(out.scale_span(), of)) bad(name, std::string("shares memory with ") + what);
}

PyObject* none() {
  Py_INCREF(Py_None);
  return Py_None;
}

// ---- the residual connection --------------------------------------------------------------------

// A norm as Python has it: None, or (kind, gamma, beta, eps).
struct RowNorm {
  moc_row_norm n = {};
  Vector gamma, beta, mean, rstd;
  THPObjectPtr stats;   // (mean or None, rstd)
  bool on() const { return n.kind != MOC_NORM_NONE; }
  const moc_row_norm* get() const { return on() ? &n : nullptr; }
};
RowNorm row_norm_of(PyObject* x, int64_t cols, const char* what, const at::Tensor& beside) {
  RowNorm r;
  if (x == Py_None) return r;
  if (!PyTuple_Check(x) || PyTuple_GET_SIZE(x) != 4) refuse(PyExc_TypeError, std::string(what) + ": a Norm or None expected");
  PyObject* const kind = PyTuple_GET_ITEM(x, 0);
  const bool text = PyUnicode_Check(kind);
  r.n.kind = text && PyUnicode_CompareWithASCIIString(kind, "layer") == 0 ? MOC_NORM_LAYER : text && PyUnicode_CompareWithASCIIString(kind, "rms") == 0 ? MOC_NORM_RMS : -1;
  if (r.n.kind < 0) bad(what, "a norm's kind is \"layer\" or \"rms\"");
  r.gamma = vector(PyTuple_GET_ITEM(x, 1), cols, what, beside);
  r.beta = vector(PyTuple_GET_ITEM(x, 2), cols, what, beside);
  if (r.beta.data && r.n.kind == MOC_NORM_RMS) bad(what, "a norm of kind \"rms\" has no beta");
  if (r.gamma.data && r.beta.data && r.gamma.type != r.beta.type) bad(what, "gamma and beta must have one type");
  const double eps = number(PyTuple_GET_ITEM(x, 3));
  if (!(eps >= 0.0)) bad(what, "eps is a number of 0 or more");
  r.n.gamma = r.gamma.data;
  r.n.beta = r.beta.data;
  r.n.param_type = r.gamma.data ? r.gamma.type : r.beta.type;
  r.n.eps = (float)eps;
  return r;
}
// Room for a norm's statistics.
void room_for_statistics(RowNorm& r, int64_t rows, const at::Tensor& like) {
  if (!r.on()) {
    r.stats = THPObjectPtr(none());
    return;
  }
  THPObjectPtr mean(none()), rstd;
  if (r.n.kind == MOC_NORM_LAYER) {
    at::Tensor x = room_for(like, at::kFloat, {rows});
    r.n.mean = static_cast<float*>(x.data_ptr());
    mean = wrapped(std::move(x));
  }
  at::Tensor x = room_for(like, at::kFloat, {rows});
  r.n.rstd = static_cast<float*>(x.data_ptr());
  rstd = wrapped(std::move(x));
  r.stats = THPObjectPtr(PyTuple_Pack(2, mean.get(), rstd.get()));
  if (!r.stats) throw python_error();
}
// A norm's statistics as the forward pass has returned them.
void take_statistics(RowNorm& r, PyObject* x, int64_t rows, const char* what, const at::Tensor& beside) {
  if (!r.on()) return;
  if (!PyTuple_Check(x) || PyTuple_GET_SIZE(x) != 2) bad(what, "the statistics (mean, rstd) of the forward pass expected");
  if (r.n.kind == MOC_NORM_LAYER) {
    r.mean = vector(PyTuple_GET_ITEM(x, 0), rows, what, beside, true);
    r.n.mean = static_cast<float*>(r.mean.data);
  }
  r.rstd = vector(PyTuple_GET_ITEM(x, 1), rows, what, beside, true);
  r.n.rstd = static_cast<float*>(r.rstd.data);
}

// A gate for every rows / gates rows: [gates][cols], or [cols] for all of them.
Held gate_of(PyObject* x, int64_t rows, int64_t cols, const at::Tensor& beside) {
  Held h;
  if (x == Py_None) return h;
  if (THPVariable_Check(x) && THPVariable_Unpack(x).dim() == 1) {
    THPObjectPtr row = wrapped(THPVariable_Unpack(x).unsqueeze(0));
    h = held(row, "gate", 1, cols);
  } else {
    h = held(x, "gate", -1, cols);
  }
  if (h.kept) bad("gate", "a tensor expected");
  if (h.rows < 1 || h.rows > std::max<int64_t>(rows, 1) || rows % h.rows != 0) bad("gate", "a number of rows that divides " + std::to_string(rows) + " expected");
  same_device(beside, h.values);
  return h;
}

void apart_from_norm(const Held& out, const char* name, const RowNorm& r) {
  for (const Vector* v : {&r.gamma, &r.beta, &r.mean, &r.rstd}) apart(out, name, *v, "a norm's vector");
}

at::ScalarType first_type(std::initializer_list<const Held*> of, at::ScalarType otherwise) {
  for (const Held* h : of)
    if (h->there && !h->kept) return h->values.scalar_type();
  return otherwise;
}

// residual_forward(x, block, gate, scale, after, before, keep, dtype, want_stream, out, out_norm) -> (code, r, n, after's statistics, before's, kept)
PyObject* residual_forward(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 11, "residual_forward");
  const Held b = held(a[1], "block"), x = held(a[0], "x", b.rows, b.cols, true);
  if (x.kept) bad("x", "a tensor expected");
  same_device(b.values, x.values);
  const Held gate = gate_of(a[2], b.rows, b.cols, b.values);
  const double scale = number(a[3]);
  RowNorm after = row_norm_of(a[4], b.cols, "after", b.values), before = row_norm_of(a[5], b.cols, "before", b.values);
  if (!before.on() && a[6] != Py_None) bad("keep", "there is no norm to keep");
  if (!before.on() && a[10] != Py_None) bad("out_norm", "there is no norm before the next block");
  const bool stream_too = truth(a[8]);
  if (!stream_too && !before.on()) bad("want_stream", "neither the stream nor a norm of it is wanted");
  THPObjectPtr r, n, kept;
  r = stream_too ? result(a[9], b.values, first_type({&x, &b}, dtype_of(a[7], at::kFloat)), b.rows, b.cols) : THPObjectPtr(none());
  n = before.on() ? result(a[10], b.values, dtype_of(a[7], first_type({&b, &x}, at::kFloat)), b.rows, b.cols) : THPObjectPtr(none());
  kept = room_kept(a[6], b.values, b.rows, b.cols);
  const Held hr = held(r, "out", b.rows, b.cols, true), hn = held(n, "out_norm", b.rows, b.cols, true), hk = held(kept, "keep", b.rows, b.cols, true);
  for (const Held* h : {&hr, &hn, &hk}) same_device(b.values, h->values);
  for (const Held* h : {&hr, &hn}) {
    const char* const name = h == &hr ? "out" : "out_norm";
    apart(*h, name, x, "x", true);
    apart(*h, name, b, "block", true);
    apart(*h, name, gate, "gate");
    apart_from_norm(*h, name, after);
    apart_from_norm(*h, name, before);
  }
  apart(hn, "out_norm", hr, "out");
  for (const Held* h : {&x, &b, &gate, &hr, &hn}) apart(hk, "keep", *h, "another argument");
  apart_from_norm(hk, "keep", after);
  apart_from_norm(hk, "keep", before);
  room_for_statistics(after, b.rows, b.values);
  room_for_statistics(before, b.rows, b.values);
  void* const stream = stream_for(b.values);
  const int code = released([&] {
    return calls.residual_forward(b.rows, b.cols, x.get(), b.get(), gate.get(), gate.there ? gate.rows : 0, (float)scale, after.get(), before.get(), hr.get(), hn.get(), hk.get(), stream);
  });
  changed(code, {{&hr, a[9]}, {&hn, a[10]}, {&hk, a[6]}});
  return Py_BuildValue("iNNNNN", code, r.release(), n.release(), after.stats.release(), before.stats.release(), kept.release());
  END_HANDLE_TH_ERRORS
}

// residual_backward(dr, dn, r, block, gate, scale, after, after_stats, before, before_stats, want_x, want_params, dtype, out_x, out_block, work)
//   -> (code, dx, dblock, gate, after_gamma, after_beta, before_gamma, before_beta)
PyObject* residual_backward(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 16, "residual_backward");
  const bool by_dr = a[0] != Py_None;
  const Held lead = held(by_dr ? a[0] : a[1], by_dr ? "dr" : "dn");
  const int64_t rows = lead.rows, cols = lead.cols;
  const Held dr = held(a[0], "dr", rows, cols, true), dn = held(a[1], "dn", rows, cols, true), r = held(a[2], "r", rows, cols, true), b = held(a[3], "block", rows, cols, true);
  if (dr.kept || dn.kept) bad(dr.kept ? "dr" : "dn", "a tensor expected");
  for (const Held* h : {&dr, &dn, &r, &b}) same_device(lead.values, h->values);
  const Held gate = gate_of(a[4], rows, cols, lead.values);
  const double scale = number(a[5]);
  RowNorm after = row_norm_of(a[6], cols, "after", lead.values), before = row_norm_of(a[8], cols, "before", lead.values);
  take_statistics(after, a[7], rows, "after_stats", lead.values);
  take_statistics(before, a[9], rows, "before_stats", lead.values);
  if (before.on() != dn.there) bad("dn", before.on() ? "the gradient of the norm is missing" : "there is no norm before the next block");
  if (before.on() && !r.there) bad("r", "the stream is missing");
  const bool params = truth(a[11]);
  if (!b.there && (after.on() || (gate.there && params))) bad("block", "the block's output is missing");
  THPObjectPtr x_out, b_out;
  x_out = a[13] != Py_None || truth(a[10]) ? result(a[13], lead.values, first_type({&dr, &r, &dn}, at::kFloat), rows, cols) : THPObjectPtr(none());
  b_out = result(a[14], lead.values, dtype_of(a[12], first_type({&b, &dn, &dr}, at::kFloat)), rows, cols);
  const Held dx = held(x_out, "out_x", rows, cols, true), db = held(b_out, "out_block", rows, cols);
  for (const Held* h : {&dx, &db}) {
    const char* const name = h == &dx ? "out_x" : "out_block";
    same_device(lead.values, h->values);
    apart(*h, name, dr, "dr", h == &dx);
    apart(*h, name, r, "r", h == &dx);
    apart(*h, name, dn, "dn", h == &db);
    apart(*h, name, b, "block", h == &db);
    apart(*h, name, gate, "gate");
    apart_from_norm(*h, name, after);
    apart_from_norm(*h, name, before);
  }
  apart(dx, "out_x", db, "out_block");
  moc_residual_grads grads = {};
  THPObjectPtr got[5];   // gate, after's gamma and beta, before's
  float** const at[5] = {&grads.gate, &grads.after_gamma, &grads.after_beta, &grads.before_gamma, &grads.before_beta};
  const bool wanted[5] = {gate.there, after.gamma.data != nullptr, after.beta.data != nullptr, before.gamma.data != nullptr, before.beta.data != nullptr};
  for (int i = 0; i < 5; ++i) {
    if (!params || !wanted[i]) {
      got[i] = THPObjectPtr(none());
      continue;
    }
    at::Tensor t = i == 0 ? room_for(lead.values, at::kFloat, {gate.rows, cols}) : room_for(lead.values, at::kFloat, {cols});
    *at[i] = static_cast<float*>(t.data_ptr());
    got[i] = wrapped(std::move(t));
  }
  const int64_t gates = gate.there ? gate.rows : 0;
  const Work work = workspace(a[15], a[15] == Py_None && params ? calls.residual_backward_work(rows, cols, gates) : 0, lead.values);
  void* const stream = stream_for(lead.values);
  const int code = released([&] {
    return calls.residual_backward(rows, cols, dr.get(), dn.get(), r.get(), b.get(), gate.get(), gates, (float)scale, after.get(), before.get(), dx.get(), db.get(), &grads, work.data,
                                   work.bytes, stream);
  });
  changed(code, {{&dx, a[13]}, {&db, a[14]}});
  return Py_BuildValue("iNNNNNNN", code, x_out.release(), b_out.release(), got[0].release(), got[1].release(), got[2].release(), got[3].release(), got[4].release());
  END_HANDLE_TH_ERRORS
}

// ---- log probabilities --------------------------------------------------------------------------

// n signed numbers of 4 or 8 bytes, or none.
struct Tokens {
  Vector v;
  int32_t bytes = 0;
};
Tokens tokens_of(PyObject* p, int64_t n, const at::Tensor& beside) {
  Tokens t;
  if (p == Py_None) return t;
  if (THPVariable_Check(p)) t.v.x = THPVariable_Unpack(p);
  const at::Tensor& x = t.v.x;
  if (!x.defined() || !x.is_cuda() || !x.is_contiguous() || x.dim() != 1 || x.numel() != n || (x.scalar_type() != at::kInt && x.scalar_type() != at::kLong))
    bad("tokens", "a contiguous int32 or int64 CUDA tensor of " + std::to_string(n) + " values expected");
  same_device(beside, x);
  t.v.data = x.data_ptr();
  t.bytes = (int32_t)x.element_size();
  return t;
}

// logprob_forward(logits, tokens, scale, top, work) -> (code, logp, lse, entropy, top_logp, top_tokens)
PyObject* logprob_forward(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 5, "logprob_forward");
  const Held x = held(a[0], "logits");
  if (x.kept) bad("logits", "a tensor expected");
  const Tokens tokens = tokens_of(a[1], x.rows, x.values);
  const double scale = number(a[2]);
  const long top = PyLong_AsLong(a[3]);
  if (top == -1 && PyErr_Occurred()) throw python_error();
  if (top < 0 || top > 64 || top > x.cols) bad("top", "a number from 0 to 64, at most that of the columns, expected");
  // tensors of their own: views of one would share its version, and autograd refuses changes of a function's views
  at::Tensor logp, lse = room_for(x.values, at::kFloat, {x.rows}), entropy = room_for(x.values, at::kFloat, {x.rows}), top_logp, top_tokens;
  if (tokens.bytes) logp = room_for(x.values, at::kFloat, {x.rows});
  if (top > 0) {
    top_logp = room_for(x.values, at::kFloat, {x.rows, top});
    top_tokens = room_for(x.values, at::kLong, {x.rows, top});
  }
  const Work work = workspace(a[4], a[4] == Py_None ? calls.logprob_forward_work(x.rows, x.cols, (int32_t)top) : 0, x.values);
  const auto floats = [](const at::Tensor& t) { return t.defined() ? static_cast<float*>(t.data_ptr()) : nullptr; };
  void* const stream = stream_for(x.values);
  const int code = released([&] {
    return calls.logprob_forward(x.rows, x.cols, x.get(), tokens.v.data, tokens.bytes, (float)scale, (int32_t)top, floats(logp), floats(lse), floats(entropy), floats(top_logp),
                                 top > 0 ? static_cast<int64_t*>(top_tokens.data_ptr()) : nullptr, work.data, work.bytes,
                                 stream);
  });
  return Py_BuildValue("iNNNNN", code, tokens.bytes ? wrapped(std::move(logp)).release() : none(), wrapped(std::move(lse)).release(), wrapped(std::move(entropy)).release(),
                       top > 0 ? wrapped(std::move(top_logp)).release() : none(), top > 0 ? wrapped(std::move(top_tokens)).release() : none());
  END_HANDLE_TH_ERRORS
}

// logprob_backward(logits, lse, tokens, dlogp, entropy, dentropy, scale, dtype, out) -> (code, out)
PyObject* logprob_backward(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 9, "logprob_backward");
  const Held x = held(a[0], "logits");
  if (x.kept) bad("logits", "a tensor expected");
  const Vector lse = vector(a[1], x.rows, "lse", x.values, true), dlogp = floats_or_none(a[3], x.rows, "dlogp", x.values), entropy = floats_or_none(a[4], x.rows, "entropy", x.values),
               dentropy = floats_or_none(a[5], x.rows, "dentropy", x.values);
  const Tokens tokens = tokens_of(a[2], x.rows, x.values);
  if (a[2] == Py_None && a[3] != Py_None) bad("dlogp", "tokens are missing");
  if (a[5] != Py_None && a[4] == Py_None) bad("dentropy", "the entropy is missing");
  const double scale = number(a[6]);
  THPObjectPtr out = result(a[8], x.values, dtype_of(a[7], x.values.scalar_type()), x.rows, x.cols);
  const Held d = held(out, "out", x.rows, x.cols);
  same_device(x.values, d.values);
  apart(d, "out", x, "logits", true);
  for (const Vector* v : {&lse, &dlogp, &entropy, &dentropy, &tokens.v}) apart(d, "out", *v, "a vector of the call");
  void* const stream = stream_for(x.values);
  const int code = released([&] {
    return calls.logprob_backward(x.rows, x.cols, x.get(), static_cast<const float*>(lse.data), static_cast<const float*>(entropy.data), dlogp.data ? tokens.v.data : nullptr, tokens.bytes,
                                  static_cast<const float*>(dlogp.data), static_cast<const float*>(dentropy.data), (float)scale, d.get(), stream);
  });
  changed(code, {{&d, a[8]}});
  return Py_BuildValue("iN", code, out.release());
  END_HANDLE_TH_ERRORS
}

// ---- many tensors at once -----------------------------------------------------------------------

// The items of a sequence.
struct Items {
  THPObjectPtr seq;
  int64_t count = 0;
  Items(PyObject* x, const char* what, int64_t wanted = -1) : seq(PySequence_Fast(x, "")) {
    if (!seq) {
      PyErr_Clear();
      refuse(PyExc_TypeError, std::string(what) + ": a sequence expected");
    }
    count = PySequence_Fast_GET_SIZE(seq.get());
    if (wanted >= 0 && count != wanted) bad(what, std::to_string(wanted) + " items expected, got " + std::to_string(count));
  }
  // as they are in hand: what the caller gave may be an iterator
  PyObject* items() const { return const_cast<PyObject*>(seq.get()); }
  PyObject* operator[](int64_t i) const { return PySequence_Fast_GET_ITEM(items(), i); }
};

std::string item(const char* what, int64_t i) { return std::string(what) + "[" + std::to_string(i) + "]"; }

// What a call over many tensors has in hand: their device, and which memory it reads and writes.
struct Many {
  struct Piece {
    uintptr_t at, end;
    bool written;
  };
  std::vector<Piece> pieces;
  std::vector<at::Tensor> outputs;
  at::Tensor like;
  void expect(int64_t read, int64_t written) {
    pieces.reserve((size_t)(read + written));
    outputs.reserve((size_t)written);
  }
  // A contiguous CUDA tensor of n values (n < 0: any number).
  at::Tensor take(PyObject* x, const char* what, int64_t i, int64_t n, bool written) {
    if (!THPVariable_Check(x)) refuse(PyExc_TypeError, item(what, i) + ": a CUDA tensor expected");
    const at::Tensor& t = THPVariable_Unpack(x);
    if (!t.is_cuda() || !t.is_contiguous() || (n >= 0 && t.numel() != n)) bad(item(what, i).c_str(), n >= 0 ? "a contiguous CUDA tensor of " + std::to_string(n) + " values expected" : "a contiguous CUDA tensor expected");
    if (!like.defined()) like = t;
    same_device(like, t);
    const uintptr_t at = reinterpret_cast<uintptr_t>(t.data_ptr());
    if (t.numel() > 0) pieces.push_back({at, at + t.nbytes(), written});
    if (written) outputs.push_back(t);
    return t;
  }
  void written(int code) const {
    if (code != MOC_OK) return;
    for (const at::Tensor& t : outputs) changed(t);
  }
  // What is written is apart from everything else.
  void check(const char* what) {
    std::sort(pieces.begin(), pieces.end(), [](const Piece& a, const Piece& b) { return a.at < b.at; });
    uintptr_t any = 0, written = 0;
    for (const Piece& p : pieces) {
      if (p.at < written || (p.written && p.at < any)) bad(what, "memory that is written is shared between the tensors of a call");
      any = std::max(any, p.end);
      if (p.written) written = std::max(written, p.end);
    }
  }
};

struct Pair {   // a tensor's moments
  at::Tensor m, v, m_scales, v_scales;
  int32_t type;
};
Pair moments_of(PyObject* x, int64_t i, int64_t n, Many& many, bool written) {
  PyObject* const names[4] = {name_m, name_v, name_m_scales, name_v_scales};
  THPObjectPtr got[4];
  for (int k = 0; k < 4; ++k) {
    got[k] = THPObjectPtr(PyObject_GetAttr(x, names[k]));
    if (!got[k]) {
      PyErr_Clear();
      refuse(PyExc_TypeError, item("moments", i) + ": Moments expected");
    }
  }
  Pair p;
  p.m = many.take(got[0], "moments", i, n, written);
  p.v = many.take(got[1], "moments", i, p.m.numel(), written);
  const auto kind = p.m.scalar_type();
  if (kind != p.v.scalar_type() || (kind != at::kFloat && kind != at::kByte)) bad(item("moments", i).c_str(), "both float32, or both bytes");
  p.type = kind == at::kFloat ? MOC_F32 : MOC_E4M3;
  if (p.type == MOC_E4M3) {
    const int64_t blocks = (p.m.numel() + MOC_BLOCK - 1) / MOC_BLOCK;
    p.m_scales = many.take(got[2], "moments", i, blocks, written);
    p.v_scales = many.take(got[3], "moments", i, blocks, written);
    if (p.m_scales.scalar_type() != at::kByte || p.v_scales.scalar_type() != at::kByte) bad(item("moments", i).c_str(), "scales are bytes");
  } else if (got[2] != Py_None || got[3] != Py_None) {
    bad(item("moments", i).c_str(), "moments in 32 bits have no scales");
  }
  return p;
}

// A number, or where the device finds it: a tensor of one value.
template <class T>
const T* on_device(PyObject* x, const char* what, at::ScalarType type, Many& many) {
  if (!THPVariable_Check(x)) return nullptr;
  const at::Tensor t = many.take(x, what, 0, 1, false);
  if (t.scalar_type() != type) bad(what, std::string("a number or a ") + c10::toString(type) + " tensor of one value expected");
  return static_cast<const T*>(t.data_ptr());
}

// adamw_step(params, grads, moments, copies, decay, lr, step, beta1, beta2, eps, grad_scale, seed) -> code
PyObject* adamw_step(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 12, "adamw_step");
  const Items params(a[0], "params"), grads(a[1], "grads", params.count), moments(a[2], "moments", params.count);
  const int64_t tensors = params.count;
  const bool copied = a[3] != Py_None, same_decay = PyFloat_Check(a[4]) || PyLong_Check(a[4]);
  const Items copies(copied ? a[3] : params.items(), "copies", tensors), decay(same_decay ? params.items() : a[4], "weight_decay", tensors);
  Many many;
  many.expect(tensors + 3, 6 * tensors);
  std::vector<moc_adamw_tensor> list((size_t)tensors);
  for (int64_t i = 0; i < tensors; ++i) {
    moc_adamw_tensor& t = list[(size_t)i];
    t = {};
    const at::Tensor p = many.take(params[i], "params", i, -1, true), g = many.take(grads[i], "grads", i, p.numel(), false);
    if (p.sizes() != g.sizes()) bad(item("grads", i).c_str(), "of params' shape expected");
    t.param_type = type_of(p.scalar_type(), "params");
    t.grad_type = type_of(g.scalar_type(), "grads");
    t.param = p.data_ptr();
    t.grad = g.data_ptr();
    t.count = p.numel();
    const Pair pair = moments_of(moments[i], i, t.count, many, true);
    t.m = pair.m.data_ptr();
    t.v = pair.v.data_ptr();
    t.moment_type = pair.type;
    if (pair.type == MOC_E4M3) {
      t.m_scales = static_cast<uint8_t*>(pair.m_scales.data_ptr());
      t.v_scales = static_cast<uint8_t*>(pair.v_scales.data_ptr());
    }
    if (copied && copies[i] != Py_None) {
      const at::Tensor c = many.take(copies[i], "copies", i, t.count, true);
      if (p.sizes() != c.sizes()) bad(item("copies", i).c_str(), "of params' shape expected");
      t.copy_type = type_of(c.scalar_type(), "copies");
      if (t.copy_type == MOC_F32) bad(item("copies", i).c_str(), "float16 or bfloat16 expected");
      t.copy = c.data_ptr();
    }
    const double d = number(same_decay ? a[4] : decay[i]);
    if (!(d >= 0.0)) bad("weight_decay", "a number of 0 or more expected");
    t.decay = (float)d;
  }
  moc_adamw_rule rule = {};
  rule.lr_at = on_device<float>(a[5], "lr", at::kFloat, many);
  rule.step_at = on_device<int64_t>(a[6], "step", at::kLong, many);
  rule.grad_scale_at = a[10] == Py_None ? nullptr : on_device<float>(a[10], "grad_scale", at::kFloat, many);
  rule.lr = rule.lr_at ? 0.0 : number(a[5]);
  rule.step = rule.step_at ? 1 : PyLong_AsLongLong(a[6]);
  if (rule.step == -1 && PyErr_Occurred()) throw python_error();
  rule.grad_scale = a[10] == Py_None || rule.grad_scale_at ? 1.0 : number(a[10]);
  rule.beta1 = number(a[7]);
  rule.beta2 = number(a[8]);
  rule.eps = number(a[9]);
  rule.seed = PyLong_AsUnsignedLongLongMask(a[11]);
  if (PyErr_Occurred()) throw python_error();
  if (tensors == 0) return PyLong_FromLong(MOC_OK);
  many.check("adamw_step");
  void* const stream = stream_for(many.like);
  const int code = released([&] { return calls.adamw_step(tensors, list.data(), &rule, stream); });
  many.written(code);
  return PyLong_FromLong(code);
  END_HANDLE_TH_ERRORS
}

// moments_read(moments, dtype, out) -> (code, [(m, v)..])
PyObject* moments_read(PyObject*, PyObject* const* a, Py_ssize_t count) {
  HANDLE_TH_ERRORS
  arguments(count, 3, "moments_read");
  const Items moments(a[0], "moments"), out(a[2] == Py_None ? moments.items() : a[2], "out", moments.count);
  Many many;
  many.expect(4 * moments.count, 2 * moments.count);
  std::vector<moc_moments_tensor> list((size_t)moments.count);
  THPObjectPtr results(PyList_New(moments.count));
  if (!results) throw python_error();
  for (int64_t i = 0; i < moments.count; ++i) {
    moc_moments_tensor& t = list[(size_t)i];
    t = {};
    const Pair pair = moments_of(moments[i], i, -1, many, false);
    t.m = pair.m.data_ptr();
    t.v = pair.v.data_ptr();
    t.count = pair.m.numel();
    t.moment_type = pair.type;
    if (pair.type == MOC_E4M3) {
      t.m_scales = static_cast<const uint8_t*>(pair.m_scales.data_ptr());
      t.v_scales = static_cast<const uint8_t*>(pair.v_scales.data_ptr());
    }
    THPObjectPtr made;
    if (a[2] == Py_None) {
      const at::ScalarType type = dtype_of(a[1], at::kFloat);
      made = THPObjectPtr(PyTuple_Pack(2, wrapped(room_for(pair.m, type, pair.m.sizes())).get(), wrapped(room_for(pair.m, type, pair.m.sizes())).get()));
      if (!made) throw python_error();
    } else {
      Py_INCREF(out[i]);
      made = THPObjectPtr(out[i]);
    }
    const Items two(made, "out", 2);
    const at::Tensor m = many.take(two[0], "out", i, t.count, true), v = many.take(two[1], "out", i, t.count, true);
    if (m.scalar_type() != v.scalar_type()) bad(item("out", i).c_str(), "tensors of one type expected");
    t.value_type = type_of(m.scalar_type(), "out");
    t.m_values = m.data_ptr();
    t.v_values = v.data_ptr();
    PyList_SET_ITEM(results.get(), i, made.release());
  }
  if (moments.count == 0) return Py_BuildValue("iN", MOC_OK, results.release());
  many.check("moments_read");
  void* const stream = stream_for(many.like);
  const int code = released([&] { return calls.moments_read(moments.count, list.data(), stream); });
  if (a[2] != Py_None) many.written(code);
  return Py_BuildValue("iN", code, results.release());
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
  take(c.residual_forward, "moc_residual_forward");
  take(c.residual_backward, "moc_residual_backward");
  take(c.residual_backward_work, "moc_residual_backward_work");
  take(c.logprob_forward_work, "moc_logprob_forward_work");
  take(c.logprob_forward, "moc_logprob_forward");
  take(c.logprob_backward, "moc_logprob_backward");
  take(c.adamw_step, "moc_adamw_step");
  take(c.moments_read, "moc_moments_read");
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
                         MOC_METHOD(linear_backward_input), MOC_METHOD(linear_backward_weight), MOC_METHOD(residual_forward), MOC_METHOD(residual_backward), MOC_METHOD(logprob_forward), MOC_METHOD(logprob_backward), MOC_METHOD(adamw_step), MOC_METHOD(moments_read), MOC_METHOD(shares), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_training", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// training_version: of the header that this was built with.
PyMODINIT_FUNC PyInit__training() {
  name_codes = PyUnicode_InternFromString("codes");
  name_scales = PyUnicode_InternFromString("scales");
  name_fmt = PyUnicode_InternFromString("fmt");
  name_m = PyUnicode_InternFromString("m");
  name_v = PyUnicode_InternFromString("v");
  name_m_scales = PyUnicode_InternFromString("m_scales");
  name_v_scales = PyUnicode_InternFromString("v_scales");
  PyObject* const made = name_codes && name_scales && name_fmt && name_m && name_v && name_m_scales && name_v_scales ? PyModule_Create(&module) : nullptr;
  if (made && PyModule_AddIntConstant(made, "training_version", MOC_TRAINING_VERSION) != 0) {
    Py_DECREF(made);
    return nullptr;
  }
  return made;
}
