// Argument marshalling for the calls on lists of gradients, on activations and on losses: checks torch tensors,
// makes the outputs and the scratch memory, and hands addresses and layouts to the C ABI
// (include/efcp.h) on the current stream.  The same in Python takes longer than the kernels of a
// small model: 23 us a call, 7 to 10 here, 3 to 10 on the device.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/InferenceMode.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <map>
#include <optional>
#include <utility>
#include <vector>

#include "efcp.h"

namespace {

// A refusal, raised as the Python exception of that kind.
struct Refused {
  PyObject* kind;
  std::string what;
};
[[noreturn]] void refuse(PyObject* kind, const std::string& what) { throw Refused{kind, what}; }
void require(bool ok, const char* what) {
  if (!ok) refuse(PyExc_ValueError, what);
}
struct PythonError {};  // one is set already

// No C++ exception leaves a function of this module.
template <class F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const PythonError&) {
  } catch (const Refused& r) {
    PyErr_SetString(r.kind, r.what.c_str());
  } catch (const c10::OutOfMemoryError& e) {
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* kind = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    PyErr_Clear();
    PyErr_SetString(kind ? kind : PyExc_RuntimeError, e.what_without_backtrace());
    Py_XDECREF(kind);
    Py_XDECREF(torch);
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

int dtype_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return EFCP_F32;
    case at::kBFloat16: return EFCP_BF16;
    case at::kHalf: return EFCP_F16;
    default: return -1;
  }
}

const at::Tensor& tensor_of(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(PyExc_TypeError, std::string(name) + ": a tensor expected");
  return THPVariable_Unpack(o);
}
// None: an empty optional
std::optional<at::Tensor> maybe_tensor(PyObject* o, const char* name) {
  if (o == Py_None) return std::nullopt;
  return tensor_of(o, name);
}

// Runs with the tensor's device current and knows its current stream.
struct Place {
  c10::cuda::CUDAGuard guard;
  c10::cuda::CUDAStream stream;
  explicit Place(c10::Device d)
      : guard(d), stream(c10::cuda::getCurrentCUDAStream(d.index())) {}

  // An output, without the way through the operators' dispatch (a call makes up to four).
  at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type = at::kFloat) const {
    return at::detail::empty_cuda(sizes, type, stream.device(), std::nullopt);
  }
  // Scratch memory until the end of the call, in the stream's order like a tensor's.
  c10::DataPtr scratch(int64_t bytes) const {
    return c10::cuda::CUDACachingAllocator::get()->allocate(size_t(bytes));
  }
};

// ------------------------------------------------------------------ lists of gradients
enum class Use { kRead, kWrite, kGather };

// One entry of the list: a tensor on `device`, or the number of elements of an absent gradient.
void describe(PyObject* o, c10::Device device, Use use, Py_ssize_t i, efcp_tensor* out) {
  const auto at = [&] { return "entry " + std::to_string(i) + ": "; };
  if (!THPVariable_Check(o)) {
    if (use != Use::kGather || !PyLong_Check(o))
      refuse(PyExc_TypeError, at() + (use == Use::kGather ? "a tensor or an element count expected"
                                                           : "a tensor expected"));
    const long long n = PyLong_AsLongLong(o);
    if (n == -1 && PyErr_Occurred()) throw PythonError{};
    out->data = nullptr;
    out->numel = n;
    out->dtype = EFCP_F32;
    out->rank = 0;
    return;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.layout() != at::kStrided || t.device() != device)
    refuse(PyExc_ValueError, at() + "a dense tensor on " + device.str() + " expected");
  out->dtype = dtype_of(t);
  if (out->dtype < 0) refuse(PyExc_ValueError, at() + "fp32, bfloat16 or fp16 expected");
  if (t.is_neg()) refuse(PyExc_ValueError, at() + "a lazily negated view");
  out->numel = t.numel();
  out->rank = 0;
  out->data = nullptr;
  if (!out->numel) return;
  if (use == Use::kWrite) {
    if (t.is_inference() && !c10::InferenceMode::is_enabled())
      refuse(PyExc_RuntimeError, at() + "an inference tensor changed outside of inference mode");
    out->data = t.mutable_data_ptr();
  } else {
    out->data = const_cast<void*>(t.const_data_ptr());
  }
  if (!t.is_contiguous()) {
    const int64_t nd = t.dim();
    if (nd > EFCP_MAX_RANK) refuse(PyExc_ValueError, at() + "too many dimensions");
    out->rank = int32_t(nd);
    for (int64_t k = 0; k < nd; ++k) {
      out->size[k] = t.size(k);
      out->stride[k] = t.stride(k);
    }
  }
}

// Autograd's record of a change in place, once the call has succeeded.  (Inference tensors have none.)
void written(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void written(const std::optional<at::Tensor>& t) {
  if (t) written(*t);
}

// The list's device: that of `first` if given, else of its first tensor, else the current one.
c10::Device list_device(PyObject* seq, const std::optional<at::Tensor>& first) {
  if (!PyList_Check(seq) && !PyTuple_Check(seq))
    refuse(PyExc_TypeError, "a list or tuple of tensors expected");
  c10::Device d(c10::kCUDA, 0);
  bool found = false;
  if (first) {
    d = first->device();
    found = true;
  }
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
  PyObject** items = PySequence_Fast_ITEMS(seq);
  for (Py_ssize_t i = 0; i < n && !found; ++i) {
    if (THPVariable_Check(items[i])) {
      d = THPVariable_Unpack(items[i]).device();
      found = true;
    }
  }
  if (!found) d = c10::Device(c10::kCUDA, c10::cuda::current_device());
  require(d.is_cuda(), "CUDA tensors expected");
  return d;
}

std::vector<efcp_tensor> describe_list(PyObject* seq, c10::Device device, Use use) {
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
  PyObject** items = PySequence_Fast_ITEMS(seq);
  std::vector<efcp_tensor> out{size_t(n)};
  for (Py_ssize_t i = 0; i < n; ++i) describe(items[i], device, use, i, &out[size_t(i)]);
  return out;
}

// Scratch memory for the list calls on one stream; a graph being captured gets its own, since it may be
// replayed on any stream.  (Never freed: streams live as long as the process.)
at::Tensor list_workspace(const Place& place) {
  static const int64_t bytes = efcp_grads_workspace_bytes();
  const auto fresh = [&] {
    return at::zeros({bytes}, at::TensorOptions().dtype(at::kByte).device(place.stream.device()));
  };
  if (c10::cuda::currentStreamCaptureStatusMayInitCtx() != c10::cuda::CaptureStatus::None)
    return fresh();
  static auto* known = new std::map<std::pair<int, void*>, at::Tensor>;  // (under the GIL)
  at::Tensor& ws = (*known)[{place.stream.device_index(), place.stream.stream()}];
  if (!ws.defined()) ws = fresh();
  return ws;
}

at::Tensor norm_out(const std::optional<at::Tensor>& out, const Place& place) {
  if (!out) return place.empty({});
  require(out->scalar_type() == at::kFloat && out->numel() == 1 &&
              out->device() == place.stream.device(),
          "out: one fp32 value on the gradients' device expected");
  return *out;
}

// A tensor, or the EFCP_* code of the call when it is not EFCP_OK.
PyObject* result(int rc, const at::Tensor& t) {
  return rc == EFCP_OK ? THPVariable_Wrap(t) : PyLong_FromLong(rc);
}

PyObject* grads_norm(PyObject*, PyObject* args) {
  PyObject *seq, *out_;
  float scale;
  if (!PyArg_ParseTuple(args, "OfO", &seq, &scale, &out_)) return nullptr;
  return guarded([&] {
    const auto out = maybe_tensor(out_, "out");
    const Place place(list_device(seq, out));
    const auto list = describe_list(seq, place.stream.device(), Use::kRead);
    const at::Tensor norm = norm_out(out, place), ws = list_workspace(place);
    const int rc = efcp_grads_norm(list.data(), int32_t(list.size()), scale,
                                   norm.mutable_data_ptr<float>(), ws.mutable_data_ptr(),
                                   place.stream.stream());
    if (rc == EFCP_OK) written(out);
    return result(rc, norm);
  });
}

PyObject* grads_clip(PyObject*, PyObject* args) {
  PyObject *seq, *out_;
  float max_norm, scale;
  if (!PyArg_ParseTuple(args, "OffO", &seq, &max_norm, &scale, &out_)) return nullptr;
  return guarded([&] {
    const auto out = maybe_tensor(out_, "out");
    const Place place(list_device(seq, out));
    const auto list = describe_list(seq, place.stream.device(), Use::kWrite);
    const at::Tensor norm = norm_out(out, place), ws = list_workspace(place);
    const int rc = efcp_grads_clip(list.data(), int32_t(list.size()), max_norm, scale,
                                   norm.mutable_data_ptr<float>(), ws.mutable_data_ptr(),
                                   place.stream.stream());
    if (rc == EFCP_OK) {
      for (Py_ssize_t i = 0; i < Py_ssize_t(list.size()); ++i)
        if (list[size_t(i)].numel) written(THPVariable_Unpack(PySequence_Fast_GET_ITEM(seq, i)));
      written(out);
    }
    return result(rc, norm);
  });
}

PyObject* grads_gather(PyObject*, PyObject* args) {
  PyObject *seq, *flat_, *out_;
  float max_norm, scale;
  int want;
  if (!PyArg_ParseTuple(args, "OOffpO", &seq, &flat_, &max_norm, &scale, &want, &out_))
    return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor& flat = tensor_of(flat_, "flat");
    const auto out = maybe_tensor(out_, "out");
    const Place place(list_device(seq, flat));
    require(flat.scalar_type() == at::kFloat && flat.is_contiguous(),
            "flat: a contiguous fp32 tensor expected");
    const auto list = describe_list(seq, place.stream.device(), Use::kGather);
    at::Tensor norm, ws;
    if (want || out) norm = norm_out(out, place);
    if (norm.defined() || max_norm > 0.f) ws = list_workspace(place);
    const int rc = efcp_grads_gather(
        list.data(), int32_t(list.size()), flat.mutable_data_ptr<float>(), flat.numel(), max_norm,
        scale, norm.defined() ? norm.mutable_data_ptr<float>() : nullptr,
        ws.defined() ? ws.mutable_data_ptr() : nullptr, place.stream.stream());
    if (rc == EFCP_OK) {
      written(flat);
      written(out);
      if (!norm.defined()) Py_RETURN_NONE;
    }
    return result(rc, norm);
  });
}

// ------------------------------------------------------------------ group normalisation
struct Rows {
  int64_t batch, row;  // elements between samples and between positions
};

// Whether the channels of x (n, channels, *positions) lie side by side and its positions at one
// distance, and which.
std::optional<Rows> rows_of(const at::Tensor& x) {
  const int64_t channels = x.size(1);
  if (x.numel() == 0) return Rows{channels, channels};
  if (channels != 1 && x.stride(1) != 1) return std::nullopt;
  int64_t row = 0, count = 1;  // the merged positions so far, from the last dimension on
  for (int64_t k = x.dim() - 1; k >= 2; --k) {
    if (x.size(k) == 1) continue;
    if (count == 1) row = x.stride(k);
    else if (x.stride(k) != row * count) return std::nullopt;
    count *= x.size(k);
  }
  if (count == 1) row = channels;
  if (row < channels) return std::nullopt;
  return Rows{x.size(0) != 1 ? x.stride(0) : row * count, row};
}

// x itself, or a channels-last copy when its layout is another.
at::Tensor channels_last(const at::Tensor& x, Rows* rows) {
  if (const auto r = rows_of(x)) {
    *rows = *r;
    return x;
  }
  std::vector<int64_t> to{0}, back{0, x.dim() - 1};
  for (int64_t k = 2; k < x.dim(); ++k) {
    to.push_back(k);
    back.push_back(k - 1);
  }
  to.push_back(1);
  // (clone, not contiguous(): a tensor of overlapping rows may count as contiguous)
  const at::Tensor y = x.permute(to).clone(at::MemoryFormat::Contiguous).permute(back);
  *rows = *rows_of(y);
  return y;
}

// An empty channels-last tensor of x's shape and type.
at::Tensor new_channels_last(const at::Tensor& x, Rows* rows) {
  const int64_t nd = x.dim();
  std::vector<int64_t> strides(static_cast<size_t>(nd));
  int64_t step = x.size(1);
  for (int64_t k = nd - 1; k >= 2; --k) {
    strides[size_t(k)] = step;
    step *= x.size(k);
  }
  strides[0] = step;
  strides[1] = 1;
  *rows = Rows{step, x.size(1)};
  if (x.is_cuda())
    return at::detail::empty_strided_cuda(x.sizes(), strides, x.scalar_type(), x.device());
  return at::empty_strided(x.sizes(), strides, x.options());
}

efcp_group_norm group_norm_desc(const at::Tensor& x, int groups,
                                const std::optional<at::Tensor>& weight,
                                const std::optional<at::Tensor>& bias, float eps, const char* act) {
  require(x.layout() == at::kStrided && x.dim() >= 2 && dtype_of(x) >= 0 && !x.is_neg(),
          "x: (n, channels, ...) in fp32, bfloat16 or fp16 expected");
  require(x.is_cuda(), "x: a CUDA tensor expected");
  efcp_group_norm d{};
  d.act = !std::strcmp(act, "none")   ? EFCP_ACT_NONE
          : !std::strcmp(act, "relu") ? EFCP_ACT_RELU
          : !std::strcmp(act, "silu") ? EFCP_ACT_SILU
                                      : -1;
  require(d.act >= 0, "act: one of none, relu, silu expected");
  int param = -1;
  for (const auto* t : {&weight, &bias}) {
    if (!*t) continue;
    const at::Tensor& v = **t;
    const int dt = dtype_of(v);
    require(v.layout() == at::kStrided && v.device() == x.device() && dt >= 0 &&
                (param < 0 || dt == param) && v.numel() == x.size(1) && v.is_contiguous() &&
                !v.is_neg(),
            "weight, bias: contiguous, one value per channel, one type (fp32, bfloat16 or fp16), "
            "on x's device");
    param = dt;
  }
  d.n = x.size(0);
  d.channels = x.size(1);
  d.rows = 1;
  for (int64_t k = 2; k < x.dim(); ++k) d.rows *= x.size(k);
  d.groups = groups;
  d.dtype = dtype_of(x);
  d.param_dtype = param < 0 ? EFCP_F32 : param;
  d.eps = eps;
  return d;
}

const void* data_of(const std::optional<at::Tensor>& t) {
  return t ? t->const_data_ptr() : nullptr;
}

PyObject* wrap_or_none(const at::Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}

PyObject* triple(int rc, const at::Tensor& a, const at::Tensor& b, const at::Tensor& c) {
  if (rc != EFCP_OK) return PyLong_FromLong(rc);
  return Py_BuildValue("(NNN)", wrap_or_none(a), wrap_or_none(b), wrap_or_none(c));
}

PyObject* group_norm_forward(PyObject*, PyObject* args) {
  PyObject *x_, *w_, *b_;
  int groups;
  float eps;
  const char* act;
  if (!PyArg_ParseTuple(args, "OiOOfs", &x_, &groups, &w_, &b_, &eps, &act)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor& given = tensor_of(x_, "x");
    const auto weight = maybe_tensor(w_, "weight"), bias = maybe_tensor(b_, "bias");
    efcp_group_norm d = group_norm_desc(given, groups, weight, bias, eps, act);
    const Place place(given.device());
    const int64_t bytes = efcp_group_norm_workspace_bytes(&d, false);
    if (bytes < 0) return PyLong_FromLong(EFCP_EINVAL);
    const c10::DataPtr ws = place.scratch(bytes);
    Rows in, out;
    const at::Tensor x = channels_last(given, &in), y = new_channels_last(x, &out);
    d.x_batch = in.batch;
    d.x_row = in.row;
    d.y_batch = out.batch;
    d.y_row = out.row;
    const at::Tensor mean = place.empty({d.n, groups});
    const at::Tensor rstd = place.empty({d.n, groups});
    const int rc = efcp_group_norm_forward(
        &d, x.const_data_ptr(), data_of(weight), data_of(bias), y.mutable_data_ptr(),
        mean.mutable_data_ptr<float>(), rstd.mutable_data_ptr<float>(), ws.get(), bytes,
        place.stream.stream());
    return triple(rc, y, mean, rstd);
  });
}

PyObject* group_norm_backward(PyObject*, PyObject* args) {
  PyObject *dy_, *x_, *m_, *r_, *w_, *b_;
  int groups;
  const char* act;
  if (!PyArg_ParseTuple(args, "OOOOiOOs", &dy_, &x_, &m_, &r_, &groups, &w_, &b_, &act))
    return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor &given = tensor_of(x_, "x"), &given_dy = tensor_of(dy_, "dy");
    const at::Tensor &mean = tensor_of(m_, "mean"), &rstd = tensor_of(r_, "rstd");
    const auto weight = maybe_tensor(w_, "weight"), bias = maybe_tensor(b_, "bias");
    efcp_group_norm d = group_norm_desc(given, groups, weight, bias, 0.f, act);
    require(given_dy.layout() == at::kStrided && given_dy.sizes() == given.sizes() &&
                given_dy.scalar_type() == given.scalar_type() &&
                given_dy.device() == given.device() && !given_dy.is_neg(),
            "dy: x's shape, type and device expected");
    for (const at::Tensor* t : {&mean, &rstd})
      require(t->scalar_type() == at::kFloat && t->numel() == d.n * groups && t->is_contiguous() &&
                  t->device() == given.device(),
              "mean, rstd: as group_norm_forward returned them");
    const Place place(given.device());
    const int64_t bytes = efcp_group_norm_workspace_bytes(&d, true);
    if (bytes < 0) return PyLong_FromLong(EFCP_EINVAL);
    const c10::DataPtr ws = place.scratch(bytes);
    Rows in, grad, out;
    const at::Tensor x = channels_last(given, &in), dy = channels_last(given_dy, &grad);
    const at::Tensor dx = new_channels_last(x, &out);
    d.x_batch = in.batch;
    d.x_row = in.row;
    d.dy_batch = grad.batch;
    d.dy_row = grad.row;
    d.y_batch = out.batch;
    d.y_row = out.row;
    const at::Tensor dw = weight ? place.empty(weight->sizes(), weight->scalar_type()) : at::Tensor();
    const at::Tensor db = bias ? place.empty(bias->sizes(), bias->scalar_type()) : at::Tensor();
    const int rc = efcp_group_norm_backward(
        &d, dy.const_data_ptr(), x.const_data_ptr(), mean.const_data_ptr<float>(),
        rstd.const_data_ptr<float>(), data_of(weight), data_of(bias), dx.mutable_data_ptr(),
        dw.defined() ? dw.mutable_data_ptr() : nullptr,
        db.defined() ? db.mutable_data_ptr() : nullptr, ws.get(), bytes,
        place.stream.stream());
    return triple(rc, dx, dw, db);
  });
}

// ------------------------------------------------------------------ rows: RMS norm, dropout
// t itself, or a contiguous copy, as rows of its last dimension `row` elements apart.
at::Tensor as_rows(const at::Tensor& t, int64_t* row) {
  const int64_t d = t.size(-1);
  *row = d;
  if (t.is_contiguous()) return t;
  bool ok = t.numel() > 0 && (d == 1 || t.stride(-1) == 1);
  int64_t count = 1;  // the merged dimensions so far, from the last but one on
  for (int64_t k = t.dim() - 2; ok && k >= 0; --k) {
    if (t.size(k) == 1) continue;
    if (count == 1) *row = t.stride(k);
    else ok = t.stride(k) == *row * count;
    count *= t.size(k);
  }
  if (ok) return t;
  *row = d;
  return t.clone(at::MemoryFormat::Contiguous);
}

void require_like(const at::Tensor& t, const at::Tensor& x, const char* what) {
  require(t.layout() == at::kStrided && t.sizes() == x.sizes() &&
              t.scalar_type() == x.scalar_type() && t.device() == x.device() && !t.is_neg(),
          what);
}

efcp_rms_norm rms_desc(const at::Tensor& x, const char* name) {
  if (!(x.layout() == at::kStrided && x.dim() >= 1 && dtype_of(x) >= 0 && !x.is_neg()))
    refuse(PyExc_ValueError, std::string(name) + ": (..., d) in fp32, bfloat16 or fp16 expected");
  if (!x.is_cuda()) refuse(PyExc_ValueError, std::string(name) + ": a CUDA tensor expected");
  efcp_rms_norm d{};
  d.d = x.size(-1);
  d.rows = 1;
  for (int64_t k = 0; k + 1 < x.dim(); ++k) d.rows *= x.size(k);
  d.dtype = dtype_of(x);
  d.param_dtype = EFCP_F32;
  return d;
}

void rms_weight(const std::optional<at::Tensor>& weight, const at::Tensor& x, efcp_rms_norm* d) {
  if (!weight) return;
  const int dt = dtype_of(*weight);
  require(weight->layout() == at::kStrided && weight->device() == x.device() && dt >= 0 &&
              weight->numel() == d->d && weight->is_contiguous() && !weight->is_neg(),
          "weight: contiguous, one value per column, fp32, bfloat16 or fp16, on x's device");
  d->param_dtype = dt;
}

// (seed, offset): two numbers, or an int64 tensor of them on x's device.  Not looked at without dropout.
void rms_drop(double p, PyObject* rng, const at::Tensor& x, efcp_rms_norm* d) {
  d->p = p;
  if (!(p > 0)) return;
  if (THPVariable_Check(rng)) {
    const at::Tensor& t = THPVariable_Unpack(rng);
    require(t.layout() == at::kStrided && t.scalar_type() == at::kLong && t.numel() == 2 &&
                t.is_contiguous() && t.device() == x.device(),
            "rng: an int64 tensor of (seed, offset) on x's device expected");
    d->rng = reinterpret_cast<const uint64_t*>(t.const_data_ptr());
    return;
  }
  if (!PyTuple_Check(rng) || PyTuple_GET_SIZE(rng) != 2 || !PyLong_Check(PyTuple_GET_ITEM(rng, 0)) ||
      !PyLong_Check(PyTuple_GET_ITEM(rng, 1)))
    refuse(PyExc_TypeError, "rng: two ints (seed, offset) or an int64 tensor of them expected");
  d->seed = PyLong_AsUnsignedLongLongMask(PyTuple_GET_ITEM(rng, 0));
  d->offset = PyLong_AsUnsignedLongLongMask(PyTuple_GET_ITEM(rng, 1));
}

PyObject* rms_norm_forward(PyObject*, PyObject* args) {
  PyObject *x_, *w_, *r_, *rng;
  float eps;
  double p;
  if (!PyArg_ParseTuple(args, "OOfOdO", &x_, &w_, &eps, &r_, &p, &rng)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor& given = tensor_of(x_, "x");
    const auto weight = maybe_tensor(w_, "weight"), residual = maybe_tensor(r_, "residual");
    efcp_rms_norm d = rms_desc(given, "x");
    d.eps = eps;
    rms_weight(weight, given, &d);
    rms_drop(p, rng, given, &d);
    if (residual) require_like(*residual, given, "residual: x's shape, type and device expected");
    const Place place(given.device());
    int64_t x_row = 0, r_row = 0;
    const at::Tensor x = as_rows(given, &x_row);
    const at::Tensor r = residual ? as_rows(*residual, &r_row) : at::Tensor();
    const at::Tensor y = place.empty(x.sizes(), x.scalar_type());
    const bool summed = residual || p > 0;
    const at::Tensor h = summed ? place.empty(x.sizes(), x.scalar_type()) : x;
    const at::Tensor rstd = place.empty(x.sizes().slice(0, size_t(x.dim() - 1)));
    const int rc = efcp_rms_norm_forward(
        &d, x.const_data_ptr(), x_row, residual ? r.const_data_ptr() : nullptr, r_row,
        data_of(weight), y.mutable_data_ptr(), summed ? h.mutable_data_ptr() : nullptr,
        rstd.mutable_data_ptr<float>(), place.stream.stream());
    return triple(rc, y, h, rstd);
  });
}

PyObject* rms_norm_quantize(PyObject*, PyObject* args) {
  PyObject *x_, *w_, *r_;
  float eps;
  int block;
  const char* format;
  if (!PyArg_ParseTuple(args, "OOfOis", &x_, &w_, &eps, &r_, &block, &format)) return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor& given = tensor_of(x_, "x");
    const auto weight = maybe_tensor(w_, "weight"), residual = maybe_tensor(r_, "residual");
    efcp_rms_norm d = rms_desc(given, "x");
    d.eps = eps;
    rms_weight(weight, given, &d);
    if (residual) require_like(*residual, given, "residual: x's shape, type and device expected");
    const bool e4m3 = !std::strcmp(format, "e4m3");
    require(e4m3 || !std::strcmp(format, "int8"), "format: one of e4m3, int8 expected");
    require(block == 0 || block == 32 || block == 64 || block == 128,
            "block: 0 (a row), 32, 64 or 128 expected");
    const Place place(given.device());
    int64_t x_row = 0, r_row = 0;
    const at::Tensor x = as_rows(given, &x_row);
    const at::Tensor r = residual ? as_rows(*residual, &r_row) : at::Tensor();
    const at::Tensor q = place.empty(x.sizes(), e4m3 ? at::kFloat8_e4m3fn : at::kChar);
    const at::Tensor h = residual ? place.empty(x.sizes(), x.scalar_type()) : x;
    std::vector<int64_t> shape(x.sizes().begin(), x.sizes().end());
    shape.back() = block ? (d.d + block - 1) / block : 1;
    const at::Tensor scales = place.empty(shape);
    const int rc = efcp_rms_norm_quantize(
        &d, e4m3 ? EFCP_E4M3 : EFCP_INT8, block, x.const_data_ptr(), x_row,
        residual ? r.const_data_ptr() : nullptr, r_row, data_of(weight), q.mutable_data_ptr(),
        scales.mutable_data_ptr<float>(), residual ? h.mutable_data_ptr() : nullptr, nullptr,
        place.stream.stream());
    return triple(rc, q, scales, h);
  });
}

PyObject* rms_norm_backward(PyObject*, PyObject* args) {
  PyObject *dy_, *h_, *r_, *w_, *dh_, *rng;
  double p;
  int want_x, want_residual, want_weight;
  if (!PyArg_ParseTuple(args, "OOOOOdOppp", &dy_, &h_, &r_, &w_, &dh_, &p, &rng, &want_x,
                        &want_residual, &want_weight))
    return nullptr;
  return guarded([&]() -> PyObject* {
    const at::Tensor &given = tensor_of(h_, "h"), &given_dy = tensor_of(dy_, "dy");
    const at::Tensor& rstd = tensor_of(r_, "rstd");
    const auto weight = maybe_tensor(w_, "weight"), given_dh = maybe_tensor(dh_, "dh");
    efcp_rms_norm d = rms_desc(given, "h");
    rms_weight(weight, given, &d);
    rms_drop(p, rng, given, &d);
    require_like(given_dy, given, "dy: h's shape, type and device expected");
    if (given_dh) require_like(*given_dh, given, "dh: h's shape, type and device expected");
    require(rstd.scalar_type() == at::kFloat && rstd.numel() == d.rows && rstd.is_contiguous() &&
                rstd.device() == given.device(),
            "rstd: as rms_norm_forward returned it");
    const Place place(given.device());
    const bool both = p > 0 && want_x && want_residual, gradient = want_x || want_residual;
    want_weight = want_weight && weight;
    c10::DataPtr ws;
    int64_t bytes = 0;
    if (want_weight) {
      bytes = efcp_rms_norm_workspace_bytes(&d);
      if (bytes < 0) return PyLong_FromLong(EFCP_EINVAL);
      ws = place.scratch(bytes);
    }
    int64_t dy_row = 0, h_row = 0, dh_row = 0;
    const at::Tensor dy = as_rows(given_dy, &dy_row), h = as_rows(given, &h_row);
    const at::Tensor dh = given_dh ? as_rows(*given_dh, &dh_row) : at::Tensor();
    const at::Tensor dx = gradient ? place.empty(h.sizes(), h.scalar_type()) : at::Tensor();
    const at::Tensor dres = both ? place.empty(h.sizes(), h.scalar_type()) : dx;
    const at::Tensor dw =
        want_weight ? place.empty(weight->sizes(), weight->scalar_type()) : at::Tensor();
    const bool dropped = p > 0 && want_x;
    const int rc = efcp_rms_norm_backward(
        &d, dy.const_data_ptr(), dy_row, h.const_data_ptr(), h_row,
        given_dh ? dh.const_data_ptr() : nullptr, dh_row, rstd.const_data_ptr<float>(),
        data_of(weight), gradient && (dropped || p <= 0) ? dx.mutable_data_ptr() : nullptr,
        gradient && p > 0 && want_residual ? dres.mutable_data_ptr() : nullptr,
        dw.defined() ? dw.mutable_data_ptr() : nullptr, ws.get(), bytes, place.stream.stream());
    return triple(rc, want_x ? dx : at::Tensor(), want_residual ? dres : at::Tensor(), dw);
  });
}

PyObject* dropout(PyObject*, PyObject* args) {
  PyObject *x_, *rng, *r_;
  double p;
  if (!PyArg_ParseTuple(args, "OdOO", &x_, &p, &rng, &r_)) return nullptr;
  return guarded([&]() -> PyObject* {
    at::Tensor given = tensor_of(x_, "x");
    auto residual = maybe_tensor(r_, "residual");
    rms_desc(given, "x");
    if (residual) require_like(*residual, given, "residual: x's shape, type and device expected");
    // what lies in one piece is one row: the mask goes by the logical order alone
    if (given.is_contiguous() && (!residual || residual->is_contiguous())) {
      int64_t row = 1;
      while (row < 4096 && given.numel() % (2 * row) == 0) row *= 2;
      if (row < 256 && given.numel() < (1ll << 30)) row = given.numel();
      if (row >= 256) {
        given = given.view({-1, row});
        if (residual) residual = residual->view({-1, row});
      }
    }
    efcp_rms_norm d = rms_desc(given, "x");
    rms_drop(p, rng, given, &d);
    const Place place(given.device());
    int64_t x_row = 0, r_row = 0;
    const at::Tensor x = as_rows(given, &x_row);
    const at::Tensor r = residual ? as_rows(*residual, &r_row) : at::Tensor();
    const at::Tensor y = place.empty(tensor_of(x_, "x").sizes(), x.scalar_type());
    const int rc = efcp_dropout(&d, x.const_data_ptr(), x_row,
                                residual ? r.const_data_ptr() : nullptr, r_row,
                                y.mutable_data_ptr(), place.stream.stream());
    return result(rc, y);
  });
}

// ------------------------------------------------------------------ linear cross entropy
// The description of a call, with hidden and weight as rows (copied where they do not lie so).
efcp_cross_entropy xent_desc(at::Tensor* hidden, at::Tensor* weight, const at::Tensor& targets,
                             long long ignore, const char* reduction) {
  const at::Tensor &h = *hidden, &w = *weight;
  require(h.layout() == at::kStrided && h.dim() >= 1 && dtype_of(h) >= 0 && !h.is_neg(),
          "hidden: (..., d) in fp32, bfloat16 or fp16 expected");
  require(w.layout() == at::kStrided && w.dim() == 2 && w.scalar_type() == h.scalar_type() &&
              w.size(1) == h.size(-1) && w.device() == h.device() && !w.is_neg(),
          "weight: (vocabulary, d) of hidden's type and device expected");
  require(targets.layout() == at::kStrided && targets.scalar_type() == at::kLong &&
              targets.sizes() == h.sizes().slice(0, size_t(h.dim() - 1)) && targets.device() == h.device(),
          "targets: int64, one for each row of hidden, on its device expected");
  require(h.is_cuda(), "hidden: a CUDA tensor expected");
  efcp_cross_entropy d{};
  d.reduction = !std::strcmp(reduction, "none")   ? EFCP_LOSS_NONE
                : !std::strcmp(reduction, "mean") ? EFCP_LOSS_MEAN
                : !std::strcmp(reduction, "sum")  ? EFCP_LOSS_SUM
                                                  : -1;
  require(d.reduction >= 0, "reduction: one of none, mean, sum expected");
  d.tokens = targets.numel();
  d.vocab = w.size(0);
  d.d = w.size(1);
  d.dtype = dtype_of(h);
  d.ignore_index = ignore;
  const c10::cuda::CUDAGuard guard(h.device());
  *hidden = as_rows(h, &d.hidden_row);
  *weight = as_rows(w, &d.weight_row);
  return d;
}

PyObject* cross_entropy_forward(PyObject*, PyObject* args) {
  PyObject *h_, *w_, *t_;
  long long ignore;
  const char* reduction;
  if (!PyArg_ParseTuple(args, "OOOLs", &h_, &w_, &t_, &ignore, &reduction)) return nullptr;
  return guarded([&]() -> PyObject* {
    at::Tensor hidden = tensor_of(h_, "hidden"), weight = tensor_of(w_, "weight");
    const at::Tensor& given = tensor_of(t_, "targets");
    const efcp_cross_entropy d = xent_desc(&hidden, &weight, given, ignore, reduction);
    const Place place(hidden.device());
    const at::Tensor targets = given.is_contiguous() ? given : given.clone(at::MemoryFormat::Contiguous);
    const int64_t bytes = efcp_cross_entropy_workspace_bytes(&d, weight.const_data_ptr(), false);
    if (bytes < 0) return PyLong_FromLong(EFCP_EINVAL);
    const c10::DataPtr ws = place.scratch(bytes);
    const at::Tensor losses =
        d.reduction ? place.empty({}) : place.empty(targets.sizes());
    const at::Tensor lse = place.empty(targets.sizes());
    const int rc = efcp_cross_entropy_forward(
        &d, hidden.const_data_ptr(), weight.const_data_ptr(), targets.const_data_ptr<int64_t>(),
        losses.mutable_data_ptr<float>(), lse.mutable_data_ptr<float>(), ws.get(), bytes,
        place.stream.stream());
    if (rc != EFCP_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NN)", THPVariable_Wrap(losses), THPVariable_Wrap(lse));
  });
}

PyObject* cross_entropy_backward(PyObject*, PyObject* args) {
  PyObject *g_, *h_, *w_, *t_, *l_;
  long long ignore;
  const char* reduction;
  int want_hidden, want_weight;
  if (!PyArg_ParseTuple(args, "OOOOOLspp", &g_, &h_, &w_, &t_, &l_, &ignore, &reduction, &want_hidden,
                        &want_weight))
    return nullptr;
  return guarded([&]() -> PyObject* {
    at::Tensor hidden = tensor_of(h_, "hidden"), weight = tensor_of(w_, "weight");
    at::Tensor grad = tensor_of(g_, "grad");
    const at::Tensor &given = tensor_of(t_, "targets"), &lse = tensor_of(l_, "lse");
    const efcp_cross_entropy d = xent_desc(&hidden, &weight, given, ignore, reduction);
    require(grad.layout() == at::kStrided && grad.scalar_type() == at::kFloat &&
                grad.device() == hidden.device() && !grad.is_neg() &&
                (d.reduction ? grad.numel() == 1 : grad.sizes() == given.sizes()),
            "grad: fp32, one value for each loss, on hidden's device expected");
    require(lse.scalar_type() == at::kFloat && lse.numel() == d.tokens && lse.is_contiguous() &&
                lse.device() == hidden.device(),
            "lse: as cross_entropy_forward returned it");
    const Place place(hidden.device());
    const at::Tensor targets = given.is_contiguous() ? given : given.clone(at::MemoryFormat::Contiguous);
    int64_t step = 1;
    if (!grad.is_contiguous()) {
      step = 0;
      for (int64_t k = 0; k < grad.dim(); ++k) step |= grad.size(k) > 1 ? grad.stride(k) : 0;
      if (step) {
        grad = grad.clone(at::MemoryFormat::Contiguous);
        step = 1;
      }
    }
    const int64_t bytes = efcp_cross_entropy_workspace_bytes(&d, weight.const_data_ptr(), true);
    if (bytes < 0) return PyLong_FromLong(EFCP_EINVAL);
    const c10::DataPtr ws = place.scratch(bytes);
    const at::Tensor dh = want_hidden ? place.empty(hidden.sizes(), hidden.scalar_type()) : at::Tensor();
    const at::Tensor dw = want_weight ? place.empty(weight.sizes(), weight.scalar_type()) : at::Tensor();
    const int rc = efcp_cross_entropy_backward(
        &d, grad.const_data_ptr<float>(), step, hidden.const_data_ptr(), weight.const_data_ptr(),
        targets.const_data_ptr<int64_t>(), lse.const_data_ptr<float>(),
        want_hidden ? dh.mutable_data_ptr() : nullptr, want_weight ? dw.mutable_data_ptr() : nullptr,
        ws.get(), bytes, place.stream.stream());
    if (rc != EFCP_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NN)", wrap_or_none(dh), wrap_or_none(dw));
  });
}

// rows_layout(x): (elements between samples, between positions), or None when a copy would be made;
// as_channels_last(x): x or that copy; like_channels_last(x): an empty output for x.  What the calls
// above do to layouts, on tensors of any device.
PyObject* rows_layout(PyObject*, PyObject* x) {
  return guarded([&]() -> PyObject* {
    const auto r = rows_of(tensor_of(x, "x"));
    if (!r) Py_RETURN_NONE;
    return Py_BuildValue("(LL)", (long long)r->batch, (long long)r->row);
  });
}
PyObject* as_channels_last(PyObject*, PyObject* x) {
  return guarded([&] {
    Rows r;
    return THPVariable_Wrap(channels_last(tensor_of(x, "x"), &r));
  });
}
PyObject* like_channels_last(PyObject*, PyObject* x) {
  return guarded([&] {
    Rows r;
    return THPVariable_Wrap(new_channels_last(tensor_of(x, "x"), &r));
  });
}

PyMethodDef methods[] = {
    {"grads_norm", grads_norm, METH_VARARGS, "efcp_grads_norm"},
    {"grads_clip", grads_clip, METH_VARARGS, "efcp_grads_clip"},
    {"grads_gather", grads_gather, METH_VARARGS, "efcp_grads_gather"},
    {"group_norm_forward", group_norm_forward, METH_VARARGS, "efcp_group_norm_forward"},
    {"group_norm_backward", group_norm_backward, METH_VARARGS, "efcp_group_norm_backward"},
    {"rms_norm_forward", rms_norm_forward, METH_VARARGS, "efcp_rms_norm_forward"},
    {"rms_norm_backward", rms_norm_backward, METH_VARARGS, "efcp_rms_norm_backward"},
    {"rms_norm_quantize", rms_norm_quantize, METH_VARARGS, "efcp_rms_norm_quantize"},
    {"dropout", dropout, METH_VARARGS, "efcp_dropout"},
    {"cross_entropy_forward", cross_entropy_forward, METH_VARARGS, "efcp_cross_entropy_forward"},
    {"cross_entropy_backward", cross_entropy_backward, METH_VARARGS, "efcp_cross_entropy_backward"},
    {"rows_layout", rows_layout, METH_O, "strides of samples and positions, or None"},
    {"as_channels_last", as_channels_last, METH_O, "the tensor, or a channels-last copy"},
    {"like_channels_last", like_channels_last, METH_O, "an empty channels-last tensor"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
