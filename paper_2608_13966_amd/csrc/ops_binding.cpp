// ops_binding.cpp -- the Python calls of ops.py: argument checks, output
// tensors and the C entry points of quasar_ops.h, in C++ because at the
// smallest sizes the host's side of a call is what counts.  (One token's norm
// with four outputs: 14.9 us a call through ctypes and torch's Python
// functions, most of it neither launch nor kernel.)
//
// Every function returns the dict of outputs, or the int status of a call that
// the library refused; ops.py raises for it.  Argument errors that the library
// cannot see (shapes, devices, types of tensors) are ValueError and TypeError.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include <ATen/ATen.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/StreamGuard.h>

#include "quasar_ops.h"

namespace py = pybind11;

namespace {

using at::Tensor;
using Maybe = std::optional<Tensor>;

py::object g_stream;        // handle of torch's current stream on a tensor's device (refuses tensors that are on no GPU)
py::object g_torch_stream;  // torch's stream of a handle and a device

std::string shape_str(at::IntArrayRef s) {
  std::string r = "(";
  for (size_t i = 0; i < s.size(); i++) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + (s.size() == 1 ? ",)" : ")");
}

// fp32 or bf16; the dtype code
int code(const Tensor& t, const char* what) {
  if (t.scalar_type() == at::kBFloat16) return QUASAR_BF16;
  if (t.scalar_type() == at::kFloat) return QUASAR_F32;
  TORCH_CHECK_TYPE(false, what, ": unsupported dtype ", t.dtype());
}

const Tensor& matrix(const Tensor& t, const char* what, int64_t rows, int64_t cols, const at::Device& dev) {
  TORCH_CHECK_VALUE(t.dim() == 2 && t.size(0) == rows && t.size(1) == cols, what, " must be a tensor of shape (", rows,
                    ", ", cols, "), not ", shape_str(t.sizes()));
  TORCH_CHECK_VALUE(t.device() == dev, what, " is on ", t.device(), ", not on ", dev);
  TORCH_CHECK_VALUE(t.stride(1) == 1 || cols == 1 || rows == 0, what, ": the last dimension must have unit stride");
  return t;
}

const Tensor& vector(const Tensor& t, const char* what, int64_t n, const at::Device& dev) {
  TORCH_CHECK_VALUE(t.dim() == 1 && t.size(0) == n && t.device() == dev && t.is_contiguous(), what,
                    " must be a contiguous tensor of ", n, " elements on ", dev);
  return t;
}
const Tensor& vector_f32(const Tensor& t, const char* what, int64_t n, const at::Device& dev) {
  TORCH_CHECK_VALUE(t.scalar_type() == at::kFloat, what, " must be float32, not ", t.dtype());
  return vector(t, what, n, dev);
}

Tensor fresh(at::IntArrayRef shape, at::ScalarType type, const at::Device& dev) {
  return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
}

// The buffer of one output: out's, which has to be one of this shape and type, or without an out a new one.
Tensor result(const py::object& out, const char* name, at::IntArrayRef shape, at::ScalarType type, const at::Device& dev) {
  if (out.is_none()) return fresh(shape, type, dev);
  py::object v = out.attr("get")(name);
  TORCH_CHECK_VALUE(!v.is_none() && THPVariable_Check(v.ptr()), "out['", name, "'] must be a tensor");
  Tensor t = THPVariable_Unpack(v.ptr());
  TORCH_CHECK_VALUE(t.sizes() == shape && t.scalar_type() == type && t.device() == dev, "out['", name, "'] must be a ",
                    type, " tensor of shape ", shape_str(shape), " on ", dev);
  if (shape.size() == 1) {
    TORCH_CHECK_VALUE(t.is_contiguous(), "out['", name, "'] must be contiguous");
  } else {
    TORCH_CHECK_VALUE(t.stride(1) == 1 || shape[1] == 1, "out['", name, "'] must have unit stride in its last dimension");
    TORCH_CHECK_VALUE(t.stride(0) >= shape[1] || shape[0] <= 1, "out['", name, "']: its rows overlap");
  }
  return t;
}

Maybe workspace(const py::object& out, size_t bytes, const at::Device& dev) {
  if (bytes == 0) return std::nullopt;
  if (!out.is_none()) {
    py::object v = out.attr("get")("workspace");
    if (!v.is_none() && THPVariable_Check(v.ptr())) {
      Tensor t = THPVariable_Unpack(v.ptr());
      if (t.scalar_type() == at::kByte && t.is_contiguous() && (size_t)t.numel() >= bytes && t.device() == dev) return t;
    }
  }
  return fresh({(int64_t)bytes}, at::kByte, dev);
}

void* ptr(const Tensor& t) { return t.data_ptr(); }
void* ptr(const Maybe& t) { return t ? t->data_ptr() : nullptr; }
int64_t stride(const Maybe& t) { return t ? t->stride(0) : 0; }
py::object obj(const Maybe& t) { return t ? py::cast(*t) : py::none(); }

// The device and stream of a call, current while it lasts.  The device because
// the handle of a default stream is 0 on every one: the launch would go to the
// device that is current, whatever the tensors' is.  The stream, where the
// caller names one, because what is allocated or filled on the way then belongs
// to it: memory that is freed again (a workspace, or an output that is dropped)
// goes to no other stream's work while this one's kernels use it, nor comes from
// there.
class Stream {
 public:
  Stream(const py::object& given, const at::Device& dev) : given_(given) {
    if (!dev.is_cpu()) device_.reset_device(dev);
    if (given.is_none()) return;
    TORCH_CHECK_VALUE(dev.is_cuda(), "tensors on ", dev, " with a stream: they have to be on its GPU");
    const py::object s = g_torch_stream(given, (int)dev.index());
    stream_.emplace(c10::Stream(c10::Stream::UNSAFE, dev, s.attr("stream_id").cast<c10::StreamId>()));
  }
  void* handle(const Tensor& t) const {
    return reinterpret_cast<void*>((given_.is_none() ? g_stream(t) : given_).cast<uintptr_t>());
  }

 private:
  const py::object& given_;
  c10::OptionalDeviceGuard device_;
  std::optional<c10::StreamGuard> stream_;
};

at::ScalarType type_of(int c) { return c == QUASAR_BF16 ? at::kBFloat16 : at::kFloat; }

// y_dtype, dx_dtype: a dtype code, or -1 for the default
py::object add_rms_norm(const Tensor& x, const Tensor& weight, const Maybe& residual, double eps, int y_dtype, bool want_y,
                        bool quantize, const py::object& out, const py::object& stream) {
  TORCH_CHECK_VALUE(x.dim() == 2, "add_rms_norm: x must be 2-D");
  const int64_t rows = x.size(0), cols = x.size(1);
  const at::Device dev = x.device();
  const Stream on(stream, dev);
  matrix(x, "x", rows, cols, dev);
  vector(weight, "weight", cols, dev);
  quasar_norm a{};
  a.rows = rows;
  a.cols = cols;
  a.x_dtype = code(x, "x");
  a.weight_dtype = code(weight, "weight");
  if (residual) a.residual_dtype = code(matrix(*residual, "residual", rows, cols, dev), "residual");
  Maybe h, y, q, scale;
  if (residual) h = result(out, "h", {rows, cols}, residual->scalar_type(), dev);
  const Tensor rstd = result(out, "rstd", {rows}, at::kFloat, dev);
  a.y_dtype = y_dtype < 0 ? a.x_dtype : y_dtype;
  if (want_y) y = result(out, "y", {rows, cols}, type_of(a.y_dtype), dev);
  if (quantize) {
    q = result(out, "q", {rows, cols}, at::kFloat8_e4m3fn, dev);
    scale = result(out, "scale", {rows}, at::kFloat, dev);
  }
  a.x = ptr(x);
  a.residual = ptr(residual);
  a.weight = ptr(weight);
  a.h = ptr(h);
  a.y = ptr(y);
  a.q = static_cast<uint8_t*>(ptr(q));
  a.scale = static_cast<float*>(ptr(scale));
  a.rstd = static_cast<float*>(ptr(rstd));
  a.x_stride = x.stride(0);
  a.residual_stride = stride(residual);
  a.h_stride = stride(h);
  a.y_stride = stride(y);
  a.q_stride = stride(q);
  a.eps = (float)eps;
  const int s = quasar_add_rms_norm(&a, on.handle(x));
  if (s != QUASAR_OK) return py::int_(s);
  py::dict o;
  o["h"] = h ? *h : x;
  o["rstd"] = rstd;
  o["y"] = obj(y);
  o["q"] = obj(q);
  o["scale"] = obj(scale);
  return std::move(o);
}

py::object add_rms_norm_backward(const Tensor& dy, const Tensor& h, const Tensor& weight, const Tensor& rstd, const Maybe& dh,
                                 int dx_dtype, bool want_dweight, const py::object& out, const py::object& stream) {
  TORCH_CHECK_VALUE(dy.dim() == 2, "add_rms_norm_backward: dy must be 2-D");
  const int64_t rows = dy.size(0), cols = dy.size(1);
  const at::Device dev = dy.device();
  const Stream on(stream, dev);
  matrix(dy, "dy", rows, cols, dev);
  matrix(h, "h", rows, cols, dev);
  vector(weight, "weight", cols, dev);
  vector_f32(rstd, "rstd", rows, dev);
  quasar_norm_backward a{};
  a.rows = rows;
  a.cols = cols;
  a.dy_dtype = code(dy, "dy");
  a.h_dtype = code(h, "h");
  a.weight_dtype = code(weight, "weight");
  a.dx_dtype = dx_dtype < 0 ? a.h_dtype : dx_dtype;
  if (dh) {
    const int c = code(matrix(*dh, "dh", rows, cols, dev), "dh");
    TORCH_CHECK_VALUE(dx_dtype < 0 || dx_dtype == c, "add_rms_norm_backward: dx has dh's type");
    a.dx_dtype = c;
  }
  const Tensor dx = result(out, "dx", {rows, cols}, type_of(a.dx_dtype), dev);
  Maybe dw, ws;
  if (want_dweight) {
    dw = result(out, "dw", {cols}, at::kFloat, dev);
    a.workspace_bytes = quasar_add_rms_norm_backward_workspace_bytes(rows, cols);
    ws = workspace(out, a.workspace_bytes, dev);
    if (rows == 0) dw->zero_();
  }
  a.dy = ptr(dy);
  a.h = ptr(h);
  a.weight = ptr(weight);
  a.rstd = static_cast<float*>(ptr(rstd));
  a.dh = ptr(dh);
  a.dx = ptr(dx);
  a.dweight = static_cast<float*>(ptr(dw));
  a.workspace = ptr(ws);
  a.dy_stride = dy.stride(0);
  a.h_stride = h.stride(0);
  a.dh_stride = stride(dh);
  a.dx_stride = dx.stride(0);
  const int s = quasar_add_rms_norm_backward(&a, on.handle(dy));
  if (s != QUASAR_OK) return py::int_(s);
  py::dict o;
  o["dx"] = dx;
  o["dw"] = obj(dw);
  o["workspace"] = obj(ws);
  return std::move(o);
}

// what: 0 the loss, 1 the gradient, 2 both
py::object distill(int what, const Tensor& logits, const Tensor& index, const Tensor& teacher, double temperature,
                   const Maybe& row_weight, const Maybe& saved, const Maybe& grad_loss, double grad_scale,
                   const py::object& out, const py::object& stream) {
  static const char* const names[] = {"distill_topk", "distill_topk_backward", "distill_topk_grad"};
  const char* const where = names[what];
  TORCH_CHECK_VALUE(logits.dim() == 2, where, ": logits must be 2-D");
  const int64_t rows = logits.size(0), classes = logits.size(1);
  const at::Device dev = logits.device();
  const Stream on(stream, dev);
  matrix(logits, "logits", rows, classes, dev);
  quasar_distill a{};
  a.rows = rows;
  a.classes = classes;
  a.logits_dtype = code(logits, "logits");
  TORCH_CHECK_VALUE(index.dim() == 2 && index.size(0) == rows, where, ": index must be [rows, listed]");
  const int64_t k = index.size(1);
  TORCH_CHECK_TYPE(index.scalar_type() == at::kLong || index.scalar_type() == at::kInt, "index: unsupported dtype ",
                   index.dtype());
  a.index_bits = index.scalar_type() == at::kLong ? 64 : 32;
  for (const auto* t : {&index, &teacher})
    TORCH_CHECK_VALUE(t->dim() == 2 && t->size(0) == rows && t->size(1) == k && t->device() == dev && t->is_contiguous(),
                      where, ": ", t == &index ? "index" : "teacher", " must be a contiguous tensor of shape (", rows, ", ",
                      k, ") on ", dev);
  a.listed = (int32_t)std::min<int64_t>(k, INT32_MAX);
  a.teacher_dtype = code(teacher, "teacher");
  if (row_weight) vector_f32(*row_weight, "row_weight", rows, dev);
  Maybe loss, lse, grad, ws;
  if (what == 1) {
    TORCH_CHECK_TYPE(saved, where, ": lse must be a tensor, not None");
    lse = vector_f32(*saved, "lse", rows, dev);
    if (grad_loss) vector_f32(*grad_loss, "grad_loss", rows, dev);
  } else {
    loss = result(out, "loss", {rows}, at::kFloat, dev);
    lse = result(out, "lse", {rows}, at::kFloat, dev);
    a.workspace_bytes = quasar_distill_topk_workspace_bytes(rows, classes);
    ws = workspace(out, a.workspace_bytes, dev);
  }
  if (what != 0) grad = result(out, "grad", {rows, classes}, logits.scalar_type(), dev);
  a.logits = ptr(logits);
  a.index = ptr(index);
  a.teacher = ptr(teacher);
  a.row_weight = static_cast<float*>(ptr(row_weight));
  a.grad_loss = static_cast<float*>(ptr(grad_loss));
  a.loss = static_cast<float*>(ptr(loss));
  a.lse = static_cast<float*>(ptr(lse));
  a.grad = ptr(grad);
  a.workspace = ptr(ws);
  a.logits_stride = logits.stride(0);
  a.grad_stride = stride(grad);
  a.temperature = (float)temperature;
  a.grad_scale = (float)grad_scale;
  void* const st = on.handle(logits);
  const int s = what == 0   ? quasar_distill_topk(&a, st)
                : what == 1 ? quasar_distill_topk_backward(&a, st)
                            : quasar_distill_topk_grad(&a, st);
  if (s != QUASAR_OK) return py::int_(s);
  py::dict o;
  if (what != 1) {
    o["loss"] = *loss;
    o["lse"] = *lse;
  }
  if (what != 0) o["grad"] = *grad;
  o["workspace"] = obj(ws);
  return std::move(o);
}

// A packed weight: its descriptor and buffers, held as long as this is.
struct Packed {
  quasar_desc desc{};
  float clip = 1.0f;  // the descriptor's (unused) clip grid
  Tensor codes, scales;
  Maybe zeros, tensor_scale;

  Packed(int64_t rows, int64_t cols, int format, int bits, int group, Tensor c, Tensor s, Maybe z, Maybe t)
      : codes(std::move(c)), scales(std::move(s)), zeros(std::move(z)), tensor_scale(std::move(t)) {
    desc.rows = rows;
    desc.cols = cols;
    desc.w_dtype = QUASAR_BF16;
    desc.format = format;
    desc.bits = bits;
    desc.group = group;
    desc.clip_ratios = &clip;
    desc.n_clips = 1;
    desc.g_dtype = QUASAR_BF16;
    desc.beta2 = 0.999f;
  }
  Packed(const Packed&) = delete;
};

py::object linear_codes(const Tensor& x, const Packed& w, const Maybe& x_scale, const Maybe& bias, const Maybe& residual,
                        int act, int y_dtype, const py::object& out, const py::object& stream) {
  TORCH_CHECK_VALUE(x.dim() == 2, "linear_codes: x must be 2-D");
  const int64_t tokens = x.size(0), rows = w.desc.rows;
  const at::Device dev = w.codes.device();
  const Stream on(stream, dev);
  matrix(x, "x", tokens, w.desc.cols, dev);
  quasar_linear a{};
  a.tokens = tokens;
  TORCH_CHECK_TYPE(x.scalar_type() == at::kBFloat16 || x.scalar_type() == at::kFloat8_e4m3fn, "x: unsupported dtype ",
                   x.dtype());
  a.x_dtype = x.scalar_type() == at::kBFloat16 ? QUASAR_BF16 : QUASAR_E4M3;
  if (x_scale) vector_f32(*x_scale, "x_scale", tokens, dev);
  if (bias) a.bias_dtype = code(vector(*bias, "bias", rows, dev), "bias");
  if (residual) a.residual_dtype = code(matrix(*residual, "residual", tokens, rows, dev), "residual");
  if (y_dtype < 0) y_dtype = QUASAR_BF16;
  const Tensor y = result(out, "y", {tokens, rows}, type_of(y_dtype), dev);
  a.workspace_bytes = quasar_linear_codes_workspace_bytes(&w.desc, tokens, a.x_dtype);
  const Maybe ws = workspace(out, a.workspace_bytes, dev);
  a.x = ptr(x);
  a.x_scale = static_cast<float*>(ptr(x_scale));
  a.codes = static_cast<uint8_t*>(ptr(w.codes));
  a.scales = ptr(w.scales);
  a.zeros = static_cast<float*>(ptr(w.zeros));
  a.tensor_scale = static_cast<float*>(ptr(w.tensor_scale));
  a.bias = ptr(bias);
  a.residual = ptr(residual);
  a.y = ptr(y);
  a.workspace = ptr(ws);
  a.x_stride = x.stride(0);
  a.residual_stride = stride(residual);
  a.y_stride = y.stride(0);
  a.y_dtype = y_dtype;
  a.act = act;
  const int s = quasar_linear_codes(&w.desc, &a, on.handle(x));
  if (s != QUASAR_OK) return py::int_(s);
  py::dict o;
  o["y"] = y;
  o["workspace"] = obj(ws);
  return std::move(o);
}

}  // namespace

PYBIND11_MODULE(_ops_binding, m) {
  m.def("set_stream_functions", [](py::object current, py::object of_handle) {
    g_stream = std::move(current);
    g_torch_stream = std::move(of_handle);
  });
  m.def("add_rms_norm", &add_rms_norm);
  m.def("add_rms_norm_backward", &add_rms_norm_backward);
  m.def("distill", &distill);
  m.def("linear_codes", &linear_codes);
  py::class_<Packed>(m, "Packed")
      .def(py::init<int64_t, int64_t, int, int, int, Tensor, Tensor, Maybe, Maybe>());
  // released before the interpreter is
  py::module_::import("atexit").attr("register")(py::cpp_function([] { g_stream = g_torch_stream = py::object(); }));
}
