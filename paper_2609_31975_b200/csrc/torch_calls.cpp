// The Python side of the training calls: checks torch tensors, allocates what a call returns and its workspace through torch, and
// fills in the C ABI's argument structures.  In C++ because a call on a small model takes the device less time than the same steps
// take the interpreter (host time of a call, in Python / here: forward, 64 tokens, 50 / 16 us; backward 63 / 26; norm of four tensors
// 22 / 9; AdamW over 64 tensors 208 / 23).
//
// The C entry points come in as addresses (`bind`), from the library that the binding has loaded.
#include <ATen/ATen.h>
#include <ATen/Context.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>
#include <pybind11/stl.h>

#include <cmath>
#include <string>
#include <vector>

#include "sparse_ffn.h"

namespace py = pybind11;
using at::Tensor;
using OptTensor = std::optional<Tensor>;

namespace {

struct Entry {
  decltype(&sffn_train_workspace_bytes) workspace_bytes;
  decltype(&gated_ffn_forward) forward;
  decltype(&gated_ffn_backward) backward;
  decltype(&sffn_grad_norm) grad_norm;
  decltype(&sffn_adamw_step) adamw_step;
  decltype(&sffn_adamw_state_values) adamw_state_values;
  decltype(&sffn_block_norm_forward) block_forward;
  decltype(&sffn_block_norm_workspace_bytes) block_workspace_bytes;
  decltype(&sffn_block_norm_backward) block_backward;
  decltype(&sffn_orthogonalize_workspace_bytes) orthogonalize_workspace_bytes;
  decltype(&sffn_orthogonalize) orthogonalize;
  decltype(&sffn_muon_workspace_bytes) muon_workspace_bytes;
  decltype(&sffn_muon_step) muon_step;
} entry;

void bind(const std::vector<uintptr_t>& a) {
  if (a.size() != 13) throw py::value_error("thirteen addresses");
  entry.workspace_bytes = reinterpret_cast<decltype(entry.workspace_bytes)>(a[0]);
  entry.forward = reinterpret_cast<decltype(entry.forward)>(a[1]);
  entry.backward = reinterpret_cast<decltype(entry.backward)>(a[2]);
  entry.grad_norm = reinterpret_cast<decltype(entry.grad_norm)>(a[3]);
  entry.adamw_step = reinterpret_cast<decltype(entry.adamw_step)>(a[4]);
  entry.adamw_state_values = reinterpret_cast<decltype(entry.adamw_state_values)>(a[5]);
  entry.block_forward = reinterpret_cast<decltype(entry.block_forward)>(a[6]);
  entry.block_workspace_bytes = reinterpret_cast<decltype(entry.block_workspace_bytes)>(a[7]);
  entry.block_backward = reinterpret_cast<decltype(entry.block_backward)>(a[8]);
  entry.orthogonalize_workspace_bytes = reinterpret_cast<decltype(entry.orthogonalize_workspace_bytes)>(a[9]);
  entry.orthogonalize = reinterpret_cast<decltype(entry.orthogonalize)>(a[10]);
  entry.muon_workspace_bytes = reinterpret_cast<decltype(entry.muon_workspace_bytes)>(a[11]);
  entry.muon_step = reinterpret_cast<decltype(entry.muon_step)>(a[12]);
}

[[noreturn]] void type_error(const std::string& what) { throw py::type_error(what); }

std::string shape_text(at::IntArrayRef s) {
  std::string t = "[";
  for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
  return t + "]";
}
[[noreturn]] void expected(const char* name, at::IntArrayRef shape, at::ScalarType dtype, const at::Device& dev, const Tensor& t, const char* how) {
  type_error(std::string(name) + ": " + how + shape_text(shape) + " " + at::toString(dtype) + " on " + dev.str() + " expected, got " +
             shape_text(t.sizes()) + " " + at::toString(t.scalar_type()) + " on " + t.device().str());
}
void check_plain(const char* name, const Tensor& t, at::IntArrayRef shape, at::ScalarType dtype, const at::Device& dev, const char* how = "") {
  if (t.sizes() != shape || t.scalar_type() != dtype || t.device() != dev || t.layout() != at::kStrided) expected(name, shape, dtype, dev, t, how);
}
// Contiguous: its address.
void* whole(const char* name, const Tensor& t, at::IntArrayRef shape, at::ScalarType dtype, const at::Device& dev) {
  check_plain(name, t, shape, dtype, dev, "contiguous ");
  if (!t.is_contiguous()) expected(name, shape, dtype, dev, t, "contiguous ");
  return t.data_ptr();
}
// A matrix of rows at one stride, consecutive entries in a row: that stride (a single row has any).
int64_t rows(const char* name, const Tensor& t, int64_t r, int64_t c, at::ScalarType dtype, const at::Device& dev) {
  check_plain(name, t, {r, c}, dtype, dev);
  if (c > 1 && t.stride(1) != 1) type_error(std::string(name) + ": entries of a row must be consecutive");
  return r > 1 ? t.stride(0) : (c + 7) / 8 * 8;
}
int dtype_code(at::ScalarType t, const char* what) {
  if (t == at::kFloat) return SFFN_F32;
  if (t == at::kBFloat16) return SFFN_BF16;
  type_error(std::string(what) + " must be torch.float32 or torch.bfloat16");
}
void on_cuda(const Tensor& t) {
  if (!t.is_cuda()) type_error("tensors must be on a CUDA device");
}
// Straight from torch's allocator, as the way through its dispatcher takes longer than the allocation: unless something looks on there (a
// dispatch mode, a transform), or torch is to fill memory that nothing has written yet.
Tensor make(at::IntArrayRef shape, at::ScalarType dtype, const at::Device& dev) {
  const bool seen = !(c10::impl::tls_local_dispatch_key_set().included_ - c10::default_included_set).empty();
  const auto& context = at::globalContext();
  if (seen || (context.deterministicAlgorithms() && context.deterministicFillUninitializedMemory())) return at::empty(shape, at::TensorOptions().dtype(dtype).device(dev));
  return Tensor(at::detail::empty_cuda(shape, dtype, dev, std::nullopt));
}
// [T, H] with rows a multiple of 16 bytes apart.
Tensor make_hidden(int64_t T, int64_t H, at::ScalarType dtype, const at::Device& dev) {
  const int64_t ld = (H + 7) / 8 * 8;
  Tensor t = make({T, ld}, dtype, dev);
  return ld == H ? t : t.narrow(1, 0, H);
}
// Torch's graph is to know of what a call has written into a caller's tensor, as of its own operations in place: a backward pass that
// saved it before then raises.  (Tensors made in inference mode are not in any graph, and count nothing.)
void written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void* current_stream(const at::Device& dev) { return c10::cuda::getCurrentCUDAStream(dev.index()).stream(); }

bool capturing() { return c10::cuda::currentStreamCaptureStatusMayInitCtx() != c10::cuda::CaptureStatus::None; }

// A zeroed buffer that outlives a call.  It comes from a stream of its own, and is there, zeroed, when this returns: the calls that use it
// may be on any stream, and one that is being captured leaves neither the buffer nor its zeros to the graph.
Tensor kept(int64_t bytes, int index) {
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)index);
  const c10::cuda::CUDAStreamCaptureModeGuard relaxed(cudaStreamCaptureModeRelaxed);
  for (int i = 0; i < 64; ++i) {  // torch hands out its streams in turn: not one that is being captured
    const c10::cuda::CUDAStreamGuard on(c10::cuda::getStreamFromPool(false, (c10::DeviceIndex)index));
    if (capturing()) continue;
    const Tensor t = at::zeros({bytes}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, index));
    on.current_stream().synchronize();
    return t;
  }
  throw std::runtime_error("every stream is being captured");
}

// What both passes hand over; the workspace in `ws`.
sffn_train_call make_call(const Tensor& x, const Tensor& W_g, const Tensor& W_up, const Tensor& W_down, int act, int act_up, const Tensor& status, bool backward,
                          Tensor& ws, int* rc) {
  if (x.dim() != 2 || W_g.dim() != 2) type_error("x is [T, D], weights are [H, D]");
  const at::Device dev = x.device();
  const at::ScalarType dtype = W_g.scalar_type();
  const int64_t T = x.size(0), D = x.size(1), H = W_g.size(0);
  if (T > INT32_MAX || D > INT32_MAX || H > INT32_MAX) type_error("sizes beyond 32 bits");
  sffn_train_call c{};
  c.T = (int32_t)T; c.D = (int32_t)D; c.H = (int32_t)H;
  c.dtype = dtype_code(dtype, "weights");
  c.act = act; c.act_up = act_up;
  c.ld_x = rows("x", x, T, D, dtype, dev);
  c.x = x.data_ptr();
  c.W_g = whole("W_g", W_g, {H, D}, dtype, dev);
  c.W_up = whole("W_up", W_up, {H, D}, dtype, dev);
  c.W_down = whole("W_down", W_down, {H, D}, dtype, dev);
  c.status = static_cast<int32_t*>(status.data_ptr());
  size_t bytes = 0;
  *rc = entry.workspace_bytes(c.T, c.D, c.H, c.dtype, backward, &bytes);
  if (*rc == SFFN_OK) {
    ws = make({(int64_t)bytes}, at::kByte, dev);  // torch's blocks start on 512 bytes
    c.workspace = ws.data_ptr();
    c.workspace_bytes = bytes;
  }
  return c;
}

py::tuple ffn_forward(const Tensor& x, const Tensor& W_g, const OptTensor& b_g, const Tensor& W_up, const Tensor& W_down, int act, int act_up, bool save,
                      const OptTensor& y_out, const OptTensor& z_out, const OptTensor& u_out, const Tensor& status) {
  on_cuda(x);
  const c10::cuda::CUDAGuard guard(x.device());
  const at::Device dev = x.device();
  Tensor ws;
  int rc = 0;
  sffn_train_call c = make_call(x, W_g, W_up, W_down, act, act_up, status, false, ws, &rc);
  const at::ScalarType dtype = W_g.scalar_type();
  if (b_g) c.b_g = static_cast<const float*>(whole("b_g", *b_g, {c.H}, at::kFloat, dev));
  const Tensor y = y_out ? *y_out : make({c.T, c.D}, dtype, dev);
  const int64_t ld_y = rows("y", y, c.T, c.D, dtype, dev);
  if (!save) {
    if (rc == SFFN_OK) rc = entry.forward(&c, y.data_ptr(), ld_y, current_stream(dev));
    if (rc == SFFN_OK && y_out) written(y);
    return py::make_tuple(rc, y, py::none(), py::none());
  }
  const Tensor z = z_out ? *z_out : make_hidden(c.T, c.H, dtype, dev), u = u_out ? *u_out : make_hidden(c.T, c.H, dtype, dev);
  c.ld_hidden = rows("z", z, c.T, c.H, dtype, dev);
  if (rows("u", u, c.T, c.H, dtype, dev) != c.ld_hidden) type_error("z and u must have the same row stride");
  c.z = z.data_ptr();
  c.u = u.data_ptr();
  if (rc == SFFN_OK) rc = entry.forward(&c, y.data_ptr(), ld_y, current_stream(dev));
  if (rc == SFFN_OK) {
    if (y_out) written(y);
    if (z_out) written(z);
    if (u_out) written(u);
  }
  return py::make_tuple(rc, y, z, u);
}

// need: bits dx, dW_g, dW_up, dW_down, db_g; out: those five, None where they are made here.
py::tuple ffn_backward(const Tensor& dy, const Tensor& x, const Tensor& z, const Tensor& u, const Tensor& W_g, const Tensor& W_up, const Tensor& W_down, int act,
                       int act_up, int need, const std::vector<OptTensor>& out, const Tensor& status) {
  on_cuda(x);
  const c10::cuda::CUDAGuard guard(x.device());
  const at::Device dev = x.device();
  Tensor ws;
  int rc = 0;
  sffn_train_call c = make_call(x, W_g, W_up, W_down, act, act_up, status, true, ws, &rc);
  const at::ScalarType dtype = W_g.scalar_type();
  const int64_t ld_dy = rows("dy", dy, c.T, c.D, dtype, dev);
  c.ld_hidden = rows("z", z, c.T, c.H, dtype, dev);
  if (rows("u", u, c.T, c.H, dtype, dev) != c.ld_hidden) type_error("z and u must have the same row stride");
  c.z = z.data_ptr();
  c.u = u.data_ptr();
  sffn_train_grads g{};
  OptTensor got[5];
  auto take = [&](int i, at::IntArrayRef shape, at::ScalarType t) -> const Tensor& {
    got[i] = (size_t)i < out.size() && out[i] ? *out[i] : make(shape, t, dev);
    return *got[i];
  };
  if (need & 1) {
    const Tensor& t = take(0, {c.T, c.D}, dtype);
    g.ld_dx = rows("dx", t, c.T, c.D, dtype, dev);
    g.dx = t.data_ptr();
  }
  if (need & 2) g.dW_g = whole("dW_g", take(1, {c.H, c.D}, dtype), {c.H, c.D}, dtype, dev);
  if (need & 4) g.dW_up = whole("dW_up", take(2, {c.H, c.D}, dtype), {c.H, c.D}, dtype, dev);
  if (need & 8) g.dW_down = whole("dW_down", take(3, {c.H, c.D}, dtype), {c.H, c.D}, dtype, dev);
  if (need & 16) g.db_g = static_cast<float*>(whole("db_g", take(4, {c.H}, at::kFloat), {c.H}, at::kFloat, dev));
  if (rc == SFFN_OK) rc = entry.backward(&c, dy.data_ptr(), ld_dy, &g, current_stream(dev));
  for (size_t i = 0; rc == SFFN_OK && i < 5 && i < out.size(); ++i)
    if (got[i] && out[i]) written(*got[i]);
  return py::make_tuple(rc, got[0], got[1], got[2], got[3], got[4]);
}

const Tensor& tensor_of(PyObject* o, const char* name) {
  if (!o || !THPVariable_Check(o)) type_error(std::string(name) + ": a tensor expected");
  return THPVariable_Unpack(o);
}
// The items of a list or tuple, borrowed.
struct Items {
  PyObject* seq;
  Py_ssize_t n;
  explicit Items(const py::handle& h) : seq(h.ptr()), n(0) {
    if (!PyList_Check(seq) && !PyTuple_Check(seq)) type_error("a list of tensors expected");
    n = PySequence_Fast_GET_SIZE(seq);
  }
  PyObject* operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(seq, i); }
};

py::tuple grad_norm(const py::object& tensors, const OptTensor& norm_out, const Tensor& ws) {
  const Items list(tensors);
  std::vector<sffn_tensor> t((size_t)list.n);
  const at::Device dev = ws.device();
  for (Py_ssize_t i = 0; i < list.n; ++i) {
    const Tensor& g = tensor_of(list[i], "gradient");
    if (g.device() != dev) type_error("tensors must be on one device");
    if (!g.is_contiguous()) type_error("gradients must be contiguous fp32 or bf16 tensors");
    t[i].data = g.data_ptr();
    t[i].n = g.numel();
    t[i].dtype = dtype_code(g.scalar_type(), "gradients");
  }
  const c10::cuda::CUDAGuard guard(dev);
  // `ws` is this stream's, whose calls run one after another.  A graph may be replayed beside them: each captured call has its own,
  // zeroed by every replay.
  const Tensor own = capturing() ? at::zeros({ws.numel()}, ws.options()) : ws;
  const Tensor norm = norm_out ? *norm_out : make({}, at::kFloat, dev);
  float* out = static_cast<float*>(whole("norm", norm, {}, at::kFloat, dev));
  const int rc = entry.grad_norm(t.data(), (int)list.n, out, own.data_ptr(), (size_t)own.numel(), current_stream(dev));
  if (rc == SFFN_OK && norm_out) written(norm);
  return py::make_tuple(rc, norm);
}

// One number for all of n tensors, or a sequence of n.
struct Numbers {
  std::vector<double> v;
  double one = 0;
  Numbers(const py::object& o, Py_ssize_t n, const char* name) {
    if (PyList_Check(o.ptr()) || PyTuple_Check(o.ptr())) {
      v = o.cast<std::vector<double>>();
      if ((Py_ssize_t)v.size() != n) throw py::value_error(std::string(name) + ": one value, or one for each tensor");
    } else {
      one = o.cast<double>();
    }
  }
  double operator[](Py_ssize_t i) const { return v.empty() ? one : v[i]; }
};

// The moments of a tensor of this shape.
void put_state(sffn_adamw_tensor& a, PyObject* state, at::IntArrayRef shape, const at::Device& dev) {
  if (!PyDict_Check(state)) type_error("a state is a dict of m and v, and for 8 bits m_scale and v_scale");
  a.n = 1;
  for (int64_t s : shape) a.n *= s;
  PyObject* scale = PyDict_GetItemString(state, "m_scale");
  const at::ScalarType tm = scale ? at::kChar : at::kFloat, tv = scale ? at::kByte : at::kFloat;
  a.state_bits = scale ? 8 : 32;
  a.m = whole("m", tensor_of(PyDict_GetItemString(state, "m"), "m"), shape, tm, dev);
  a.v = whole("v", tensor_of(PyDict_GetItemString(state, "v"), "v"), shape, tv, dev);
  if (scale) {
    const int64_t groups = (a.n + 255) / 256;
    a.m_scale = static_cast<float*>(whole("m_scale", tensor_of(scale, "m_scale"), {groups}, at::kFloat, dev));
    a.v_scale = static_cast<float*>(whole("v_scale", tensor_of(PyDict_GetItemString(state, "v_scale"), "v_scale"), {groups}, at::kFloat, dev));
  }
}

int adamw_step(const py::object& params, const py::object& grads, const py::object& states, const py::object& masters, int64_t step, const py::object& lr,
               double beta1, double beta2, double eps, const py::object& weight_decay, const OptTensor& grad_norm, double max_norm) {
  const Items p(params), g(grads), s(states);
  const bool copies = !masters.is_none();
  const Items w(copies ? masters : params);
  if (g.n != p.n || s.n != p.n || w.n != p.n) throw py::value_error("params, grads, states and masters must be lists of one length");
  if (p.n == 0) return SFFN_OK;
  const Numbers rates(lr, p.n, "lr"), decays(weight_decay, p.n, "weight_decay");
  std::vector<sffn_adamw_tensor> t((size_t)p.n);
  const at::Device dev = tensor_of(p[0], "parameter").device();
  on_cuda(tensor_of(p[0], "parameter"));
  for (Py_ssize_t i = 0; i < p.n; ++i) {
    const Tensor &pi = tensor_of(p[i], "parameter"), &gi = tensor_of(g[i], "gradient");
    sffn_adamw_tensor& a = t[i];
    a.p_dtype = dtype_code(pi.scalar_type(), "parameters");
    a.g_dtype = dtype_code(gi.scalar_type(), "gradients");
    a.p = whole("parameter", pi, pi.sizes(), pi.scalar_type(), dev);
    a.g = whole("gradient", gi, pi.sizes(), gi.scalar_type(), dev);
    if (copies && w[i] != Py_None) a.master = static_cast<float*>(whole("master", tensor_of(w[i], "master"), pi.sizes(), at::kFloat, dev));
    put_state(a, s[i], pi.sizes(), dev);
    a.lr = rates[i];
    a.weight_decay = decays[i];
  }
  sffn_adamw_config c{};
  c.beta1 = beta1; c.beta2 = beta2; c.eps = eps; c.step = step; c.max_norm = max_norm;
  if (grad_norm) c.grad_norm = static_cast<const float*>(whole("grad_norm", *grad_norm, {}, at::kFloat, dev));
  const c10::cuda::CUDAGuard guard(dev);
  const int rc = entry.adamw_step(t.data(), (int)p.n, &c, current_stream(dev));
  for (Py_ssize_t i = 0; rc == SFFN_OK && i < p.n; ++i) {
    written(THPVariable_Unpack(p[i]));
    if (t[i].master) written(THPVariable_Unpack(w[i]));
    for (const char* name : {"m", "v"}) written(THPVariable_Unpack(PyDict_GetItemString(s[i], name)));
    if (t[i].state_bits != 8) continue;
    for (const char* name : {"m_scale", "v_scale"}) written(THPVariable_Unpack(PyDict_GetItemString(s[i], name)));
  }
  return rc;
}

int adamw_state_values(const py::object& states, const py::object& out) {
  const Items s(states), o(out);
  if (o.n != s.n) throw py::value_error("out: one dict for each state");
  if (s.n == 0) return SFFN_OK;
  std::vector<sffn_adamw_tensor> t((size_t)s.n);
  std::vector<float*> m((size_t)s.n), v((size_t)s.n);
  at::Device dev(at::kCPU);
  for (Py_ssize_t i = 0; i < s.n; ++i) {
    if (!PyDict_Check(s[i]) || !PyDict_Check(o[i])) type_error("states and out: lists of dicts");
    if (!PyDict_GetItemString(s[i], "m_scale")) type_error("these moments are held in 32 bits");
    const Tensor& mi = tensor_of(PyDict_GetItemString(s[i], "m"), "m");
    on_cuda(mi);
    if (i == 0) dev = mi.device();
    put_state(t[i], s[i], mi.sizes(), dev);
    m[i] = static_cast<float*>(whole("m", tensor_of(PyDict_GetItemString(o[i], "m"), "m"), mi.sizes(), at::kFloat, dev));
    v[i] = static_cast<float*>(whole("v", tensor_of(PyDict_GetItemString(o[i], "v"), "v"), mi.sizes(), at::kFloat, dev));
  }
  const c10::cuda::CUDAGuard guard(dev);
  const int rc = entry.adamw_state_values(t.data(), (int)s.n, m.data(), v.data(), current_stream(dev));
  for (Py_ssize_t i = 0; rc == SFFN_OK && i < s.n; ++i)
    for (const char* name : {"m", "v"}) written(THPVariable_Unpack(PyDict_GetItemString(o[i], name)));
  return rc;
}

// Steps of (a, b, c), one after another.
sffn_newton_schulz newton_schulz(const std::vector<double>& coefficients, double eps, int bits) {
  if (coefficients.empty() || coefficients.size() % 3) throw py::value_error("coefficients: three for every step");
  sffn_newton_schulz ns{};
  ns.steps = (int32_t)(coefficients.size() / 3);
  ns.bits = bits;
  ns.coefficients = coefficients.data();
  ns.eps = eps;
  return ns;
}
// rows x cols of a tensor of a matrix.
void matrix_of(const char* name, const Tensor& t, int32_t* r, int32_t* c) {
  if (t.dim() != 2) type_error(std::string(name) + ": a matrix expected, got " + shape_text(t.sizes()));
  if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX) type_error("sizes beyond 32 bits");
  *r = (int32_t)t.size(0);
  *c = (int32_t)t.size(1);
}

// (status, list of O): out: None, or a list of tensors to write to.
py::tuple orthogonalize(const py::object& updates, const py::object& out, const std::vector<double>& coefficients, double eps, int bits, const Tensor& status) {
  const Items u(updates);
  const bool given = !out.is_none();
  const Items o(given ? out : updates);
  if (o.n != u.n) throw py::value_error("updates and out must be lists of one length");
  const sffn_newton_schulz ns = newton_schulz(coefficients, eps, bits);
  std::vector<sffn_orthogonal> t((size_t)u.n);
  std::vector<Tensor> made((size_t)u.n);
  const at::Device dev = status.device();
  const c10::cuda::CUDAGuard guard(dev);
  for (Py_ssize_t i = 0; i < u.n; ++i) {
    const Tensor& ui = tensor_of(u[i], "update");
    sffn_orthogonal& a = t[i];
    a.dtype = dtype_code(ui.scalar_type(), "updates");
    matrix_of("update", ui, &a.rows, &a.cols);
    a.ld_u = rows("update", ui, a.rows, a.cols, ui.scalar_type(), dev);
    a.u = ui.data_ptr();
    made[i] = given ? tensor_of(o[i], "out") : make({a.rows, a.cols}, ui.scalar_type(), dev);
    a.ld_o = rows("out", made[i], a.rows, a.cols, ui.scalar_type(), dev);
    a.o = made[i].data_ptr();
  }
  size_t bytes = 0;
  int rc = entry.orthogonalize_workspace_bytes(t.data(), (int)u.n, &ns, &bytes);
  if (rc == SFFN_OK) {
    const Tensor ws = make({(int64_t)bytes}, at::kByte, dev);
    rc = entry.orthogonalize(t.data(), (int)u.n, &ns, ws.data_ptr(), bytes, static_cast<int32_t*>(status.data_ptr()), current_stream(dev));
  }
  if (rc == SFFN_OK && given)
    for (const Tensor& m : made) written(m);
  return py::make_tuple(rc, made);
}

int muon_step(const py::object& params, const py::object& grads, const py::object& states, const py::object& masters, const py::object& lr, double momentum,
              bool nesterov, const py::object& weight_decay, const py::object& scale, const std::vector<double>& coefficients, double eps, int bits,
              const OptTensor& grad_norm, double max_norm, const Tensor& status) {
  const Items p(params), g(grads), s(states);
  const bool copies = !masters.is_none();
  const Items w(copies ? masters : params);
  if (g.n != p.n || s.n != p.n || w.n != p.n) throw py::value_error("params, grads, states and masters must be lists of one length");
  const Numbers rates(lr, p.n, "lr"), decays(weight_decay, p.n, "weight_decay"), scales(scale, p.n, "scale");
  std::vector<sffn_muon_tensor> t((size_t)p.n);
  const at::Device dev = status.device();
  for (Py_ssize_t i = 0; i < p.n; ++i) {
    const Tensor &pi = tensor_of(p[i], "parameter"), &gi = tensor_of(g[i], "gradient");
    sffn_muon_tensor& a = t[i];
    a.p_dtype = dtype_code(pi.scalar_type(), "parameters");
    a.g_dtype = dtype_code(gi.scalar_type(), "gradients");
    matrix_of("parameter", pi, &a.rows, &a.cols);
    a.p = whole("parameter", pi, pi.sizes(), pi.scalar_type(), dev);
    a.g = whole("gradient", gi, pi.sizes(), gi.scalar_type(), dev);
    if (copies && w[i] != Py_None) a.master = static_cast<float*>(whole("master", tensor_of(w[i], "master"), pi.sizes(), at::kFloat, dev));
    if (!PyDict_Check(s[i])) type_error("a state is a dict of m");
    a.m = static_cast<float*>(whole("m", tensor_of(PyDict_GetItemString(s[i], "m"), "m"), pi.sizes(), at::kFloat, dev));
    a.lr = rates[i];
    a.weight_decay = decays[i];
    a.scale = scales[i];
  }
  sffn_muon_config c{};
  c.newton_schulz = newton_schulz(coefficients, eps, bits);
  c.momentum = momentum;
  c.nesterov = nesterov;
  c.max_norm = max_norm;
  if (grad_norm) c.grad_norm = static_cast<const float*>(whole("grad_norm", *grad_norm, {}, at::kFloat, dev));
  const c10::cuda::CUDAGuard guard(dev);
  size_t bytes = 0;
  int rc = entry.muon_workspace_bytes(t.data(), (int)p.n, &c.newton_schulz, &bytes);
  if (rc != SFFN_OK) return rc;
  const Tensor ws = make({(int64_t)bytes}, at::kByte, dev);
  rc = entry.muon_step(t.data(), (int)p.n, &c, ws.data_ptr(), bytes, static_cast<int32_t*>(status.data_ptr()), current_stream(dev));
  for (Py_ssize_t i = 0; rc == SFFN_OK && i < p.n; ++i) {
    written(THPVariable_Unpack(p[i]));
    if (t[i].master) written(THPVariable_Unpack(w[i]));
    written(THPVariable_Unpack(PyDict_GetItemString(s[i], "m")));
  }
  return rc;
}

// What both passes of the norms around a block hand over, but for resid, h, n and their statistics.
sffn_block_norm make_block(const OptTensor& y, const Tensor& like, const OptTensor& post_gain, const OptTensor& pre_gain, const OptTensor& gate, double scale,
                           double eps) {
  on_cuda(like);
  if (like.dim() != 2) type_error("y, resid and h are [T, D]");
  const at::Device dev = like.device();
  const int64_t T = like.size(0), D = like.size(1);
  if (T > INT32_MAX || D > INT32_MAX) type_error("sizes beyond 32 bits");
  sffn_block_norm c{};
  c.T = (int32_t)T; c.D = (int32_t)D;
  c.scale = (float)scale; c.eps = (float)eps;
  if (y) {
    c.y_dtype = dtype_code(y->scalar_type(), "y");
    c.ld_y = rows("y", *y, T, D, y->scalar_type(), dev);
    c.y = y->data_ptr();
  }
  if (post_gain) c.post_gain = static_cast<const float*>(whole("post_gain", *post_gain, {D}, at::kFloat, dev));
  if (pre_gain) c.pre_gain = static_cast<const float*>(whole("pre_gain", *pre_gain, {D}, at::kFloat, dev));
  if (gate && gate->dim() == 1) {
    c.gate_kind = SFFN_BLOCK_GATE_CHANNEL;
    c.gate = whole("gate", *gate, {D}, at::kFloat, dev);
  } else if (gate && gate->dim() == 2 && gate->size(1) == 1 && D != 1) {
    c.gate_kind = SFFN_BLOCK_GATE_TOKEN;
    c.gate = whole("gate", *gate, {T, 1}, at::kFloat, dev);
  } else if (gate) {
    c.gate_kind = SFFN_BLOCK_GATE_FULL;  // its type is h's: checked once that is known
    c.ld_gate = rows("gate", *gate, T, D, gate->scalar_type(), dev);
    c.gate = gate->data_ptr();
  }
  return c;
}
void check_full_gate(const sffn_block_norm& c, const OptTensor& gate, at::ScalarType h_dtype) {
  if (c.gate_kind == SFFN_BLOCK_GATE_FULL) check_plain("gate", *gate, {c.T, c.D}, h_dtype, gate->device());
}

// (status, h, n, stats): h None without y, n None without pre_gain.
py::tuple block_forward(const OptTensor& y, const OptTensor& resid, const OptTensor& post_gain, const OptTensor& pre_gain, const OptTensor& gate, double scale,
                        double eps, bool save, const py::object& h_dtype, const py::object& n_dtype, const OptTensor& h_out, const OptTensor& n_out) {
  if (!y && !resid) type_error("y or resid is needed");
  const Tensor& like = resid ? *resid : *y;
  sffn_block_norm c = make_block(y, like, post_gain, pre_gain, gate, scale, eps);
  const at::Device dev = like.device();
  const c10::cuda::CUDAGuard guard(dev);
  auto asked = [](const py::object& o) { return reinterpret_cast<THPDtype*>(o.ptr())->scalar_type; };
  for (const py::object* o : {&h_dtype, &n_dtype})
    if (!o->is_none() && !THPDtype_Check(o->ptr())) type_error("h_dtype and n_dtype are torch types");
  const at::ScalarType th = resid ? resid->scalar_type() : h_out ? h_out->scalar_type() : h_dtype.is_none() ? y->scalar_type() : asked(h_dtype);
  if (!h_dtype.is_none() && asked(h_dtype) != th) type_error("h has resid's type, or that of the tensor given for it");
  const at::ScalarType tn = n_out ? n_out->scalar_type() : n_dtype.is_none() ? th : asked(n_dtype);
  if (!n_dtype.is_none() && asked(n_dtype) != tn) type_error("n has the type of the tensor given for it");
  c.h_dtype = dtype_code(th, "the residual stream");
  c.n_dtype = dtype_code(tn, "n");
  if (!y) c.y_dtype = c.h_dtype;
  check_full_gate(c, gate, th);
  if (resid) {
    c.ld_resid = rows("resid", *resid, c.T, c.D, th, dev);
    c.resid = resid->data_ptr();
  }
  OptTensor h, n, stats;
  if (y) {
    h = h_out ? *h_out : make({c.T, c.D}, th, dev);
    c.ld_h = rows("h", *h, c.T, c.D, th, dev);
    c.h = h->data_ptr();
  } else if (h_out) {
    type_error("without y, h is resid: nothing is written to it");
  }
  if (pre_gain) {
    n = n_out ? *n_out : make({c.T, c.D}, tn, dev);
    c.ld_n = rows("n", *n, c.T, c.D, tn, dev);
    c.n = n->data_ptr();
  } else if (n_out) {
    type_error("n needs pre_gain");
  }
  if (save) {
    stats = make({2, c.T}, at::kFloat, dev);
    c.stats = static_cast<float*>(stats->data_ptr());
  }
  const int rc = entry.block_forward(&c, current_stream(dev));
  if (rc == SFFN_OK) {
    if (y && h_out) written(*h);
    if (n_out) written(*n);
  }
  return py::make_tuple(rc, h, n, stats);
}

// need: bits dy, dresid, dpost_gain, dpre_gain, dgate; out: those five, None where they are made here.
py::tuple block_backward(const OptTensor& dh, const OptTensor& dn, const OptTensor& y, const Tensor& h, const OptTensor& stats, const OptTensor& post_gain,
                         const OptTensor& pre_gain, const OptTensor& gate, double scale, int need, const std::vector<OptTensor>& out) {
  sffn_block_norm c = make_block(y, h, post_gain, pre_gain, gate, scale, 0.0);
  const at::Device dev = h.device();
  const c10::cuda::CUDAGuard guard(dev);
  const at::ScalarType th = h.scalar_type();
  c.h_dtype = dtype_code(th, "the residual stream");
  c.n_dtype = dn ? dtype_code(dn->scalar_type(), "dn") : c.h_dtype;
  if (!y) c.y_dtype = c.h_dtype;
  check_full_gate(c, gate, th);
  c.ld_h = rows("h", h, c.T, c.D, th, dev);
  c.h = h.data_ptr();
  if (stats) c.stats = static_cast<float*>(whole("stats", *stats, {2, c.T}, at::kFloat, dev));
  sffn_block_grads g{};
  if (dh) {
    g.ld_dh = rows("dh", *dh, c.T, c.D, th, dev);
    g.dh = dh->data_ptr();
  }
  if (dn) {
    g.ld_dn = rows("dn", *dn, c.T, c.D, dn->scalar_type(), dev);
    g.dn = dn->data_ptr();
  }
  OptTensor got[5];
  auto take = [&](int i, at::IntArrayRef shape, at::ScalarType t) -> const Tensor& {
    got[i] = (size_t)i < out.size() && out[i] ? *out[i] : make(shape, t, dev);
    return *got[i];
  };
  if (need & 1 && y) {
    const Tensor& t = take(0, {c.T, c.D}, y->scalar_type());
    g.ld_dy = rows("dy", t, c.T, c.D, y->scalar_type(), dev);
    g.dy = t.data_ptr();
  }
  if (need & 2) {
    const Tensor& t = take(1, {c.T, c.D}, th);
    g.ld_dresid = rows("dresid", t, c.T, c.D, th, dev);
    g.dresid = t.data_ptr();
  }
  if (need & 4 && post_gain) g.dpost_gain = static_cast<float*>(whole("dpost_gain", take(2, {c.D}, at::kFloat), {c.D}, at::kFloat, dev));
  if (need & 8 && pre_gain) g.dpre_gain = static_cast<float*>(whole("dpre_gain", take(3, {c.D}, at::kFloat), {c.D}, at::kFloat, dev));
  if (need & 16 && gate) {
    const Tensor& t = take(4, gate->sizes(), gate->scalar_type());
    if (c.gate_kind == SFFN_BLOCK_GATE_FULL) g.ld_dgate = rows("dgate", t, c.T, c.D, th, dev);
    else whole("dgate", t, gate->sizes(), at::kFloat, dev);
    g.dgate = t.data_ptr();
  }
  Tensor ws;
  int rc = SFFN_OK;
  if (g.dpost_gain || g.dpre_gain || (g.dgate && c.gate_kind == SFFN_BLOCK_GATE_CHANNEL)) {
    size_t bytes = 0;
    rc = entry.block_workspace_bytes(c.D, &bytes);
    if (rc == SFFN_OK) {
      ws = make({(int64_t)bytes}, at::kByte, dev);
      g.workspace = ws.data_ptr();
      g.workspace_bytes = bytes;
    }
  }
  if (rc == SFFN_OK) rc = entry.block_backward(&c, &g, current_stream(dev));
  for (size_t i = 0; rc == SFFN_OK && i < 5 && i < out.size(); ++i)
    if (got[i] && out[i]) written(*got[i]);
  return py::make_tuple(rc, got[0], got[1], got[2], got[3], got[4]);
}

}  // namespace

PYBIND11_MODULE(_training, m) {
  m.attr("torch_version") = SFFN_TORCH;  // what it was compiled against
  m.def("bind", &bind);
  m.def("kept", &kept);
  m.def("ffn_forward", &ffn_forward);
  m.def("ffn_backward", &ffn_backward);
  m.def("grad_norm", &grad_norm);
  m.def("adamw_step", &adamw_step);
  m.def("adamw_state_values", &adamw_state_values);
  m.def("orthogonalize", &orthogonalize);
  m.def("muon_step", &muon_step);
  m.def("block_forward", &block_forward);
  m.def("block_backward", &block_backward);
}
