// The tensor side of gradient clipping, layer norm and attention: what their
// Python functions hand on, and autograd's nodes.
//
// A training step makes hundreds of these calls, of some ten microseconds of
// kernels each, and autograd runs a backward function on a thread of its own,
// where one in Python finds the interpreter's objects in another core's cache.
// Microseconds of the host with all of it in Python / here: layer norm forward 8.2 /
// 3.7, forward and backward 100 / 64 (of which torch.autograd.grad around an empty
// function is some 45), attention likewise 105 / 63, the norm of a small model's
// gradients 23 / 10.
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/csrc/utils/pybind.h>

#include <algorithm>
#include <optional>
#include <string>
#include <utility>
#include <vector>

#include "microadam.h"

namespace py = pybind11;

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

// ------------------------------------------------- what all of them share

std::string name_of(at::ScalarType t) {
  return py::str(py::cast<py::object>(py::handle((PyObject*)torch::getTHPDtype(t))));
}

[[noreturn]] void not_implemented(const std::string& what) {
  PyErr_SetString(PyExc_NotImplementedError, what.c_str());
  throw py::error_already_set();
}

// Raises the package's own error where a call has been refused.
void check(int rc, const char* where) {
  if (rc != MICROADAM_OK) py::module_::import("paper_2405_15593_amd").attr("_check")(rc, where);
}

// ... of a backward pass, on autograd's thread.
void check_here(int rc, const char* where) {
  TORCH_CHECK(rc == MICROADAM_OK, where, ": ", microadam_last_error());
}

bool is_known(at::ScalarType t) { return t == at::kFloat || t == at::kBFloat16; }
int32_t code_of(at::ScalarType t) { return t == at::kBFloat16 ? MICROADAM_BF16 : MICROADAM_F32; }

void check_dtype(const Tensor& t, const char* what) {
  if (!is_known(t.scalar_type()))
    throw py::type_error(std::string(what) + ": float32 or bfloat16, not " + name_of(t.scalar_type()));
}

// These functions have no forward-mode derivatives: a result without a tangent
// would silently be a constant.
void refuse_tangent(const Tensor& t, const char* what) {
  if (t.defined() && t._fw_grad(0).defined()) not_implemented(std::string(what) + ": no derivatives in forward mode");
}

// Whether a graph of torch's operators is being recorded (torch.jit.trace, make_fx
// and torch.export).  It would hold the allocations made here and none of the
// launches: a function that returns memory that nothing wrote.  Other dispatch modes
// only watch.
bool is_traced() {
  return torch::jit::tracer::isTracing() || c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::PreDispatch) ||
         c10::impl::TorchDispatchModeTLS::get_mode(c10::impl::TorchDispatchModeKey::PROXY).has_value();
}

void refuse_trace(const char* what) {
  if (is_traced()) not_implemented(std::string(what) + ": not recorded by torch's tracers");
}

// ... of a backward pass, whose forward pass was not recorded.
void refuse_trace_here(const char* what) {
  TORCH_CHECK_NOT_IMPLEMENTED(!is_traced(), what, ": the backward pass is not recorded by torch's tracers");
}

typedef std::optional<Tensor> Perhaps;  // (autograd's functions take a tensor that is not there as none at all)
Perhaps perhaps(const Tensor& t) { return t.defined() ? Perhaps(t) : Perhaps(); }
Tensor given(const Perhaps& t) { return t.value_or(Tensor()); }

bool wants_grad(const Tensor& t) { return t.defined() && t.requires_grad(); }

void* stream_of(const Tensor& t) { return c10::hip::getCurrentHIPStream(t.get_device()).stream(); }

Tensor bytes(uint64_t n, const Tensor& like) {
  return n ? at::empty({(int64_t)n}, like.options().dtype(at::kByte)) : Tensor();
}

void* address(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// The results of a backward pass, which is not differentiable itself: where a
// graph of it is made, through a node that raises.
class Once : public torch::autograd::Function<Once> {
 public:
  static Tensor forward(AutogradContext*, const Tensor& t) { return t.detach(); }
  static variable_list backward(AutogradContext*, const variable_list&) {
    TORCH_CHECK(false, "the backward pass has no derivative");
  }
};

variable_list once(variable_list grads) {
  if (c10::GradMode::is_enabled())
    for (Tensor& t : grads)
      if (t.defined()) t = Once::apply(t.detach().requires_grad_());
  return grads;
}

// ------------------------------------------------- gradient norm and clipping

// Whether t's elements fill one run of memory, each place once, in any order of
// the dimensions.
bool is_dense(const Tensor& t) {
  if (t.is_contiguous() || t.numel() == 0) return true;
  std::vector<std::pair<int64_t, int64_t>> d;
  for (int64_t i = 0; i < t.dim(); ++i)
    if (t.size(i) != 1) d.emplace_back(t.stride(i), t.size(i));
  std::sort(d.begin(), d.end());
  int64_t want = 1;
  for (const auto& x : d) {
    if (x.first != want) return false;
    want *= x.second;
  }
  return true;
}

Tensor clip(const char* what, const std::vector<Tensor>& grads, bool scale, double max_norm, double eps,
            const Perhaps& workspace) {
  refuse_trace(what);
  if (grads.empty()) throw py::value_error("grads: at least one tensor");
  const Tensor& first = grads[0];
  const bool grad_mode = c10::GradMode::is_enabled();
  for (const Tensor& g : grads) refuse_tangent(g, what);
  for (const Tensor& g : grads)
    if (!g.is_cuda() || g.device() != first.device() || g.layout() != at::kStrided)
      throw py::value_error("grads: tensors on one ROCm device");
  for (const Tensor& g : grads) check_dtype(g, "grads");
  const size_t n = grads.size();
  std::vector<void*> at(n);
  std::vector<int64_t> numels(n);
  std::vector<int32_t> dtypes(n);
  for (size_t i = 0; i < n; ++i) {
    const Tensor& g = grads[i];
    if (grad_mode && g.requires_grad()) not_implemented("grads: no derivative; a gradient requires grad");
    if (!is_dense(g)) throw py::value_error("grads: a gradient with gaps or overlaps in memory");
    at[i] = g.data_ptr();
    numels[i] = g.numel();
    dtypes[i] = code_of(g.scalar_type());
  }
  if (workspace && (workspace->scalar_type() != at::kByte || !workspace->is_contiguous() || workspace->device() != first.device()))
    throw py::value_error("workspace: a contiguous uint8 tensor on the gradients' device");
  const c10::DeviceGuard guard(first.device());
  const Tensor norm = at::empty({}, at::TensorOptions().dtype(at::kFloat).device(first.device()));
  uint64_t need = 0;
  check(microadam_clip_workspace(&need), "microadam_clip_workspace");
  const Tensor store = workspace ? *workspace : bytes(need, first);
  const uint64_t size = (uint64_t)store.numel();
  if (!scale) {
    check(microadam_grad_norm(at.data(), numels.data(), dtypes.data(), (int32_t)n, norm.data_ptr<float>(), store.data_ptr(),
                              size, stream_of(first)),
          "microadam_grad_norm");
    return norm;
  }
  check(microadam_clip_grads(at.data(), numels.data(), dtypes.data(), (int32_t)n, max_norm, eps, norm.data_ptr<float>(),
                             store.data_ptr(), size, stream_of(first)),
        "microadam_clip_grads");
  for (const Tensor& g : grads)
    if (!g.is_inference()) g.unsafeGetTensorImpl()->bump_version();
  return norm;
}

Tensor grad_norm(const std::vector<Tensor>& grads, const Perhaps& workspace) {
  return clip("grad_norm", grads, false, 0.0, 0.0, workspace);
}

Tensor clip_grads(const std::vector<Tensor>& grads, double max_norm, double eps, const Perhaps& workspace) {
  return clip("clip_grads", grads, true, max_norm, eps, workspace);
}

// ------------------------------------------------- layer norm

// A tensor's rows of `cols` elements at one stride: where it lies, or a copy.
struct Matrix {
  Tensor t;
  int64_t ld;
};

Matrix matrix(const Tensor& t) {
  const int64_t cols = t.size(-1);
  if (t.is_contiguous()) return {t, cols};
  if (cols == 1 || t.stride(-1) == 1) {
    int64_t ld = 0, next = 0;  // of the last dimension before the row; what one further out steps by
    bool even = true;
    for (int64_t i = t.dim() - 2; i >= 0 && even; --i) {
      if (t.size(i) == 1) continue;
      if (!ld)
        ld = t.stride(i);
      else
        even = t.stride(i) == next;
      even = even && ld >= cols;
      next = t.stride(i) * t.size(i);
    }
    if (even) return {t, ld ? ld : cols};
  }
  return {t.contiguous(), cols};
}

microadam_rows rows_of(const Matrix& x, const Tensor& weight, const Tensor& bias, double eps) {
  const Tensor& side = weight.defined() ? weight : bias.defined() ? bias : x.t;
  const int64_t cols = x.t.size(-1);
  return {x.t.data_ptr(), address(weight), address(bias),          x.t.numel() / cols,         cols,
          x.ld,           eps,             code_of(x.t.scalar_type()), code_of(side.scalar_type())};
}

Tensor dense(const Tensor& t) { return t.defined() ? t.contiguous() : t; }

// (y, and where they are kept each row's mean, then each row's rstd)
std::pair<Tensor, Tensor> norm_rows(const Tensor& x, const Tensor& weight, const Tensor& bias, double eps, bool keep) {
  const c10::DeviceGuard guard(x.device());
  const Matrix in = matrix(x);
  const Tensor w = dense(weight), b = dense(bias);
  const microadam_rows rows = rows_of(in, w, b, eps);
  const Tensor y = at::empty(x.sizes(), x.options());
  const Tensor stats = keep ? at::empty({2 * rows.rows}, x.options().dtype(at::kFloat)) : Tensor();
  float* mean = keep ? stats.data_ptr<float>() : nullptr;
  check(microadam_layer_norm(&rows, y.data_ptr(), rows.cols, mean, keep ? mean + rows.rows : nullptr, stream_of(x)),
        "microadam_layer_norm");
  return {y, stats};
}

class LayerNorm : public torch::autograd::Function<LayerNorm> {
 public:
  static Tensor forward(AutogradContext* ctx, const Tensor& x, const Perhaps& given_weight, const Perhaps& given_bias,
                        double eps) {
    const Tensor weight = given(given_weight), bias = given(given_bias);
    auto [y, stats] = norm_rows(x, weight, bias, eps, true);
    const Tensor& side = weight.defined() ? weight : bias.defined() ? bias : x;
    ctx->save_for_backward({x, weight, stats});
    ctx->saved_data["eps"] = eps;
    ctx->saved_data["side"] = (int64_t)side.scalar_type();
    ctx->saved_data["bias"] = bias.defined();
    return y;
  }

  static variable_list backward(AutogradContext* ctx, const variable_list& grads) {
    refuse_trace_here("layer_norm");
    variable_list result(4);
    {
      const c10::AutoGradMode off(false);
      const variable_list saved = ctx->get_saved_variables();
      const Tensor &x = saved[0], w = dense(saved[1]), &stats = saved[2];
      const c10::DeviceGuard guard(x.device());
      const Matrix in = matrix(x), dy = matrix(grads[0]);
      const auto side = (at::ScalarType)ctx->saved_data["side"].toInt();
      microadam_rows rows = rows_of(in, w, Tensor(), ctx->saved_data["eps"].toDouble());
      rows.weight_dtype = code_of(side);
      uint64_t need = 0;
      // (numbered among the tensors that there are)
      size_t number = 1;
      if (ctx->needs_input_grad(0)) result[0] = at::empty(x.sizes(), x.options());
      if (w.defined() && ctx->needs_input_grad(number++)) result[1] = at::empty({rows.cols}, x.options().dtype(side));
      if (ctx->saved_data["bias"].toBool() && ctx->needs_input_grad(number))
        result[2] = at::empty({rows.cols}, x.options().dtype(side));
      if (result[1].defined() || result[2].defined())
        check_here(microadam_layer_norm_workspace(&rows, &need), "microadam_layer_norm_workspace");
      const Tensor store = bytes(need, x);
      const float* mean = stats.data_ptr<float>();
      check_here(microadam_layer_norm_grad(&rows, mean, mean + rows.rows, dy.t.data_ptr(), dy.ld, address(result[0]), rows.cols,
                                           address(result[1]), address(result[2]), address(store), need, stream_of(x)),
                 "microadam_layer_norm_grad");
    }
    return once(std::move(result));
  }
};

Tensor layer_norm(const Tensor& x, const Perhaps& given_weight, const Perhaps& given_bias, double eps) {
  const Tensor weight = given(given_weight), bias = given(given_bias);
  refuse_trace("layer_norm");
  for (const Tensor* t : {&x, &weight, &bias}) refuse_tangent(*t, "layer_norm");
  check_dtype(x, "x");
  if (!x.is_cuda()) throw py::value_error("x: a tensor on a ROCm device");
  if (x.dim() < 1 || x.size(-1) < 1) throw py::value_error("x: at least one element in the last dimension");
  for (const auto& [t, what] : {std::pair<const Tensor&, const char*>{weight, "weight"}, {bias, "bias"}}) {
    if (!t.defined()) continue;
    check_dtype(t, what);
    if (weight.defined() && t.scalar_type() != weight.scalar_type()) throw py::type_error("weight and bias: one dtype");
    if (t.dim() != 1 || t.size(0) != x.size(-1) || t.device() != x.device())
      throw py::value_error(std::string(what) + ": one element for each of x's last dimension, on x's device");
  }
  if (c10::GradMode::is_enabled() && (wants_grad(x) || wants_grad(weight) || wants_grad(bias)))
    return LayerNorm::apply(x, perhaps(weight), perhaps(bias), eps);
  return norm_rows(x, weight, bias, eps, false).first;
}

// ------------------------------------------------- attention

constexpr int64_t kFar = (int64_t)1 << 23;  // elements from position to position that the C ABI takes

// t, or a copy where its rows are not contiguous, share elements or lie too far apart.
Tensor in_rows(const Tensor& t) {
  const int64_t pos = t.stride(1);
  return t.stride(3) == 1 && ((pos >= t.size(3) && pos <= kFar) || t.size(1) <= 1) ? t : t.contiguous();
}

microadam_heads heads_of(const Tensor& t) { return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)}; }

microadam_attention attention_of(const Tensor& q, const Tensor& k, const Tensor& v, const Tensor& lengths, bool causal,
                                 double scale) {
  return {heads_of(q), heads_of(k), heads_of(v), (const int32_t*)address(lengths), q.size(0), q.size(1), k.size(1),
          q.size(2),   k.size(2),   q.size(3),   scale,                            code_of(q.scalar_type()), causal ? 1 : 0};
}

// (out, and where it is kept what the backward pass takes besides)
std::pair<Tensor, Tensor> attend(const Tensor& given_q, const Tensor& given_k, const Tensor& given_v, const Tensor& lengths,
                                 bool causal, double scale, bool keep) {
  const c10::DeviceGuard guard(given_q.device());
  const Tensor q = in_rows(given_q), k = in_rows(given_k), v = in_rows(given_v);
  const microadam_attention a = attention_of(q, k, v, lengths, causal, scale);
  uint64_t need = 0, kept = 0;
  check(microadam_attention_workspace(&a, 0, &need), "microadam_attention_workspace");
  if (keep) check(microadam_attention_saved(&a, &kept), "microadam_attention_saved");
  const Tensor out = at::empty(q.sizes(), q.options());
  const Tensor store = bytes(need, q), saved = bytes(kept, q);
  const microadam_heads to = heads_of(out);
  check(microadam_attention_forward(&a, &to, address(saved), kept, address(store), need, stream_of(q)),
        "microadam_attention_forward");
  return {out, saved};
}

class Attention : public torch::autograd::Function<Attention> {
 public:
  static Tensor forward(AutogradContext* ctx, const Tensor& q, const Tensor& k, const Tensor& v,
                        const Perhaps& given_lengths, bool causal, double scale) {
    const Tensor lengths = given(given_lengths);
    auto [out, saved] = attend(q, k, v, lengths, causal, scale, true);
    ctx->save_for_backward({q, k, v, lengths, out, saved});
    ctx->saved_data["causal"] = causal;
    ctx->saved_data["scale"] = scale;
    return out;
  }

  static variable_list backward(AutogradContext* ctx, const variable_list& grads) {
    refuse_trace_here("attention");
    variable_list result(6);
    {
      const c10::AutoGradMode off(false);
      const variable_list saved = ctx->get_saved_variables();
      const c10::DeviceGuard guard(saved[0].device());
      const Tensor q = in_rows(saved[0]), k = in_rows(saved[1]), v = in_rows(saved[2]), dout = in_rows(grads[0]);
      const microadam_attention a = attention_of(q, k, v, saved[3], ctx->saved_data["causal"].toBool(),
                                                 ctx->saved_data["scale"].toDouble());
      for (int i = 0; i < 3; ++i) result[i] = at::empty(saved[i].sizes(), saved[i].options());
      uint64_t need = 0;
      check_here(microadam_attention_workspace(&a, 1, &need), "microadam_attention_workspace");
      const Tensor store = bytes(need, q);
      const microadam_heads out = heads_of(saved[4]), to = heads_of(dout), dq = heads_of(result[0]),
                            dk = heads_of(result[1]), dv = heads_of(result[2]);
      check_here(microadam_attention_grad(&a, &out, address(saved[5]), saved[5].defined() ? saved[5].numel() : 0, &to, &dq,
                                          &dk, &dv, address(store), need, stream_of(q)),
                 "microadam_attention_grad");
    }
    return once(std::move(result));
  }
};

Tensor attention(const Tensor& q, const Tensor& k, const Tensor& v, bool causal, double scale,
                 const Perhaps& key_lengths) {
  refuse_trace("attention");
  for (const Tensor* t : {&q, &k, &v}) refuse_tangent(*t, "attention");
  for (const auto& [t, what] : {std::pair<const Tensor&, const char*>{q, "q"}, {k, "k"}, {v, "v"}}) {
    check_dtype(t, what);
    if (t.dim() != 4) throw py::value_error(std::string(what) + ": (batch, positions, heads, dim)");
    if (!t.is_cuda() || t.device() != q.device()) throw py::value_error("q, k and v: tensors on one ROCm device");
    if (t.scalar_type() != q.scalar_type()) throw py::type_error("q, k and v: one dtype");
  }
  if (k.sizes() != v.sizes() || k.size(0) != q.size(0) || k.size(3) != q.size(3))
    throw py::value_error("k and v: one shape, with q's batch and dim");
  Tensor lengths;
  if (key_lengths) {
    if (key_lengths->scalar_type() != at::kInt)
      throw py::type_error("key_lengths: int32, not " + name_of(key_lengths->scalar_type()));
    if (key_lengths->dim() != 1 || key_lengths->size(0) != q.size(0) || key_lengths->device() != q.device())
      throw py::value_error("key_lengths: one for each sequence, on q's device");
    const c10::DeviceGuard guard(q.device());
    lengths = key_lengths->contiguous();
  }
  if (c10::GradMode::is_enabled() && (wants_grad(q) || wants_grad(k) || wants_grad(v)))
    return Attention::apply(q, k, v, perhaps(lengths), causal, scale);
  return attend(q, k, v, lengths, causal, scale, false).first;
}

}  // namespace

PYBIND11_MODULE(_operators, m) {
  m.def("grad_norm", &grad_norm);
  m.def("clip_grads", &clip_grads);
  m.def("layer_norm", &layer_norm);
  m.def("attention", &attention);
}
