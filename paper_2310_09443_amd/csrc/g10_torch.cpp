// Marshalling between torch tensors and the C ABI of include/g10_ops.h: argument checks (ValueError, before anything is
// launched), outputs and workspaces from torch's allocator, the current stream of the tensors' device.  Host code only; in C++
// because a step of small tensors is bound by it: the checks of 300 gradients take Python 150 us and this 10.
#include <torch/extension.h>

#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>

#include <math.h>
#include <optional>
#include <unordered_map>
#include <vector>

#include "g10_ops.h"

namespace py = pybind11;
typedef std::optional<at::Tensor> Maybe;

// The library's calls, from the copy of it that paper_2310_09443_amd.binding has loaded.
static struct {
  decltype(&g10_norm_rope) norm_rope;
  decltype(&g10_norm_rope_workspace) norm_rope_workspace;
  decltype(&g10_norm_rope_backward) norm_rope_backward;
  decltype(&g10_attention_workspace) attention_workspace;
  decltype(&g10_attention) attention;
  decltype(&g10_attention_backward_workspace) attention_backward_workspace;
  decltype(&g10_attention_backward) attention_backward;
  decltype(&g10_adamw_create) adamw_create;
  decltype(&g10_adamw_step) adamw_step;
  decltype(&g10_grad_norm) grad_norm;
  decltype(&g10_adamw_free) adamw_free;
} lib;

static void bind(const std::vector<uintptr_t>& at) {
  TORCH_CHECK_VALUE(at.size() == 11, "eleven addresses");
  size_t i = 0;
  auto next = [&](auto& f) { f = (std::decay_t<decltype(f)>)at[i++]; };
  next(lib.norm_rope); next(lib.norm_rope_workspace); next(lib.norm_rope_backward);
  next(lib.attention_workspace); next(lib.attention); next(lib.attention_backward_workspace); next(lib.attention_backward);
  next(lib.adamw_create); next(lib.adamw_step); next(lib.grad_norm); next(lib.adamw_free);
}

static void check(int rc, const char* what) {
  if (!rc) return;
  TORCH_CHECK_VALUE(rc != G10_EINVAL, what, " refuses these sizes or numbers");       // (what the checks here leave to the library's)
  py::object error = py::module_::import("paper_2310_09443_amd.binding").attr("G10Error");
  PyErr_SetObject(error.ptr(), error(rc, what).ptr());
  throw py::error_already_set();
}

static int type_of(at::ScalarType t) {
  return t == at::kFloat ? G10_F32 : t == at::kHalf ? G10_F16 : t == at::kBFloat16 ? G10_BF16 : -1;
}

static void on_device(const at::Tensor& t, const char* name, const at::Device* dev) {
  TORCH_CHECK_VALUE(t.is_cuda(), name, " must lie in GPU memory");
  TORCH_CHECK_VALUE(!dev || t.device() == *dev, name, " must lie on the device of the other tensors");
}

static void* stream_of(const at::Device& dev) { return (void*)c10::hip::getCurrentHIPStream(dev.index()).stream(); }

static at::Tensor room(uint64_t bytes, const at::Device& dev) {
  return at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(dev));
}

// ---------------------------------------------------------------------------------------------------- norm and rotation
// (batch, token, head) strides of [batch, token, head, dim] or, with batch 1, of [token, head, dim]
static void put_strides(int64_t (&to)[3], const at::Tensor& t) {
  const auto s = t.strides();
  const bool four = t.dim() == 4;
  to[0] = four ? s[0] : 0;
  to[1] = s[four ? 1 : 0];
  to[2] = s[four ? 2 : 1];
}
static at::Tensor inner(const at::Tensor& t) { return t.size(-1) <= 1 || t.stride(-1) == 1 ? t : t.contiguous(); }

static py::tuple norm_rope(const Maybe& q, const Maybe& k, const at::Tensor& table, const at::Tensor& positions_in, const Maybe& q_weight,
                           const Maybe& k_weight, double eps, bool interleaved, bool back, const Maybe& dq, const Maybe& dk) {
  TORCH_CHECK_VALUE(q || k, "queries or keys are needed");
  const at::Tensor& one = q ? *q : *k;
  on_device(one, q ? "q" : "k", nullptr);
  const at::Device dev = one.device();
  const at::ScalarType dt = one.scalar_type();
  TORCH_CHECK_VALUE(type_of(dt) >= 0, "type ", dt, " is not supported: float32, float16 or bfloat16");
  TORCH_CHECK_VALUE(one.dim() == 3 || one.dim() == 4, "q and k are [batch, token, head, dim] or [token, head, dim]");
  const int64_t dim = one.size(-1);
  const auto lead = one.sizes().slice(0, one.dim() - 2);
  TORCH_CHECK_VALUE(dim > 0 && dim <= 256, "dim must be 1 to 256");
  g10_rope_args a{};
  Maybe outs[2], dws[2];
  at::Tensor keep[6];
  int kept = 0;
  std::optional<at::ScalarType> wt;
  const Maybe *xs[2] = {&q, &k}, *ws[2] = {&q_weight, &k_weight}, *dys[2] = {&dq, &dk};
  const char *names[2] = {"q", "k"}, *wnames[2] = {"q_weight", "k_weight"}, *dnames[2] = {"dq", "dk"};
  for (int i = 0; i < 2; ++i) {
    g10_rope_part& part = a.part[i];
    if (!*xs[i]) {
      TORCH_CHECK_VALUE(!*ws[i], wnames[i], " without ", names[i]);
      continue;
    }
    const at::Tensor& given = **xs[i];
    on_device(given, names[i], &dev);
    TORCH_CHECK_VALUE(given.scalar_type() == dt && given.dim() == one.dim() && given.size(-1) == dim && given.sizes().slice(0, given.dim() - 2) == lead,
                      names[i], " must have the type, tokens and dim of q");
    const at::Tensor x = keep[kept++] = inner(given);
    part.heads = (uint32_t)x.size(-2);
    part.x = x.const_data_ptr();
    put_strides(part.x_stride, x);
    if (*ws[i]) {
      const at::Tensor& w = **ws[i];
      on_device(w, wnames[i], &dev);
      TORCH_CHECK_VALUE(w.dim() == 1 && w.size(0) == dim && (w.scalar_type() == dt || w.scalar_type() == at::kFloat), wnames[i],
                        " must be [dim], of the inputs' type or float32");
      TORCH_CHECK_VALUE(!wt || *wt == w.scalar_type(), "both weights must be of one type");
      wt = w.scalar_type();
      part.weight = (keep[kept++] = w.contiguous()).const_data_ptr();
    }
    if (back) {
      TORCH_CHECK_VALUE(*dys[i], dnames[i], " is needed");
      const at::Tensor& dy = **dys[i];
      on_device(dy, dnames[i], &dev);
      TORCH_CHECK_VALUE(dy.sizes() == x.sizes() && dy.scalar_type() == dt, dnames[i], " must have the shape and type of ", names[i]);
      const at::Tensor y = keep[kept++] = inner(dy);
      part.dy = y.const_data_ptr();
      put_strides(part.dy_stride, y);
      if (part.weight) {
        dws[i] = at::empty({dim}, at::TensorOptions().dtype(*wt).device(dev));
        part.dweight = dws[i]->mutable_data_ptr();
      }
    }
  }
  on_device(table, "table", &dev);
  TORCH_CHECK_VALUE(table.scalar_type() == at::kFloat && table.dim() == 2 && table.is_contiguous(), "table must be [positions, rot], float32, contiguous");
  const int64_t rot = table.size(1);
  TORCH_CHECK_VALUE(rot % 2 == 0 && rot <= dim, "the table's width must be even and at most dim");
  on_device(positions_in, "positions", &dev);
  const bool wide = positions_in.scalar_type() == at::kLong;
  TORCH_CHECK_VALUE((wide || positions_in.scalar_type() == at::kInt) && positions_in.sizes() == lead, "positions must be int32 or int64, one for each token");
  const at::Tensor positions = positions_in.contiguous();
  TORCH_CHECK_VALUE(eps >= 0 && std::isfinite(eps), "eps must not be negative");
  a.batch = (uint32_t)(lead.size() == 2 ? lead[0] : 1);
  a.seq = (uint32_t)lead[lead.size() - 1];
  TORCH_CHECK_VALUE(!a.batch || !a.seq || table.size(0) > 0, "the table has no positions");
  for (int i = 0; i < 2; ++i)
    if (*xs[i]) {
      outs[i] = at::empty((*xs[i])->sizes(), at::TensorOptions().dtype(dt).device(dev));
      a.part[i].out = outs[i]->mutable_data_ptr();
      put_strides(a.part[i].out_stride, *outs[i]);
    }
  a.dim = (uint32_t)dim; a.rot = (uint32_t)rot;
  a.table = table.const_data_ptr<float>();
  a.n_positions = (uint32_t)std::min<int64_t>(table.size(0), 0xffffffffll);
  a.positions = positions.const_data_ptr();
  a.eps = (float)eps;
  a.type = (uint32_t)type_of(dt);
  a.weight_type = (uint32_t)type_of(wt ? *wt : dt);
  a.flags = (interleaved ? G10_ROPE_INTERLEAVED : 0) | (wide ? G10_ROPE_POSITIONS_64 : 0);
  const c10::DeviceGuard guard(dev);
  if (!back) {
    check(lib.norm_rope(&a, stream_of(dev)), "g10_norm_rope");
    return py::make_tuple(outs[0], outs[1]);
  }
  uint64_t n = 0;
  check(lib.norm_rope_workspace(&a, &n), "g10_norm_rope_workspace");
  at::Tensor ws_mem;
  if (n) ws_mem = room(n, dev);
  check(lib.norm_rope_backward(&a, n ? ws_mem.mutable_data_ptr() : nullptr, n, stream_of(dev)), "g10_norm_rope_backward");
  return py::make_tuple(outs[0], outs[1], dws[0], dws[1]);
}

// ------------------------------------------------------------------------------------------------------------ attention
// The tensor as the kernels read it: rows and heads at multiples of 16 bytes, the last dimension contiguous; copied if it is not
// so already.
static at::Tensor rows16(const at::Tensor& t) {
  const int64_t d = t.dim();
  const auto s = t.strides(), n = t.sizes();
  bool fine = !((uintptr_t)t.const_data_ptr() & 15) && s[d - 1] == 1 && s[d - 3] >= 0 && s[d - 3] <= (1 << 22);
  for (int64_t i = 0; i + 1 < d; ++i) fine = fine && (s[i] % 8 == 0 || n[i] == 1);
  return fine || !t.numel() ? t : t.clone(at::MemoryFormat::Contiguous);
}
// (a dimension of one place is never stepped over: its stride may be anything)
static void put(const void*& p, int64_t (&to)[3], const at::Tensor& t) {
  p = t.numel() ? t.const_data_ptr() : nullptr;
  const int64_t d = t.dim();
  for (int i = 0; i < 3; ++i) {
    const int64_t at = d - 4 + i;
    to[i] = at >= 0 && t.size(at) > 1 ? t.stride(at) : 0;
  }
}
static void put(void*& p, int64_t (&to)[3], const at::Tensor& t) {
  const void* q;
  put(q, to, t);
  p = const_cast<void*>(q);
}

struct AttentionCall {
  g10_attention_args a{};
  at::Tensor q, k, v, starts[2], len;
  at::Device dev{at::kCPU};
  bool packed;
};

static at::Tensor whole_numbers(const at::Tensor& t, const char* name, const at::Device& dev) {
  on_device(t, name, &dev);
  TORCH_CHECK_VALUE(t.scalar_type() == at::kInt && t.dim() == 1, name, " must be a vector of int32");
  return t.contiguous();
}

static void attention_args(AttentionCall& c, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, bool causal, int64_t window, int64_t sinks,
                           std::optional<double> scale, const Maybe& q_start, const Maybe& k_start, const Maybe& k_len, std::optional<int64_t> max_q,
                           std::optional<int64_t> max_k) {
  on_device(q, "q", nullptr);
  c.dev = q.device();
  const at::ScalarType dt = q.scalar_type();
  TORCH_CHECK_VALUE(dt == at::kHalf || dt == at::kBFloat16, "type ", dt, " is not supported: float16 or bfloat16");
  on_device(k, "k", &c.dev);
  on_device(v, "v", &c.dev);
  TORCH_CHECK_VALUE(k.scalar_type() == dt && k.dim() == q.dim(), "k must have the type and dimensions of q");
  TORCH_CHECK_VALUE(v.scalar_type() == dt && v.dim() == q.dim(), "v must have the type and dimensions of q");
  const bool packed = c.packed = q_start || k_start;
  TORCH_CHECK_VALUE(q.dim() == (packed ? 3 : 4), "q, k and v are [batch, token, head, dim], packed sequences [token, head, dim]");
  const int64_t d = q.dim(), heads = q.size(d - 2), kv = k.size(d - 2), dim = q.size(d - 1);
  TORCH_CHECK_VALUE(k.sizes() == v.sizes() && k.size(d - 1) == dim, "k and v must have one shape, and the dim of q");
  TORCH_CHECK_VALUE(kv > 0 && heads > 0 && heads % kv == 0, "the heads of q must be a multiple of those of k");
  TORCH_CHECK_VALUE(dim > 0 && dim <= 128 && dim % 8 == 0, "dim must be a multiple of 8 up to 128");
  TORCH_CHECK_VALUE(window >= 0 && window < (1 << 30) && sinks >= 0 && sinks < (1 << 30), "window and sinks must not be negative");
  const double s = scale ? *scale : 1.0 / sqrt((double)dim);
  TORCH_CHECK_VALUE(s > 0 && s < 3e38, "scale must be above zero");
  g10_attention_args& a = c.a;
  TORCH_CHECK_VALUE(q.size(d - 3) < (1 << 30) && k.size(d - 3) < (1 << 30), "too many tokens");
  a.seq_q = (uint32_t)q.size(d - 3);
  a.seq_k = (uint32_t)k.size(d - 3);
  if (packed) {
    TORCH_CHECK_VALUE(q_start && k_start && !k_len, "packed sequences need q_start and k_start, and no k_len");
    c.starts[0] = whole_numbers(*q_start, "q_start", c.dev);
    c.starts[1] = whole_numbers(*k_start, "k_start", c.dev);
    TORCH_CHECK_VALUE(c.starts[0].numel() == c.starts[1].numel() && c.starts[0].numel() > 0, "q_start and k_start must hold a number for each sequence and the end");
    a.q_start = c.starts[0].const_data_ptr<int32_t>();
    a.k_start = c.starts[1].const_data_ptr<int32_t>();
    a.batch = (uint32_t)(c.starts[0].numel() - 1);
    auto most = [](std::optional<int64_t> m, uint32_t n) { return m ? (uint32_t)std::min<int64_t>(std::max<int64_t>(*m, 0), n) : n; };
    a.max_q = most(max_q, a.seq_q);
    a.max_k = most(max_k, a.seq_k);
  } else {
    TORCH_CHECK_VALUE(k.size(0) == q.size(0), "q and k must have one batch");
    a.batch = (uint32_t)q.size(0);
    if (k_len) {
      c.len = whole_numbers(*k_len, "k_len", c.dev);
      TORCH_CHECK_VALUE(c.len.numel() == q.size(0), "k_len must hold a number for each sequence");
      a.k_len = c.len.const_data_ptr<int32_t>();
    }
  }
  a.heads = (uint32_t)heads; a.kv_heads = (uint32_t)kv; a.dim = (uint32_t)dim;
  a.causal = causal; a.window = (uint32_t)window; a.sinks = (uint32_t)sinks;
  a.scale = (float)s;
  a.type = (uint32_t)type_of(dt);
  c.q = rows16(q); c.k = rows16(k); c.v = rows16(v);
  put(a.q, a.q_stride, c.q);
  put(a.k, a.k_stride, c.k);
  put(a.v, a.v_stride, c.v);
}

static py::tuple attention(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, bool causal, int64_t window, int64_t sinks, std::optional<double> scale,
                           const Maybe& q_start, const Maybe& k_start, const Maybe& k_len, std::optional<int64_t> max_q, std::optional<int64_t> max_k) {
  AttentionCall c;
  attention_args(c, q, k, v, causal, window, sinks, scale, q_start, k_start, k_len, max_q, max_k);
  g10_attention_args& a = c.a;
  const auto opt = at::TensorOptions().device(c.dev);
  at::Tensor o = at::empty(q.sizes(), opt.dtype(q.scalar_type()));
  at::Tensor lse = c.packed ? at::empty({a.heads, a.seq_q}, opt.dtype(at::kFloat)) : at::empty({a.batch, a.heads, a.seq_q}, opt.dtype(at::kFloat));
  if (!q.numel()) return py::make_tuple(o, lse);
  if (!a.batch) return py::make_tuple(o.zero_(), lse.fill_(-INFINITY));                // (rows, and no sequence)
  put(a.o, a.o_stride, o);
  a.lse = lse.mutable_data_ptr<float>();
  const c10::DeviceGuard guard(c.dev);
  uint64_t n = 0;
  check(lib.attention_workspace(&a, &n), "g10_attention_workspace");
  at::Tensor ws;
  if (n) ws = room(n, c.dev);
  check(lib.attention(&a, n ? ws.mutable_data_ptr() : nullptr, n, stream_of(c.dev)), "g10_attention");
  return py::make_tuple(o, lse);
}

static py::tuple attention_backward(const at::Tensor& d_o, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& o, const at::Tensor& lse,
                                    bool causal, int64_t window, int64_t sinks, std::optional<double> scale, const Maybe& q_start, const Maybe& k_start,
                                    const Maybe& k_len, std::optional<int64_t> max_q, std::optional<int64_t> max_k) {
  AttentionCall c;
  attention_args(c, q, k, v, causal, window, sinks, scale, q_start, k_start, k_len, max_q, max_k);
  g10_attention_args& a = c.a;
  on_device(d_o, "do", &c.dev);
  on_device(o, "o", &c.dev);
  on_device(lse, "lse", &c.dev);
  TORCH_CHECK_VALUE(d_o.sizes() == q.sizes() && d_o.scalar_type() == q.scalar_type(), "do must have the shape and type of q");
  TORCH_CHECK_VALUE(o.sizes() == q.sizes() && o.scalar_type() == q.scalar_type(), "o must have the shape and type of q");
  TORCH_CHECK_VALUE(lse.scalar_type() == at::kFloat && lse.is_contiguous() && lse.numel() == (int64_t)a.heads * a.seq_q * (c.packed ? 1 : a.batch), "lse must be g10_attention's");
  const auto opt = at::TensorOptions().device(c.dev).dtype(q.scalar_type());
  if (!q.numel() || !a.batch) return py::make_tuple(at::zeros(q.sizes(), opt), at::zeros(k.sizes(), opt), at::zeros(v.sizes(), opt));
  at::Tensor dq = at::empty(q.sizes(), opt), dk = at::empty(k.sizes(), opt), dv = at::empty(v.sizes(), opt);
  const at::Tensor g = rows16(d_o), out = rows16(o);
  put(a.d_o, a.do_stride, g);
  put(a.o, a.o_stride, out);
  put(a.dq, a.dq_stride, dq);
  put(a.dk, a.dk_stride, dk);
  put(a.dv, a.dv_stride, dv);
  a.lse = const_cast<float*>(lse.const_data_ptr<float>());
  const c10::DeviceGuard guard(c.dev);
  uint64_t n = 0;
  check(lib.attention_backward_workspace(&a, &n), "g10_attention_backward_workspace");
  at::Tensor ws = room(n, c.dev);
  check(lib.attention_backward(&a, ws.mutable_data_ptr(), n, stream_of(c.dev)), "g10_attention_backward");
  return py::make_tuple(dq, dk, dv);
}

// ---------------------------------------------------------------------------------------------------------------- AdamW
// The parameters of an AdamW, and the library's handle for them, made at the first step.
class AdamwCore {
 public:
  AdamwCore(std::vector<at::Tensor> params, std::vector<Maybe> copies, at::Tensor m, at::Tensor v, Maybe m_scale, Maybe v_scale)
      : params_(std::move(params)), copies_(std::move(copies)), m_(m), v_(v), ms_(m_scale), vs_(v_scale), dev_(params_.at(0).device()) {
    std::unordered_map<const c10::TensorImpl*, uint32_t> of;
    auto counter = [&](const at::Tensor& t) { return of.emplace((t.is_view() ? t._base() : t).unsafeGetTensorImpl(), (uint32_t)of.size()).first->second; };
    for (const at::Tensor& t : params_) params_counter_.push_back(counter(t));
    for (const Maybe& t : copies_) copies_counter_.push_back(t ? counter(*t) : 0);
    counted_.resize(of.size() + 1);
  }
  ~AdamwCore() { close(); }

  void close() {
    if (h_) lib.adamw_free(h_);
    h_ = nullptr;
  }

  // whether there was a gradient; the norm before clipping, or None
  py::tuple step(const py::object& grads, double lr, double beta1, double beta2, double eps, double decay, uint64_t number, std::optional<double> max_norm,
                  const Maybe& coefficient) {
    TORCH_CHECK_VALUE(!max_norm || *max_norm > 0, "max_norm must be above zero");
    TORCH_CHECK_VALUE(!max_norm || !coefficient, "max_norm or coefficient");
    if (coefficient) {
      on_device(*coefficient, "coefficient", &dev_);
      TORCH_CHECK_VALUE(coefficient->scalar_type() == at::kFloat && coefficient->numel() == 1, "coefficient must be one float32 number");
    }
    if (!gather(grads)) return py::make_tuple(false, max_norm ? py::cast(at::zeros({}, at::TensorOptions().dtype(at::kFloat).device(dev_))) : py::object(py::none()));
    const c10::DeviceGuard guard(dev_);
    handle();
    g10_adamw_params p{lr, beta1, beta2, eps, decay, number, coefficient ? coefficient->const_data_ptr<float>() : nullptr};
    at::Tensor norm;
    if (max_norm) {
      norm = norms(*max_norm);
      p.coefficient = norm.const_data_ptr<float>() + 1;
    }
    check(lib.adamw_step(h_, at_.data(), &p, stream_of(dev_)), "g10_adamw_step");
    // (written past autograd: a graph made before that still needs the values of then has to notice)
    ++calls_;
    for (size_t i = 0; i < params_.size(); ++i)
      if (at_[i]) {
        written(params_[i], params_counter_[i]);
        if (copies_[i]) written(*copies_[i], copies_counter_[i]);
      }
    keep_.clear();
    return py::make_tuple(true, max_norm ? py::cast(norm.select(0, 0)) : py::object(py::none()));
  }

  py::object grad_norm(const py::object& grads, double max_norm) {
    TORCH_CHECK_VALUE(max_norm > 0, "max_norm must be above zero");
    if (!gather(grads)) return py::cast(at::zeros({}, at::TensorOptions().dtype(at::kFloat).device(dev_)));
    const c10::DeviceGuard guard(dev_);
    handle();
    at::Tensor norm = norms(max_norm);
    keep_.clear();
    return py::cast(norm.select(0, 0));
  }

 private:
  std::vector<at::Tensor> params_;
  std::vector<Maybe> copies_;
  at::Tensor m_, v_;
  Maybe ms_, vs_;
  at::Device dev_;
  g10_adamw_t* h_ = nullptr;
  at::ScalarType made_for_ = at::kFloat;           // the gradients' type of the handle
  std::vector<const void*> at_;                    // of this call: the gradients' addresses, their type, copies that had to be made
  at::ScalarType type_ = at::kFloat;
  std::vector<at::Tensor> keep_;

  // Version counters: a buffer and its views share one, which is moved once a step (an atomic operation each time).
  std::vector<uint32_t> params_counter_, copies_counter_;
  std::vector<uint64_t> counted_;                  // the call that moved it last
  uint64_t calls_ = 0;
  void written(const at::Tensor& t, uint32_t counter) {
    if (counted_[counter] == calls_) return;
    counted_[counter] = calls_;
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  }

  at::Tensor norms(double max_norm) {
    at::Tensor norm = at::empty({2}, at::TensorOptions().dtype(at::kFloat).device(dev_));
    check(lib.grad_norm(h_, at_.data(), (float)std::min(max_norm, 3e38), norm.mutable_data_ptr<float>(), stream_of(dev_)), "g10_grad_norm");
    return norm;
  }

  // how many gradients there are
  size_t gather(const py::object& grads) {
    const size_t n = params_.size();
    size_t found = 0;
    keep_.clear();
    at_.assign(n, nullptr);
    auto take = [&](size_t i, const at::Tensor& g) {
      if (!g.defined()) return;
      if (!found++) {
        type_ = g.scalar_type();
        TORCH_CHECK_VALUE(type_of(type_) >= 0, "gradients of type ", type_, " are not supported");
      }
      TORCH_CHECK_VALUE(g.device() == dev_ && g.scalar_type() == type_ && g.sizes() == params_[i].sizes(), "grads[", i,
                        "] must have its parameter's shape and device and the type of the others");
      if (g.is_contiguous()) at_[i] = g.const_data_ptr();
      else {
        keep_.push_back(g.contiguous());
        at_[i] = keep_.back().const_data_ptr();
      }
    };
    if (grads.is_none()) {
      for (size_t i = 0; i < n; ++i) take(i, params_[i].grad());
    } else {
      const py::sequence list = py::isinstance<py::list>(grads) || py::isinstance<py::tuple>(grads) ? py::reinterpret_borrow<py::sequence>(grads) : py::sequence(py::list(grads));
      TORCH_CHECK_VALUE(list.size() == n, "grads must be one for each parameter");
      for (size_t i = 0; i < n; ++i) {
        PyObject* g = PySequence_Fast_GET_ITEM(list.ptr(), (Py_ssize_t)i);
        if (g == Py_None) continue;
        TORCH_CHECK_VALUE(THPVariable_Check(g), "grads[", i, "] must be a tensor or None");
        take(i, THPVariable_Unpack(g));
      }
    }
    return found;
  }

  // Where a tensor lies: its memory and its place in it, without data_ptr's checks (a step of 300 small tensors takes as long as they do).
  typedef std::pair<const void*, int64_t> Place;
  static Place place_of(const at::Tensor& t) {
    const c10::TensorImpl* p = t.unsafeGetTensorImpl();
    return {p->unsafe_storage().unsafeGetStorageImpl()->data(), p->storage_offset()};
  }
  // what the library's tables point to
  std::vector<Place> places_;                      // of the handle
  template <class F>
  void each_place(F&& f) const {
    for (size_t i = 0; i < params_.size(); ++i) {
      f(params_[i], "params[", i);
      if (copies_[i]) f(*copies_[i], "copies[", i);
    }
    const at::Tensor* state[4] = {&m_, &v_, ms_ ? &*ms_ : nullptr, vs_ ? &*vs_ : nullptr};
    for (size_t i = 0; i < 4; ++i)
      if (state[i]) f(*state[i], "state[", i);
  }

  void handle() {
    if (h_) {
      TORCH_CHECK_VALUE(type_ == made_for_, "the gradients' type changed");
      size_t k = 0;
      each_place([&](const at::Tensor& t, const char* what, size_t i) {
        TORCH_CHECK_VALUE(place_of(t) == places_[k], what, i, "] has moved: its memory must stay in place until close()");
        ++k;
      });
      return;
    }
    // (it allocates, copies from host memory that it then frees, and waits)
    TORCH_CHECK_VALUE(c10::hip::currentStreamCaptureStatusMayInitCtx() == c10::hip::CaptureStatus::None,
                      "the first step or norm makes the library's tables, which a graph cannot hold: make one before the capture");
    std::vector<g10_adamw_tensor> ts(params_.size());
    int copy_type = 0;
    for (size_t i = 0; i < ts.size(); ++i) {
      ts[i].n = (uint64_t)params_[i].numel();
      ts[i].p = ts[i].n ? params_[i].data_ptr() : nullptr;
      ts[i].copy = copies_[i] && ts[i].n ? copies_[i]->data_ptr() : nullptr;
      if (copies_[i]) copy_type = type_of(copies_[i]->scalar_type());
    }
    g10_adamw_desc d{};
    d.tensors = ts.data(); d.count = (uint32_t)ts.size();
    d.type = (uint32_t)type_of(params_[0].scalar_type()); d.grad_type = (uint32_t)type_of(type_); d.copy_type = (uint32_t)copy_type;
    d.state_type = ms_ ? G10_E4M3 : G10_F32;
    d.m = m_.numel() ? m_.data_ptr() : nullptr;
    d.v = v_.numel() ? v_.data_ptr() : nullptr;
    if (ms_ && m_.numel()) { d.m_scale = ms_->data_ptr<float>(); d.v_scale = vs_->data_ptr<float>(); }
    check(lib.adamw_create(&d, stream_of(dev_), &h_), "g10_adamw_create");
    made_for_ = type_;
    places_.clear();
    each_place([&](const at::Tensor& t, const char*, size_t) { places_.push_back(place_of(t)); });
  }
};

PYBIND11_MODULE(_g10_torch, m) {
  m.def("bind", &bind);
  m.def("norm_rope", &norm_rope);
  m.def("attention", &attention);
  m.def("attention_backward", &attention_backward);
  py::class_<AdamwCore>(m, "AdamwCore")
      .def(py::init<std::vector<at::Tensor>, std::vector<Maybe>, at::Tensor, at::Tensor, Maybe, Maybe>())
      .def("step", &AdamwCore::step)
      .def("grad_norm", &AdamwCore::grad_norm)
      .def("close", &AdamwCore::close);
}
