// Marshalling of the operators around attention: embeddings, norms of rows, gated MLP, log probabilities.
#include "g10_torch.h"

static struct {
  decltype(&g10_embed) embed;
  decltype(&g10_embed_backward_workspace) embed_backward_workspace;
  decltype(&g10_embed_backward) embed_backward;
  decltype(&g10_norm) norm;
  decltype(&g10_norm_backward_workspace) norm_backward_workspace;
  decltype(&g10_norm_backward) norm_backward;
  decltype(&g10_log_probs_workspace) log_probs_workspace;
  decltype(&g10_log_probs) log_probs;
  decltype(&g10_log_probs_backward) log_probs_backward;
  decltype(&g10_gated_workspace) gated_workspace;
  decltype(&g10_gated) gated;
  decltype(&g10_gated_backward_workspace) gated_backward_workspace;
  decltype(&g10_gated_backward) gated_backward;
} lib;

static void bind_layer(const std::vector<uintptr_t>& at) {
  TORCH_CHECK_VALUE(at.size() == 13, "thirteen addresses");
  size_t i = 0;
  auto next = [&](auto& f) { f = (std::decay_t<decltype(f)>)at[i++]; };
  next(lib.embed); next(lib.embed_backward_workspace); next(lib.embed_backward);
  next(lib.norm); next(lib.norm_backward_workspace); next(lib.norm_backward);
  next(lib.log_probs_workspace); next(lib.log_probs); next(lib.log_probs_backward);
  next(lib.gated_workspace); next(lib.gated); next(lib.gated_backward_workspace); next(lib.gated_backward);
}

static at::Tensor empty(at::IntArrayRef sizes, at::ScalarType t, const at::Device& dev) { return at::empty(sizes, at::TensorOptions().dtype(t).device(dev)); }

// [..., width] as [rows, width] with the last dimension contiguous; copied where no strides say so.
static at::Tensor rows_of(const at::Tensor& t) {
  const int64_t width = t.size(-1);
  int64_t rows = 1;
  for (int64_t i = 0; i + 1 < t.dim(); ++i) rows *= t.size(i);
  const at::Tensor r = t.dim() == 2 ? t : t.reshape({rows, width});
  return r.stride(1) == 1 || width <= 1 ? r : r.contiguous();
}
static int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }

static at::ScalarType float_type(const at::Tensor& t, const char* name) {
  on_device(t, name, nullptr);
  TORCH_CHECK_VALUE(type_of(t.scalar_type()) >= 0, "type ", t.scalar_type(), " is not supported: float32, float16 or bfloat16");
  TORCH_CHECK_VALUE(t.dim() >= 1 && t.size(-1) > 0, name, " must have values in its last dimension");
  return t.scalar_type();
}

static at::Tensor workspace(uint64_t n, const at::Device& dev) { return n ? room(n, dev) : at::Tensor(); }
static void* at_of(const at::Tensor& t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }
static const void* in_of(const at::Tensor& t) { return t.numel() ? t.const_data_ptr() : nullptr; }

// ----------------------------------------------------------------------------------------------------------- embeddings
static at::Tensor whole_ids(const at::Tensor& ids, const at::Device& dev) {
  on_device(ids, "ids", &dev);
  TORCH_CHECK_VALUE(ids.scalar_type() == at::kInt || ids.scalar_type() == at::kLong, "ids must be int32 or int64");
  TORCH_CHECK_VALUE(ids.numel() < 0x80000000ll, "too many tokens");
  return ids.contiguous();
}

static at::Tensor embed(const at::Tensor& ids_in, const at::Tensor& table_in, double scale) {
  const at::ScalarType dt = float_type(table_in, "table");
  const at::Device dev = table_in.device();
  TORCH_CHECK_VALUE(table_in.dim() == 2 && table_in.size(0) > 0, "table must be [rows, dim]");
  TORCH_CHECK_VALUE(std::isfinite(scale), "scale must be finite");
  const at::Tensor ids = whole_ids(ids_in, dev), table = rows_of(table_in);
  std::vector<int64_t> sizes = ids.sizes().vec();
  sizes.push_back(table.size(1));
  at::Tensor out = empty(sizes, dt, dev);
  g10_embed_args a{};
  a.ids = in_of(ids); a.table = table.const_data_ptr(); a.out = out.numel() ? out.mutable_data_ptr() : nullptr;
  a.table_stride = row_stride(table); a.out_stride = table.size(1);
  a.tokens = (uint32_t)ids.numel();
  TORCH_CHECK_VALUE(table.size(0) < 0x80000000ll && table.size(1) <= 65536, "table must have fewer than 2^31 rows of up to 65536 values");
  a.vocab = (uint32_t)table.size(0); a.dim = (uint32_t)table.size(1);
  a.scale = (float)scale; a.type = (uint32_t)type_of(dt); a.ids_64 = ids.scalar_type() == at::kLong;
  const c10::DeviceGuard guard(dev);
  check(lib.embed(&a, stream_of(dev)), "g10_embed");
  return out;
}

static at::Tensor embed_backward(const at::Tensor& dout_in, const at::Tensor& ids_in, int64_t rows, double scale) {
  const at::ScalarType dt = float_type(dout_in, "dout");
  const at::Device dev = dout_in.device();
  TORCH_CHECK_VALUE(std::isfinite(scale), "scale must be finite");
  const at::Tensor ids = whole_ids(ids_in, dev);
  TORCH_CHECK_VALUE(dout_in.dim() == ids.dim() + 1 && dout_in.sizes().slice(0, ids.dim()) == ids.sizes(), "dout must have a row for each id");
  TORCH_CHECK_VALUE(rows > 0 && rows < 0x80000000ll && dout_in.size(-1) <= 65536, "the table must have 1 to 2^31 - 1 rows of up to 65536 values");
  const at::Tensor dout = rows_of(dout_in);
  at::Tensor dtable = empty({rows, dout.size(1)}, dt, dev);
  g10_embed_args a{};
  a.ids = in_of(ids); a.dout = in_of(dout); a.dtable = dtable.mutable_data_ptr();
  a.dout_stride = row_stride(dout); a.dtable_stride = dout.size(1);
  a.tokens = (uint32_t)ids.numel(); a.vocab = (uint32_t)rows; a.dim = (uint32_t)dout.size(1);
  a.scale = (float)scale; a.type = (uint32_t)type_of(dt); a.ids_64 = ids.scalar_type() == at::kLong;
  const c10::DeviceGuard guard(dev);
  uint64_t n = 0;
  check(lib.embed_backward_workspace(&a, &n), "g10_embed_backward_workspace");
  const at::Tensor ws = workspace(n, dev);
  check(lib.embed_backward(&a, at_of(ws), n, stream_of(dev)), "g10_embed_backward");
  return dtable;
}

// -------------------------------------------------------------------------------------------------------- norms of rows
static py::tuple norm(const at::Tensor& x_in, const Maybe& weight, const Maybe& bias, double eps, bool center, bool back, const Maybe& dy_in) {
  const at::ScalarType dt = float_type(x_in, "x");
  const at::Device dev = x_in.device();
  const int64_t dim = x_in.size(-1);
  TORCH_CHECK_VALUE(dim <= 65536, "rows must have up to 65536 values");
  TORCH_CHECK_VALUE(x_in.numel() / dim < 0x80000000ll, "too many rows");
  TORCH_CHECK_VALUE(eps >= 0 && std::isfinite(eps), "eps must not be negative");
  g10_norm_args a{};
  std::optional<at::ScalarType> wt;
  at::Tensor ws[2];
  Maybe dws[2];
  const Maybe* given[2] = {&weight, &bias};
  const char* names[2] = {"weight", "bias"};
  for (int i = 0; i < 2; ++i) {
    if (!*given[i]) continue;
    const at::Tensor& w = **given[i];
    on_device(w, names[i], &dev);
    TORCH_CHECK_VALUE(w.dim() == 1 && w.size(0) == dim && (w.scalar_type() == dt || w.scalar_type() == at::kFloat), names[i],
                      " must be [dim], of the inputs' type or float32");
    TORCH_CHECK_VALUE(!wt || *wt == w.scalar_type(), "weight and bias must be of one type");
    wt = w.scalar_type();
    ws[i] = w.contiguous();
    if (back) dws[i] = empty({dim}, *wt, dev);
  }
  const at::Tensor x = rows_of(x_in);
  at::Tensor dy, out = empty(x_in.sizes(), dt, dev);
  if (back) {
    TORCH_CHECK_VALUE(dy_in, "dy is needed");
    on_device(*dy_in, "dy", &dev);
    TORCH_CHECK_VALUE(dy_in->sizes() == x_in.sizes() && dy_in->scalar_type() == dt, "dy must have the shape and type of x");
    dy = rows_of(*dy_in);
    a.dy = in_of(dy);
    a.dy_stride = row_stride(dy);
  }
  a.x = in_of(x); a.out = out.numel() ? out.mutable_data_ptr() : nullptr;
  a.weight = ws[0].defined() ? ws[0].const_data_ptr() : nullptr;
  a.bias = ws[1].defined() ? ws[1].const_data_ptr() : nullptr;
  a.dweight = dws[0] ? dws[0]->mutable_data_ptr() : nullptr;
  a.dbias = dws[1] ? dws[1]->mutable_data_ptr() : nullptr;
  a.x_stride = row_stride(x); a.out_stride = dim;
  a.rows = (uint32_t)x.size(0); a.dim = (uint32_t)dim;
  a.eps = (float)eps; a.center = center;
  a.type = (uint32_t)type_of(dt); a.weight_type = (uint32_t)type_of(wt ? *wt : dt);
  const c10::DeviceGuard guard(dev);
  if (!back) {
    check(lib.norm(&a, stream_of(dev)), "g10_norm");
    return py::make_tuple(out);
  }
  uint64_t n = 0;
  check(lib.norm_backward_workspace(&a, &n), "g10_norm_backward_workspace");
  const at::Tensor mem = workspace(n, dev);
  check(lib.norm_backward(&a, at_of(mem), n, stream_of(dev)), "g10_norm_backward");
  return py::make_tuple(out, dws[0], dws[1]);
}

// ---------------------------------------------------------------------------------------------------- log probabilities
struct LogProbsCall {
  g10_log_probs_args a{};
  at::Tensor logits, tokens;
  at::Device dev{at::kCPU};
  std::vector<int64_t> lead;
};
static void log_probs_args(LogProbsCall& c, const at::Tensor& logits, const Maybe& tokens, double scale, int64_t ignore) {
  const at::ScalarType dt = float_type(logits, "logits");
  c.dev = logits.device();
  c.lead = logits.sizes().slice(0, logits.dim() - 1).vec();
  TORCH_CHECK_VALUE(scale > 0 && scale <= 2e38, "scale must be above zero, up to 2e38");
  TORCH_CHECK_VALUE(logits.size(-1) < 0x80000000ll && logits.numel() / logits.size(-1) < 0x80000000ll, "too many rows or logits in one");
  c.logits = rows_of(logits);
  g10_log_probs_args& a = c.a;
  if (tokens) {
    on_device(*tokens, "tokens", &c.dev);
    TORCH_CHECK_VALUE(tokens->scalar_type() == at::kLong || tokens->scalar_type() == at::kInt, "tokens must be int64 or int32");
    TORCH_CHECK_VALUE(tokens->sizes() == at::IntArrayRef(c.lead), "tokens must be one for each row of logits");
    c.tokens = tokens->to(at::kLong).contiguous();
    a.tokens = c.tokens.numel() ? c.tokens.const_data_ptr<int64_t>() : nullptr;
  }
  a.logits = in_of(c.logits);
  a.logits_stride = row_stride(c.logits);
  a.rows = (uint32_t)c.logits.size(0); a.vocab = (uint32_t)c.logits.size(1);
  a.scale = (float)scale; a.ignore = ignore;
  a.type = (uint32_t)type_of(dt);
}

static py::tuple log_probs(const at::Tensor& logits, const Maybe& tokens, bool entropy, int64_t top, double scale, int64_t ignore) {
  LogProbsCall c;
  log_probs_args(c, logits, tokens, scale, ignore);
  g10_log_probs_args& a = c.a;
  TORCH_CHECK_VALUE(top >= 0 && top <= (int64_t)G10_LOG_PROBS_TOP && top <= (int64_t)a.vocab, "top must be 0 to ", G10_LOG_PROBS_TOP, ", and no more than there are tokens");
  at::Tensor lse = empty(c.lead, at::kFloat, c.dev);
  Maybe logp, ent, top_logp, top_ids;
  a.lse = lse.mutable_data_ptr<float>();
  if (tokens) {
    logp = empty(c.lead, at::kFloat, c.dev);
    a.logp = logp->mutable_data_ptr<float>();
  }
  if (entropy) {
    ent = empty(c.lead, at::kFloat, c.dev);
    a.entropy = ent->mutable_data_ptr<float>();
  }
  if (top) {
    std::vector<int64_t> sizes = c.lead;
    sizes.push_back(top);
    top_logp = empty(sizes, at::kFloat, c.dev);
    top_ids = empty(sizes, at::kLong, c.dev);
    a.top = (uint32_t)top;
    a.top_logp = top_logp->mutable_data_ptr<float>();
    a.top_ids = top_ids->mutable_data_ptr<int64_t>();
  }
  const c10::DeviceGuard guard(c.dev);
  uint64_t n = 0;
  check(lib.log_probs_workspace(&a, &n), "g10_log_probs_workspace");
  const at::Tensor ws = workspace(n, c.dev);
  check(lib.log_probs(&a, at_of(ws), n, stream_of(c.dev)), "g10_log_probs");
  return py::make_tuple(logp, lse, ent, top_logp, top_ids);
}

static at::Tensor log_probs_backward(const Maybe& dlogp, const at::Tensor& logits, const Maybe& tokens, const at::Tensor& lse, const Maybe& dentropy, const Maybe& entropy,
                                     double scale, int64_t ignore) {
  LogProbsCall c;
  log_probs_args(c, logits, tokens, scale, ignore);
  g10_log_probs_args& a = c.a;
  TORCH_CHECK_VALUE(!dlogp || tokens, "dlogp without tokens");
  TORCH_CHECK_VALUE(!dentropy || entropy, "dentropy without g10_log_probs's entropy");
  at::Tensor keep[4];
  int kept = 0;
  auto number = [&](const at::Tensor& t, const char* name) {
    on_device(t, name, &c.dev);
    TORCH_CHECK_VALUE(t.scalar_type() == at::kFloat && t.sizes() == at::IntArrayRef(c.lead), name, " must be float32, one number for each row of logits");
    return (keep[kept++] = t.contiguous()).const_data_ptr<float>();
  };
  a.lse = const_cast<float*>(number(lse, "lse"));
  if (dlogp) a.dlogp = number(*dlogp, "dlogp");
  if (dentropy) {
    a.dentropy = number(*dentropy, "dentropy");
    a.entropy = const_cast<float*>(number(*entropy, "entropy"));
  }
  at::Tensor out = empty(logits.sizes(), logits.scalar_type(), c.dev);
  a.dlogits = out.numel() ? out.mutable_data_ptr() : nullptr;
  a.dlogits_stride = logits.size(-1);
  const c10::DeviceGuard guard(c.dev);
  check(lib.log_probs_backward(&a, stream_of(c.dev)), "g10_log_probs_backward");
  return out;
}

// ----------------------------------------------------------------------------------------------------------- gated MLP
struct GatedCall {
  g10_gated_args a{};
  at::Tensor x, w[2];
  at::Device dev{at::kCPU};
};
static void gated_args(GatedCall& c, const at::Tensor& x, const at::Tensor& gate, const at::Tensor& up, const std::string& act) {
  const at::ScalarType dt = float_type(x, "x");
  c.dev = x.device();
  TORCH_CHECK_VALUE(dt == at::kHalf || dt == at::kBFloat16, "type ", dt, " is not supported: float16 or bfloat16");
  on_device(gate, "gate", &c.dev);
  on_device(up, "up", &c.dev);
  TORCH_CHECK_VALUE(gate.dim() == 2 && gate.size(0) == x.size(-1) && gate.size(1) > 0 && gate.scalar_type() == dt, "gate must be [dim, inner], of the type of x");
  TORCH_CHECK_VALUE(up.sizes() == gate.sizes() && up.scalar_type() == dt, "up must have the shape and type of gate");
  TORCH_CHECK_VALUE(act == "silu" || act == "gelu", "act must be silu or gelu");
  const int64_t dim = x.size(-1), inner = gate.size(1), tokens = x.numel() / dim;
  TORCH_CHECK_VALUE(dim <= 1 << 20 && inner <= 1 << 20 && tokens < 0x80000000ll, "dim and inner must be up to 2^20, tokens below 2^31");
  const bool out_in = gate.stride(1) != 1 && gate.stride(0) == 1;                  // a linear layer's weight, transposed
  auto rows = [](const at::Tensor& t) { return (t.stride(1) == 1 || t.size(1) == 1) && row_stride(t) >= t.size(1) ? t : t.contiguous(); };
  c.w[0] = rows(out_in ? gate.t() : gate);
  c.w[1] = rows(out_in ? up.t() : up);
  c.x = rows(rows_of(x));
  g10_gated_args& a = c.a;
  a.x = in_of(c.x); a.gate = c.w[0].const_data_ptr(); a.up = c.w[1].const_data_ptr();
  a.x_stride = row_stride(c.x); a.gate_stride = row_stride(c.w[0]); a.up_stride = row_stride(c.w[1]);
  a.tokens = (uint32_t)tokens; a.dim = (uint32_t)dim; a.inner = (uint32_t)inner;
  a.act = act == "silu" ? G10_ACT_SILU : G10_ACT_GELU;
  a.out_in = out_in;
  a.type = (uint32_t)type_of(dt);
}
static std::vector<int64_t> with_last(const at::Tensor& x, int64_t n) {
  std::vector<int64_t> s = x.sizes().vec();
  s.back() = n;
  return s;
}

static at::Tensor gated(const at::Tensor& x, const at::Tensor& gate, const at::Tensor& up, const std::string& act) {
  GatedCall c;
  gated_args(c, x, gate, up, act);
  g10_gated_args& a = c.a;
  at::Tensor h = empty(with_last(x, a.inner), x.scalar_type(), c.dev);
  a.h = h.numel() ? h.mutable_data_ptr() : nullptr;
  a.h_stride = a.inner;
  const c10::DeviceGuard guard(c.dev);
  uint64_t n = 0;
  check(lib.gated_workspace(&a, &n), "g10_gated_workspace");
  const at::Tensor ws = workspace(n, c.dev);
  check(lib.gated(&a, at_of(ws), n, stream_of(c.dev)), "g10_gated");
  return h;
}

static py::tuple gated_backward(const at::Tensor& dh_in, const at::Tensor& x, const at::Tensor& gate, const at::Tensor& up, const std::string& act) {
  GatedCall c;
  gated_args(c, x, gate, up, act);
  g10_gated_args& a = c.a;
  on_device(dh_in, "dh", &c.dev);
  TORCH_CHECK_VALUE(dh_in.sizes() == at::IntArrayRef(with_last(x, a.inner)) && dh_in.scalar_type() == x.scalar_type(), "dh must have the shape and type of h");
  at::Tensor dh = rows_of(dh_in);
  if (row_stride(dh) < dh.size(1)) dh = dh.contiguous();                           // (a row for all tokens)
  at::Tensor dx = empty(x.sizes(), x.scalar_type(), c.dev), dw[2];
  for (at::Tensor& t : dw) t = empty(c.w[0].sizes(), x.scalar_type(), c.dev);
  a.dh = in_of(dh); a.dx = dx.numel() ? dx.mutable_data_ptr() : nullptr;
  a.dgate = dw[0].mutable_data_ptr(); a.dup = dw[1].mutable_data_ptr();
  a.dh_stride = row_stride(dh); a.dx_stride = a.dim; a.dw_stride = c.w[0].size(1);
  const c10::DeviceGuard guard(c.dev);
  uint64_t n = 0;
  check(lib.gated_backward_workspace(&a, &n), "g10_gated_backward_workspace");
  const at::Tensor ws = workspace(n, c.dev);
  check(lib.gated_backward(&a, at_of(ws), n, stream_of(c.dev)), "g10_gated_backward");
  return py::make_tuple(dx, a.out_in ? dw[0].t() : dw[0], a.out_in ? dw[1].t() : dw[1]);
}

void layer_calls(py::module_& m) {
  m.def("bind_layer", &bind_layer);
  m.def("embed", &embed);
  m.def("embed_backward", &embed_backward);
  m.def("norm", &norm);
  m.def("log_probs", &log_probs);
  m.def("log_probs_backward", &log_probs_backward);
  m.def("gated", &gated);
  m.def("gated_backward", &gated_backward);
}
