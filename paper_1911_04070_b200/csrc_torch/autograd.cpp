// The position-wise operators and those at the ends of a language model as PyTorch functions with gradients, in C++ over the C ABI
// of include/bpt.h: argument checks, memory from PyTorch, the current stream, and the autograd nodes.  What layer.residual_norm,
// layer.gated_feed_forward, layer.token_states, layer.clip_gradients and layer.adjust_logits call.
//
// A Python autograd function around the ctypes binding costs 130 to 160 us of host time a training step whatever the size, of
// which PyTorch's engine takes about 40; single tokens and short sequences are bound by that.
//
// Functions return None for arguments that the operators refuse; the caller then goes through binding.py, which says why.
#include <ATen/cuda/CUDAContext.h>
#include <ATen/cuda/CUDAGraphsUtils.cuh>
#include <c10/cuda/CUDAGuard.h>
#include <torch/csrc/autograd/functions/accumulate_grad.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/extension.h>

#include <algorithm>
#include <functional>
#include <unordered_set>

#include "../../include/bpt.h"

// What this file was compiled against; build.py reads it from the shared object without loading that.
extern "C" __attribute__((used, visibility("default"))) const char bpt_torch_key[] = "BPT_TORCH_KEY:" BPT_TORCH_KEY;

namespace py = pybind11;
using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

namespace {

struct Api {
    decltype(&bpt_res_norm_fwd) res_norm_fwd = nullptr;
    decltype(&bpt_res_norm_bwd_workspace_bytes) res_norm_bytes = nullptr;
    decltype(&bpt_res_norm_bwd) res_norm_bwd = nullptr;
    decltype(&bpt_gated_ff_few_rows) few_rows = nullptr;
    decltype(&bpt_gated_ff_workspace_bytes) gated_ff_bytes = nullptr;
    decltype(&bpt_gated_ff_fwd) gated_ff_fwd = nullptr;
    decltype(&bpt_gated_ff_bwd) gated_ff_bwd = nullptr;
    decltype(&bpt_embed_fwd) embed_fwd = nullptr;
    decltype(&bpt_embed_bwd_workspace_bytes) embed_bytes = nullptr;
    decltype(&bpt_embed_bwd) embed_bwd = nullptr;
    decltype(&bpt_grad_norm_workspace_bytes) grad_norm_bytes = nullptr;
    decltype(&bpt_grad_norm) grad_norm = nullptr;
    decltype(&bpt_clip_grads) clip_grads = nullptr;
    decltype(&bpt_adjust_logits) adjust_logits = nullptr;
    decltype(&bpt_adjust_logits_workspace_bytes) adjust_logits_bytes = nullptr;
} api;   // of the library that binding.py has loaded

struct Refused {};

void* ptr(const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
bool is_like(const Tensor& t, const Tensor& h) {
    return t.sizes() == h.sizes() && t.scalar_type() == h.scalar_type() && t.device() == h.device() && t.is_contiguous();
}
bool type_code(const Tensor& t, bpt_dtype* out) {
    *out = t.scalar_type() == at::kFloat ? BPT_F32 : BPT_BF16;
    return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16;
}
// Contiguous and on a 16-byte boundary, which the feed-forward kernels' loads need: a contiguous view, such as the gradient that the
// backward of a concatenation hands down, starts anywhere in its storage and is copied here.
Tensor aligned(const Tensor& t) {
    const Tensor c = t.contiguous();
    return c.is_cuda() && ((uintptr_t)c.data_ptr() & 15) ? c.clone() : c;
}
Tensor bytes(int64_t n, const Tensor& like) { return at::empty({n}, like.options().dtype(at::kByte)); }
// A leaf's accumulation node belongs to the stream on which a graph first reached the leaf, and lives as long as such a graph.
// Where that was the default stream, a backward pass under capture would have PyTorch wait there for an event of the capture,
// which breaks the capture off and can end the process: refused here, while the capture is whole.  Every leaf
// that this pass goes on to from the call's node, through whatever lies between (the call's own copy of a strided weight, a cast);
// leaves that the pass is not asked for are not reached and do not count.
void check_capture(const char* name) {
    if (at::cuda::currentStreamCaptureStatus() == at::cuda::CaptureStatus::None) return;
    const auto self = torch::autograd::get_current_node();
    if (!self) return;
    std::vector<torch::autograd::Node*> open{self.get()};
    std::unordered_set<torch::autograd::Node*> seen;
    while (!open.empty()) {
        torch::autograd::Node* node = open.back();
        open.pop_back();
        for (uint32_t i = 0; i < node->num_outputs(); ++i) {
            torch::autograd::Node* next = node->next_edge(i).function.get();
            if (!node->task_should_compute_output(i) || !seen.insert(next).second) continue;
            if (!dynamic_cast<torch::autograd::AccumulateGrad*>(next)) {
                open.push_back(next);
                continue;
            }
            const auto s = next->stream();
            TORCH_CHECK(!s.has_value() || at::cuda::CUDAStream(*s).stream() != nullptr, name,
                        " backward under capture: a graph of the same leaves, made on the default stream, is still alive; delete its outputs before the capture");
        }
    }
}
// A call past the autograd function (no argument requires a gradient) would drop a forward-mode tangent without a word, and the
// function itself has no forward-mode derivative.
void check_tangents(std::initializer_list<const Tensor*> args, const char* name) {
    for (const Tensor* t : args)
        TORCH_CHECK_NOT_IMPLEMENTED(!t->defined() || !t->_fw_grad(0).defined(), name, " has no forward-mode derivative");
}
// A trace records PyTorch's operators: of a call here only the allocation of the result, which nothing would then write.
void check_tracing(const char* name) {
    TORCH_CHECK_NOT_IMPLEMENTED(!torch::jit::tracer::isTracing(), name, " cannot be traced by torch.jit: the library's kernels leave no record");
}
// Gradients of a first-order node: asking for their gradient again is an error when it is done, as with any such function.
variable_list first_order_only(variable_list grads, const char* name) {
    if (!at::GradMode::is_enabled()) return grads;
    variable_list vars;
    for (auto& g : grads)
        if (g.defined()) vars.push_back(g);
    if (vars.empty()) return grads;
    for (auto& v : vars) v.set_requires_grad(true);
    auto fn = std::make_shared<torch::autograd::DelayedError>(std::string(name) + " can be differentiated once only", (int64_t)vars.size());
    vars = (*fn)(std::move(vars));
    size_t i = 0;
    for (auto& g : grads)
        if (g.defined()) g = vars[i++];
    return grads;
}

// ---------------------------------------------------------------------------------------------------------
// r = alpha h + gate post(b),  y = norm(r)
// ---------------------------------------------------------------------------------------------------------
struct NormCfg { int64_t norm, post; double alpha, eps; };

bool norm_args(const Tensor& h, const Tensor& b, const Tensor (&par)[4], const Tensor& gate, const NormCfg& cfg, bpt_res_norm_args* a) {
    *a = bpt_res_norm_args{};
    if (!h.is_cuda() || h.dim() < 1 || !h.is_contiguous() || !type_code(h, &a->dtype)) return false;
    const int64_t D = h.size(-1);
    if (D < 1 || D > INT32_MAX) return false;
    if (b.defined() ? !is_like(b, h) : (cfg.post != 0 || gate.defined())) return false;
    const void** slot[4] = {&a->weight, &a->bias, &a->post_weight, &a->post_bias};
    a->param_dtype = a->gate_dtype = a->dtype;
    at::ScalarType type = at::kFloat;
    bool any = false;
    for (int i = 0; i < 4; ++i) {
        const Tensor& t = par[i];
        if (!t.defined()) continue;
        if ((i < 2 ? cfg.norm : cfg.post) == 0 || t.dim() != 1 || t.size(0) != D || t.device() != h.device() || !t.is_contiguous()) return false;
        if (any && t.scalar_type() != type) return false;
        if (!type_code(t, &a->param_dtype)) return false;
        type = t.scalar_type();
        any = true;
        *slot[i] = t.data_ptr();
    }
    a->gate_groups = 1;
    if (gate.defined()) {       // a leading part of h's axes, the others of length one (or missing in front: [D])
        const int64_t n = h.dim(), missing = n - gate.dim();
        if (missing < 0 || gate.dim() < 1 || gate.size(-1) != D || gate.device() != h.device() || !gate.is_contiguous() || !type_code(gate, &a->gate_dtype))
            return false;
        auto axis = [&](int64_t i) { return i < missing ? 1 : gate.size(i - missing); };
        int64_t lead = n - 1;
        while (lead > 0 && axis(lead - 1) == 1) --lead;
        for (int64_t i = 0; i < lead; ++i) {
            if (axis(i) != h.size(i)) return false;
            a->gate_groups *= axis(i);
        }
        if (a->gate_groups < 1) a->gate_groups = 1;
        a->gate = gate.data_ptr();
    }
    a->rows = h.numel() / D;
    a->D = (int32_t)D;
    a->norm = (int32_t)cfg.norm;
    a->post_norm = (int32_t)cfg.post;
    a->alpha = (float)cfg.alpha;
    a->eps = (float)cfg.eps;
    a->h = h.data_ptr();
    a->b = ptr(b);
    return true;
}
// (r, y): undefined where not wanted
std::pair<Tensor, Tensor> norm_fwd(const Tensor& h, const Tensor& b, const Tensor (&par)[4], const Tensor& gate, const NormCfg& cfg, bool want_sum,
                                   Tensor* stats) {
    bpt_res_norm_args a;
    if (!norm_args(h, b, par, gate, cfg, &a)) throw Refused{};
    const c10::cuda::CUDAGuard guard(h.device());
    Tensor y, r;
    if (cfg.norm) y = at::empty_like(h);
    if (want_sum || !cfg.norm) r = at::empty_like(h);
    if (stats) *stats = at::empty({a.rows, 4}, h.options().dtype(at::kFloat));
    if (api.res_norm_fwd(&a, ptr(y), ptr(r), stats ? (float*)stats->data_ptr() : nullptr, at::cuda::getCurrentCUDAStream().stream()) != BPT_OK)
        throw Refused{};
    return {r, y};
}

using Opt = std::optional<Tensor>;
Opt given(const Opt& t) { return t.has_value() && t->defined() ? Opt(t->contiguous()) : Opt(); }
Tensor tensor(const Opt& t) { return t.has_value() ? *t : Tensor(); }

struct ResidualNorm : torch::autograd::Function<ResidualNorm> {
    static variable_list forward(AutogradContext* ctx, const Tensor& h, const Opt& b, const Opt& w, const Opt& c, const Opt& pw,
                                 const Opt& pb, const Opt& gate, int64_t norm, int64_t post, double alpha, double eps, bool want_sum) {
        Tensor stats;
        const auto [r, y] = norm_fwd(h, tensor(b), {tensor(w), tensor(c), tensor(pw), tensor(pb)}, tensor(gate), {norm, post, alpha, eps}, want_sum, &stats);
        ctx->save_for_backward({h, tensor(b), tensor(w), tensor(c), tensor(pw), tensor(pb), tensor(gate), stats});
        ctx->saved_data["kinds"] = norm * 4 + post;
        ctx->saved_data["alpha"] = alpha;
        ctx->saved_data["eps"] = eps;
        ctx->set_materialize_grads(false);
        if (r.defined() && y.defined()) return {r, y};
        return {r.defined() ? r : y};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        variable_list v = ctx->get_saved_variables();
        v[7] = aligned(v[7]);       // the statistics are read 16 bytes at a time; hooks on saved tensors may hand them back elsewhere
        const int64_t kinds = ctx->saved_data["kinds"].toInt();
        const NormCfg cfg{kinds / 4, kinds % 4, ctx->saved_data["alpha"].toDouble(), ctx->saved_data["eps"].toDouble()};
        Tensor dr, dy;
        if (grads.size() == 2) { dr = grads[0]; dy = grads[1]; }
        else (cfg.norm ? dy : dr) = grads[0];
        variable_list out(12);
        if (!dr.defined() && !dy.defined()) return out;
        check_tangents({&dr, &dy}, "residual_norm backward");
        check_capture("residual_norm");
        if (dr.defined()) dr = dr.contiguous();
        if (dy.defined()) dy = dy.contiguous();
        bpt_res_norm_args a;
        TORCH_CHECK(norm_args(v[0], v[1], {v[2], v[3], v[4], v[5]}, v[6], cfg, &a), "residual_norm backward: the saved tensors have changed their form");
        const c10::cuda::CUDAGuard guard(v[0].device());
        for (size_t i = 0, edge = 0; i < 7; ++i)        // the node has an edge for each tensor that was given
            if (v[i].defined() && ctx->needs_input_grad(edge++)) out[i] = at::empty_like(v[i]);
        const size_t n = api.res_norm_bytes(&a);
        const Tensor ws = bytes((int64_t)n, v[0]);
        const bpt_status s = api.res_norm_bwd(&a, (const float*)ptr(v[7]), ptr(dy), ptr(dr), ptr(out[0]), ptr(out[1]), ptr(out[2]), ptr(out[3]),
                                              ptr(out[4]), ptr(out[5]), ptr(out[6]), ws.data_ptr(), n, at::cuda::getCurrentCUDAStream().stream());
        TORCH_CHECK(s == BPT_OK, "bpt_res_norm_bwd failed (status ", (int)s, ")");
        return first_order_only(std::move(out), "residual_norm");
    }
};

py::object residual_norm(const Tensor& h_, const Opt& b_, const Opt& w_, const Opt& c_, const Opt& pw_, const Opt& pb_, const Opt& gate_, int64_t norm,
                         int64_t post, double alpha, double eps, bool want_sum) {
    check_tracing("residual_norm");
    for (const Opt* t : {&b_, &w_, &c_, &pw_, &pb_, &gate_})
        if (t->has_value()) check_tangents({&**t}, "residual_norm");
    check_tangents({&h_}, "residual_norm");
    const Tensor h = h_.contiguous();
    const Opt b = given(b_), w = given(w_), c = given(c_), pw = given(pw_), pb = given(pb_), gate = given(gate_);
    bool grad = false;
    if (at::GradMode::is_enabled()) {
        grad = h.requires_grad();
        for (const Opt* t : {&b, &w, &c, &pw, &pb, &gate}) grad = grad || (t->has_value() && (*t)->requires_grad());
    }
    try {
        if (grad) {
            const variable_list o = ResidualNorm::apply(h, b, w, c, pw, pb, gate, norm, post, alpha, eps, want_sum);
            if (o.size() == 2) return py::make_tuple(o[0], o[1]);
            return py::cast(o[0]);
        }
        const auto [r, y] = norm_fwd(h, tensor(b), {tensor(w), tensor(c), tensor(pw), tensor(pb)}, tensor(gate), {norm, post, alpha, eps}, want_sum, nullptr);
        if (r.defined() && y.defined()) return py::make_tuple(r, y);
        return py::cast(r.defined() ? r : y);
    } catch (const Refused&) {
        return py::none();
    }
}

// ---------------------------------------------------------------------------------------------------------
// y = (act(x Wg^T) * (x Wu^T)) Wd^T
// ---------------------------------------------------------------------------------------------------------
struct FfSizes { int64_t rows; int32_t D, F; };
bool ff_sizes(const Tensor& x, const Tensor& wg, const Tensor& wu, const Tensor& wd, FfSizes* s) {
    if (!x.is_cuda() || x.dim() < 1 || x.scalar_type() != at::kBFloat16 || !x.is_contiguous() || wg.dim() != 2 || wu.dim() != 2 || wd.dim() != 2) return false;
    const int64_t D = x.size(-1), F = wg.size(0);
    if (D < 1 || F < 1 || D > INT32_MAX || F > INT32_MAX) return false;
    for (const Tensor* w : {&wg, &wu, &wd})
        if (w->scalar_type() != at::kBFloat16 || w->device() != x.device() || !w->is_contiguous()) return false;
    if (wg.size(1) != D || wu.size(0) != F || wu.size(1) != D || wd.size(0) != D || wd.size(1) != F) return false;
    *s = {x.numel() / D, (int32_t)D, (int32_t)F};
    return true;
}
Tensor ff_fwd(const Tensor& x, const Tensor& wg, const Tensor& wu, const Tensor& wd, int64_t act, Tensor* status) {
    FfSizes s;
    if (!ff_sizes(x, wg, wu, wd, &s)) throw Refused{};
    const c10::cuda::CUDAGuard guard(x.device());
    const Tensor y = at::empty_like(x);
    const size_t n = api.gated_ff_bytes(s.rows, s.D, s.F, 0);
    const Tensor ws = bytes((int64_t)n, x);
    if (!api.few_rows(s.rows, s.D, s.F)) *status = bytes(256, x);      // the few-rows kernels wait for nothing
    if (api.gated_ff_fwd(ptr(x), ptr(wg), ptr(wu), ptr(wd), ptr(y), s.rows, s.D, s.F, (int32_t)act, ptr(*status), ptr(ws), n,
                         at::cuda::getCurrentCUDAStream().stream()) != BPT_OK)
        throw Refused{};
    return y;
}

struct GatedFeedForward : torch::autograd::Function<GatedFeedForward> {
    static Tensor forward(AutogradContext* ctx, const Tensor& x, const Tensor& wg, const Tensor& wu, const Tensor& wd, int64_t act, Tensor* status) {
        const Tensor y = ff_fwd(x, wg, wu, wd, act, status);
        ctx->save_for_backward({x, wg, wu, wd});
        ctx->saved_data["act"] = act;
        return y;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        variable_list v = ctx->get_saved_variables();
        check_tangents({&grads[0]}, "gated_feed_forward backward");
        check_capture("gated_feed_forward");
        for (auto& t : v) t = aligned(t);       // hooks on saved tensors may hand them back elsewhere
        const Tensor dy = aligned(grads[0]);
        variable_list out(6);
        FfSizes s;
        TORCH_CHECK(ff_sizes(v[0], v[1], v[2], v[3], &s), "gated_feed_forward backward: the saved tensors have changed their form");
        const c10::cuda::CUDAGuard guard(v[0].device());
        const bool dx = ctx->needs_input_grad(0), dw = ctx->needs_input_grad(1) || ctx->needs_input_grad(2) || ctx->needs_input_grad(3);
        if (!dx && !dw) return out;
        Tensor g[4];
        if (dx) g[0] = at::empty_like(v[0]);
        if (dw)
            for (int i = 1; i < 4; ++i) g[i] = at::empty_like(v[i]);
        const size_t n = api.gated_ff_bytes(s.rows, s.D, s.F, 1);
        const Tensor ws = bytes((int64_t)n, v[0]);
        // no status block: nobody could reach it; a wait that gives up shows in the device's record (bpt_check_device)
        const bpt_status e = api.gated_ff_bwd(ptr(v[0]), ptr(v[1]), ptr(v[2]), ptr(v[3]), ptr(dy), ptr(g[0]), ptr(g[1]), ptr(g[2]), ptr(g[3]), s.rows, s.D, s.F,
                                              (int32_t)ctx->saved_data["act"].toInt(), nullptr, ptr(ws), n, at::cuda::getCurrentCUDAStream().stream());
        TORCH_CHECK(e == BPT_OK, "bpt_gated_ff_bwd failed (status ", (int)e, ")");
        for (int i = 0; i < 4; ++i)
            if (ctx->needs_input_grad(i)) out[i] = g[i];
        return first_order_only(std::move(out), "gated_feed_forward");
    }
};

// (y, status block or None)
py::object gated_feed_forward(const Tensor& x_, const Tensor& wg_, const Tensor& wu_, const Tensor& wd_, int64_t act) {
    check_tracing("gated_feed_forward");
    check_tangents({&x_, &wg_, &wu_, &wd_}, "gated_feed_forward");
    const Tensor x = aligned(x_), wg = aligned(wg_), wu = aligned(wu_), wd = aligned(wd_);
    const bool grad = at::GradMode::is_enabled() && (x.requires_grad() || wg.requires_grad() || wu.requires_grad() || wd.requires_grad());
    try {
        Tensor status;
        const Tensor y = grad ? GatedFeedForward::apply(x, wg, wu, wd, act, &status) : ff_fwd(x, wg, wu, wd, act, &status);
        return py::make_tuple(y, status.defined() ? py::cast(status) : py::none());
    } catch (const Refused&) {
        return py::none();
    }
}

// ---------------------------------------------------------------------------------------------------------
// out[..., t] = scale * weight[ids[..., t]], zero rows behind the tokens
// ---------------------------------------------------------------------------------------------------------
struct EmbedCfg { int64_t vocab, D, out_rows, padding; at::ScalarType weight_type, out_type; double scale; };

bool embed_args(const Tensor& ids, const Tensor& lengths, const EmbedCfg& c, bpt_embed_args* a) {
    *a = bpt_embed_args{};
    if (!ids.is_cuda() || ids.dim() < 1 || !ids.is_contiguous() || (ids.scalar_type() != at::kInt && ids.scalar_type() != at::kLong)) return false;
    const auto code = [](at::ScalarType t, bpt_dtype* out) {
        *out = t == at::kFloat ? BPT_F32 : BPT_BF16;
        return t == at::kFloat || t == at::kBFloat16;
    };
    if (c.D < 1 || c.D > INT32_MAX || !code(c.weight_type, &a->weight_dtype) || !code(c.out_type, &a->out_dtype)) return false;
    if (lengths.defined() && (lengths.scalar_type() != at::kInt || lengths.device() != ids.device() || !lengths.is_contiguous() ||
                              lengths.sizes() != ids.sizes().slice(0, ids.dim() - 1)))
        return false;
    a->batch = 1;
    for (int64_t i = 0; i + 1 < ids.dim(); ++i) a->batch *= ids.size(i);
    a->tokens = ids.size(-1);
    a->out_rows = c.out_rows;
    a->vocab = c.vocab;
    a->padding_idx = c.padding;
    a->D = (int32_t)c.D;
    a->id_bytes = ids.scalar_type() == at::kInt ? 4 : 8;
    a->scale = (float)c.scale;
    a->ids = ids.data_ptr();
    a->lengths = (const int32_t*)ptr(lengths);
    return true;
}
Tensor embed_fwd(const Tensor& ids, const Tensor& weight, const Tensor& lengths, const EmbedCfg& c) {
    bpt_embed_args a;
    // the backward's padding_idx is checked here, too: nothing is left to refuse there
    if (!embed_args(ids, lengths, c, &a) || weight.device() != ids.device() || c.padding < -1 || c.padding >= c.vocab) throw Refused{};
    a.weight = weight.data_ptr();
    const c10::cuda::CUDAGuard guard(ids.device());
    std::vector<int64_t> shape(ids.sizes().begin(), ids.sizes().end());
    shape.back() = c.out_rows;
    shape.push_back(c.D);
    const Tensor out = at::empty(shape, weight.options().dtype(c.out_type));
    if (api.embed_fwd(&a, ptr(out), at::cuda::getCurrentCUDAStream().stream()) != BPT_OK) throw Refused{};
    return out;
}

struct TokenStates : torch::autograd::Function<TokenStates> {
    // the table itself is not needed again, only its form: it may change before the backward pass
    static Tensor forward(AutogradContext* ctx, const Tensor& ids, const Tensor& weight, const Opt& lengths, const EmbedCfg* c) {
        const Tensor out = embed_fwd(ids, weight, tensor(lengths), *c);
        ctx->save_for_backward({ids, tensor(lengths)});
        ctx->saved_data["sizes"] = std::vector<int64_t>{c->vocab, c->D, c->out_rows, c->padding, (int64_t)c->weight_type, (int64_t)c->out_type};
        ctx->saved_data["scale"] = c->scale;
        return out;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        const variable_list v = ctx->get_saved_variables();
        const std::vector<int64_t> s = ctx->saved_data["sizes"].toIntVector();
        const EmbedCfg c{s[0], s[1], s[2], s[3], (at::ScalarType)s[4], (at::ScalarType)s[5], ctx->saved_data["scale"].toDouble()};
        variable_list out(4);
        check_tangents({&grads[0]}, "token_states backward");
        check_capture("token_states");
        const Tensor dy = grads[0].contiguous();
        bpt_embed_args a;
        TORCH_CHECK(embed_args(v[0], v[1], c, &a) && dy.scalar_type() == c.out_type && dy.numel() == a.batch * a.out_rows * a.D,
                    "token_states backward: the saved tensors have changed their form");
        const c10::cuda::CUDAGuard guard(v[0].device());
        out[1] = at::empty({c.vocab, c.D}, dy.options().dtype(c.weight_type));
        const size_t n = api.embed_bytes(&a);
        const Tensor ws = bytes((int64_t)n, dy);
        const bpt_status e = api.embed_bwd(&a, ptr(dy), ptr(out[1]), ptr(ws), n, at::cuda::getCurrentCUDAStream().stream());
        TORCH_CHECK(e == BPT_OK, "bpt_embed_bwd failed (status ", (int)e, ")");
        return first_order_only(std::move(out), "token_states");
    }
};

py::object token_states(const Tensor& ids_, const Tensor& weight_, const Opt& lengths_, double scale, int64_t span_rows, int64_t padding, const py::object& dtype) {
    check_tracing("token_states");
    check_tangents({&weight_}, "token_states");
    if (ids_.dim() < 1 || weight_.dim() != 2 || span_rows < 0) return py::none();
    const Tensor ids = ids_.contiguous(), weight = weight_.contiguous();
    const Opt lengths = given(lengths_);
    const at::ScalarType type = dtype.is_none() ? weight.scalar_type() : torch::python::detail::py_object_to_dtype(dtype);
    const EmbedCfg c{weight.size(0), weight.size(1), ids.size(-1) + span_rows, padding, weight.scalar_type(), type, scale};
    try {
        if (at::GradMode::is_enabled() && weight.requires_grad()) return py::cast(TokenStates::apply(ids, weight, lengths, &c));
        return py::cast(embed_fwd(ids, weight, tensor(lengths), c));
    } catch (const Refused&) {
        return py::none();
    }
}

// ---------------------------------------------------------------------------------------------------------
// the norm over all gradients, and clipping
// ---------------------------------------------------------------------------------------------------------
// A tensor, or a sequence of tensors and None.
bool take_tensors(const py::object& from, std::vector<Tensor>* to) {
    if (THPVariable_Check(from.ptr())) {
        to->push_back(THPVariable_Unpack(from.ptr()));
        return true;
    }
    for (const py::handle& h : from) {
        if (h.is_none()) to->emplace_back();
        else if (THPVariable_Check(h.ptr())) to->push_back(THPVariable_Unpack(h.ptr()));
        else return false;
    }
    return true;
}

// The bytes from the first to the last element of a tensor that has some.
std::pair<uintptr_t, uintptr_t> span(const Tensor& t) {
    uintptr_t bytes = t.element_size();
    for (int64_t i = 0; i < t.dim(); ++i) bytes += (t.size(i) - 1) * t.stride(i) * t.element_size();
    return {(uintptr_t)t.data_ptr(), (uintptr_t)t.data_ptr() + bytes};
}

// Whether some element of a and one of b share a byte; with b the same tensor as a, whether two different elements do.  The distance of two elements is the
// distance of the tensors' starts plus whole multiples of the strides, each in its range; strides that both have count once.  From the
// largest stride on, only the multiples that the smaller strides can still make up for are tried: a few where strides
// nest as those of views do.  Where they do not, and it would take long, the answer is that they meet.
bool share_memory(const Tensor& a, const Tensor& b) {
    if (!a.numel() || !b.numel()) return false;
    const bool self = &a == &b;
    const auto from_a = span(a), from_b = span(b);
    if (!self && (from_a.second <= from_b.first || from_b.second <= from_a.first)) return false;
    struct Step { int64_t bytes, lo, hi; };         // lo .. hi multiples
    std::vector<Step> steps;
    for (const Tensor* t : {&a, &b}) {
        for (int64_t i = 0; i < t->dim(); ++i) {
            const int64_t n = t->size(i) - 1, bytes = t->stride(i) * (int64_t)t->element_size();
            if (n == 0) continue;
            if (bytes == 0) {
                if (self) return true;
                continue;
            }
            auto same = std::find_if(steps.begin(), steps.end(), [&](const Step& s) { return s.bytes == bytes; });
            if (self && same != steps.end()) return true;
            if (same == steps.end()) same = steps.insert(steps.end(), Step{bytes, 0, 0});
            if (t == &a) same->hi += n;
            if (t == &b) same->lo -= n;
        }
        if (self) break;
    }
    std::sort(steps.begin(), steps.end(), [](const Step& x, const Step& y) { return x.bytes > y.bytes; });
    std::vector<int64_t> low(steps.size() + 1, 0), high(steps.size() + 1, 0);      // what the steps from k on reach
    for (size_t k = steps.size(); k-- > 0;) {
        low[k] = low[k + 1] + steps[k].lo * steps[k].bytes;
        high[k] = high[k + 1] + steps[k].hi * steps[k].bytes;
    }
    // the start of a's element minus that of b's lies between these where they share a byte
    const int64_t least = 1 - (int64_t)a.element_size(), most = (int64_t)b.element_size() - 1;
    const auto down = [](int64_t x, int64_t y) { return x >= 0 ? x / y : -((-x + y - 1) / y); };
    int tries = 100000;
    const std::function<bool(size_t, int64_t, bool)> from = [&](size_t k, int64_t d, bool other) {
        if (k == steps.size()) return other && d >= least && d <= most;
        const int64_t s = steps[k].bytes;
        const int64_t first = std::max(steps[k].lo, -down(d + high[k + 1] - least, s)), last = std::min(steps[k].hi, down(most - d - low[k + 1], s));
        for (int64_t c = first; c <= last; ++c)
            if (--tries < 0 || from(k + 1, d + c * s, other || c != 0)) return true;
        return false;
    };
    return from(0, (int64_t)(from_a.first - from_b.first), !self);
}

// Whether anything that clip_gradients writes -- the results, or without any the gradients -- shares memory with another tensor of the call or with
// itself.  A result may be its own gradient.
bool overlaps(const std::vector<Tensor>& g, const std::vector<Tensor>& o) {
    struct View { const Tensor* t; uintptr_t from, to; bool write; };
    std::vector<View> views;
    const auto add = [&](const Tensor& t, bool write) {
        const auto at = span(t);
        views.push_back({&t, at.first, at.second, write});
    };
    for (size_t i = 0; i < g.size(); ++i) {
        if (!g[i].defined() || !g[i].numel()) continue;
        const Tensor& to = o.empty() ? g[i] : o[i];
        if (!to.is_non_overlapping_and_dense() && share_memory(to, to)) return true;
        add(to, true);
        if (!o.empty() && !(to.data_ptr() == g[i].data_ptr() && to.strides() == g[i].strides() && to.scalar_type() == g[i].scalar_type())) add(g[i], false);
    }
    std::sort(views.begin(), views.end(), [](const View& x, const View& y) { return x.from < y.from; });
    for (size_t i = 0; i < views.size(); ++i)
        for (size_t j = i + 1; j < views.size() && views[j].from < views[i].to; ++j)
            if ((views[i].write || views[j].write) && share_memory(*views[i].t, *views[j].t)) return true;
    return false;
}

// Elements lie one after another in memory, in whatever order, so that a tensor is a list of numbers.
py::object clip_gradients(const py::object& grads, const py::object& into, int64_t norm_type, bool clip, double max_norm, double eps) {
    check_tracing("clip_gradients");
    std::vector<Tensor> g, o;
    if (!take_tensors(grads, &g) || (!into.is_none() && (!take_tensors(into, &o) || o.size() != g.size()))) return py::none();
    const at::NoGradGuard no_grad;
    std::vector<bpt_grad> list;
    std::vector<std::pair<Tensor, Tensor>> back;    // what was computed in a copy, and where it belongs
    std::vector<Tensor> held;
    std::vector<const Tensor*> written;
    list.reserve(g.size());
    const Tensor* first = nullptr;
    for (size_t i = 0; i < g.size(); ++i) {
        if (!g[i].defined()) continue;
        check_tangents({&g[i]}, "clip_gradients");
        bpt_grad e{};
        if (g[i].layout() != at::kStrided || !g[i].is_cuda() || (first && g[i].device() != first->device()) || !type_code(g[i], &e.dtype)) return py::none();
        if (!first) first = &g[i];
        Tensor src = g[i], dst;
        // parameters in the place of their gradients, as other interfaces take them, would be scaled themselves
        if (clip && (o.empty() ? g[i] : o[i]).defined() && (o.empty() ? g[i] : o[i]).is_leaf() && (o.empty() ? g[i] : o[i]).requires_grad()) return py::none();
        if (!o.empty()) {
            if (!o[i].defined()) return py::none();
            check_tangents({&o[i]}, "clip_gradients");
            dst = o[i];
            if (dst.layout() != at::kStrided || dst.device() != src.device() || dst.sizes() != src.sizes() || !type_code(dst, &e.out_dtype)) return py::none();
            if (!(src.strides() == dst.strides() && src.is_non_overlapping_and_dense())) {
                src = src.contiguous();
                if (!dst.is_contiguous()) {
                    held.push_back(at::empty(dst.sizes(), dst.options()));
                    back.emplace_back(held.back(), dst);
                    dst = held.back();
                }
                held.push_back(src);
            }
            written.push_back(&o[i]);
        } else if (!src.is_non_overlapping_and_dense()) {
            src = src.contiguous();
            held.push_back(src);
            if (clip) back.emplace_back(src, g[i]);
        }
        if (clip && o.empty()) written.push_back(&g[i]);
        e.grad = src.data_ptr();
        e.out = ptr(dst);
        e.numel = src.numel();
        list.push_back(e);
    }
    if (clip && !held.empty() && overlaps(g, o)) return py::none();     // the library sees copies
    const c10::cuda::OptionalCUDAGuard guard(first ? std::optional<at::Device>(first->device()) : std::nullopt);
    const auto options = at::TensorOptions().device(first ? first->device() : at::Device(at::kCUDA, c10::cuda::current_device()));
    const Tensor norm = at::empty({}, options.dtype(at::kFloat));
    const size_t n = api.grad_norm_bytes(list.data(), (int32_t)list.size());
    const Tensor ws = at::empty({(int64_t)n}, options.dtype(at::kByte));
    cudaStream_t st = at::cuda::getCurrentCUDAStream().stream();
    const bpt_status s = clip ? api.clip_grads(list.data(), (int32_t)list.size(), (int32_t)norm_type, (float)max_norm, (float)eps, (float*)ptr(norm), ptr(ws), n, st)
                              : api.grad_norm(list.data(), (int32_t)list.size(), (int32_t)norm_type, (float*)ptr(norm), ptr(ws), n, st);
    if (s != BPT_OK) return py::none();
    for (const auto& [from, to] : back) to.copy_(from);
    for (const Tensor* t : written)     // what a graph has saved of them is no longer what it was
        if (!t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
    return py::cast(norm);
}

// ---------------------------------------------------------------------------------------------------------
// penalties, biases and a mask on logits
// ---------------------------------------------------------------------------------------------------------
// Elements of a row next to one another; rows as they lie, or copied where they overlap.
Tensor by_rows(const Tensor& t) {
    const bool ok = t.dim() == 2 ? (t.size(1) < 2 || t.stride(1) == 1) && (t.size(0) < 2 || t.stride(0) >= t.size(1)) : t.is_contiguous();
    return ok ? t : t.contiguous();
}
int64_t row_stride(const Tensor& t) { return t.size(0) < 2 ? t.size(1) : t.stride(0); }

// A number, or one float32 per row.
bool setting(const py::object& v, const Tensor& logits, std::vector<Tensor>* held, float* number, const float** rows) {
    if (!THPVariable_Check(v.ptr())) {
        *number = (float)v.cast<double>();
        return true;
    }
    const Tensor& t = THPVariable_Unpack(v.ptr());
    check_tangents({&t}, "adjust_logits");
    TORCH_CHECK_NOT_IMPLEMENTED(!(at::GradMode::is_enabled() && t.requires_grad()), "adjust_logits has no derivative");
    if (t.device() != logits.device() || t.dim() != 1 || t.size(0) != logits.size(0) || t.scalar_type() != at::kFloat) return false;
    held->push_back(t.contiguous());
    *rows = (const float*)held->back().data_ptr();
    return true;
}

py::object adjust_logits(const Tensor& logits_, const Opt& history_, const Opt& lengths_, const Opt& prompts_, const py::object& repetition, const py::object& presence,
                         const py::object& frequency, const Opt& bias_, const Opt& bias_ids_, const Opt& bias_values_, const Opt& allowed_, const Opt& out_) {
    check_tracing("adjust_logits");
    for (const Opt* t : {&bias_, &bias_values_, &out_})
        if (t->has_value()) {
            check_tangents({&**t}, "adjust_logits");
            TORCH_CHECK_NOT_IMPLEMENTED(!(at::GradMode::is_enabled() && (*t)->requires_grad()), "adjust_logits has no derivative");
        }
    check_tangents({&logits_}, "adjust_logits");
    TORCH_CHECK_NOT_IMPLEMENTED(!(at::GradMode::is_enabled() && logits_.requires_grad()), "adjust_logits has no derivative");
    bpt_logits_args a{};
    if (!logits_.is_cuda() || logits_.dim() != 2 || logits_.size(1) < 1 || !type_code(logits_, &a.dtype)) return py::none();
    const int64_t B = logits_.size(0), V = logits_.size(1);
    const at::Device device = logits_.device();
    std::vector<Tensor> held;       // what was copied stays until the launch
    held.reserve(12);
    const Tensor logits = by_rows(logits_);
    const auto id_type = [](const Tensor& t) { return t.scalar_type() == at::kInt || t.scalar_type() == at::kLong; };
    a.rows = B; a.vocab = V;
    a.logits = logits.data_ptr(); a.logits_stride = row_stride(logits);
    a.repetition = 1.f;
    a.history_bytes = a.bias_id_bytes = 8;
    if (history_.has_value()) {
        if (history_->dim() != 2 || history_->size(0) != B || history_->device() != device || !id_type(*history_)) return py::none();
        held.push_back(by_rows(*history_));
        const Tensor& h = held.back();
        a.history = h.data_ptr(); a.history_len = h.size(1); a.history_stride = row_stride(h); a.history_bytes = (int32_t)h.element_size();
        const int32_t** slot[2] = {&a.lengths, &a.prompt_lengths};
        const Opt* given_[2] = {&lengths_, &prompts_};
        for (int i = 0; i < 2; ++i) {
            if (!given_[i]->has_value()) continue;
            const Tensor& t = **given_[i];
            if (t.dim() != 1 || t.size(0) != B || t.device() != device || t.scalar_type() != at::kInt) return py::none();
            held.push_back(t.contiguous());
            *slot[i] = (const int32_t*)held.back().data_ptr();
        }
    } else if (lengths_.has_value() || prompts_.has_value()) {
        return py::none();
    }
    if (!setting(repetition, logits, &held, &a.repetition, &a.repetition_rows) || !setting(presence, logits, &held, &a.presence, &a.presence_rows) ||
        !setting(frequency, logits, &held, &a.frequency, &a.frequency_rows))
        return py::none();
    if (bias_.has_value()) {
        const Tensor& t = *bias_;
        if (t.dim() < 1 || t.dim() > 2 || t.size(-1) != V || (t.dim() == 2 && t.size(0) != 1 && t.size(0) != B) || t.device() != device ||
            !type_code(t, &a.bias_dtype))
            return py::none();
        held.push_back(by_rows(t));
        a.bias = held.back().data_ptr();
        a.bias_stride = t.dim() == 2 && t.size(0) > 1 ? row_stride(held.back()) : 0;
    }
    if (bias_ids_.has_value() != bias_values_.has_value()) return py::none();
    if (bias_ids_.has_value()) {
        if (bias_ids_->dim() != 2 || bias_ids_->size(0) != B || bias_ids_->device() != device || !id_type(*bias_ids_) ||
            bias_values_->sizes() != bias_ids_->sizes() || bias_values_->device() != device || bias_values_->scalar_type() != at::kFloat)
            return py::none();
        held.push_back(bias_ids_->contiguous());
        a.bias_ids = held.back().data_ptr(); a.bias_count = bias_ids_->size(1); a.bias_id_bytes = (int32_t)bias_ids_->element_size();
        held.push_back(bias_values_->contiguous());
        a.bias_values = (const float*)held.back().data_ptr();
    }
    if (allowed_.has_value()) {
        const Tensor& t = *allowed_;
        if (t.dim() < 1 || t.dim() > 2 || t.size(-1) != (V + 31) / 32 || (t.dim() == 2 && t.size(0) != 1 && t.size(0) != B) || t.device() != device ||
            t.scalar_type() != at::kInt)
            return py::none();
        held.push_back(by_rows(t));
        a.allowed = (const int32_t*)held.back().data_ptr();
        a.allowed_stride = t.dim() == 2 && t.size(0) > 1 ? row_stride(held.back()) : 0;
    }
    const c10::cuda::CUDAGuard guard(device);
    Tensor out;
    if (out_.has_value()) {
        out = *out_;
        if (out.sizes() != logits.sizes() || out.device() != device || !by_rows(out).is_same(out)) return py::none();
        // the logits themselves, or somewhere else
        if (!(out.data_ptr() == logits.data_ptr() && out.scalar_type() == logits.scalar_type() && row_stride(out) == row_stride(logits)) &&
            share_memory(out, logits))
            return py::none();
        for (const Tensor& t : held)
            if (share_memory(out, t)) return py::none();
    } else {
        out = at::empty({B, V}, logits.options());
    }
    if (!type_code(out, &a.out_dtype)) return py::none();
    a.out_stride = row_stride(out);
    const size_t n = api.adjust_logits_bytes(&a);
    const Tensor ws = n ? bytes((int64_t)n, logits) : Tensor();
    if (api.adjust_logits(&a, ptr(out), ptr(ws), n, at::cuda::getCurrentCUDAStream().stream()) != BPT_OK) return py::none();
    if (out_.has_value() && !out.is_inference()) out.unsafeGetTensorImpl()->bump_version();
    return py::cast(out);
}

void bind_library(const std::vector<uintptr_t>& f) {
    TORCH_CHECK(f.size() == 15, "fifteen functions are expected");
    api.res_norm_fwd = reinterpret_cast<decltype(api.res_norm_fwd)>(f[0]);
    api.res_norm_bytes = reinterpret_cast<decltype(api.res_norm_bytes)>(f[1]);
    api.res_norm_bwd = reinterpret_cast<decltype(api.res_norm_bwd)>(f[2]);
    api.few_rows = reinterpret_cast<decltype(api.few_rows)>(f[3]);
    api.gated_ff_bytes = reinterpret_cast<decltype(api.gated_ff_bytes)>(f[4]);
    api.gated_ff_fwd = reinterpret_cast<decltype(api.gated_ff_fwd)>(f[5]);
    api.gated_ff_bwd = reinterpret_cast<decltype(api.gated_ff_bwd)>(f[6]);
    api.embed_fwd = reinterpret_cast<decltype(api.embed_fwd)>(f[7]);
    api.embed_bytes = reinterpret_cast<decltype(api.embed_bytes)>(f[8]);
    api.embed_bwd = reinterpret_cast<decltype(api.embed_bwd)>(f[9]);
    api.grad_norm_bytes = reinterpret_cast<decltype(api.grad_norm_bytes)>(f[10]);
    api.grad_norm = reinterpret_cast<decltype(api.grad_norm)>(f[11]);
    api.clip_grads = reinterpret_cast<decltype(api.clip_grads)>(f[12]);
    api.adjust_logits = reinterpret_cast<decltype(api.adjust_logits)>(f[13]);
    api.adjust_logits_bytes = reinterpret_cast<decltype(api.adjust_logits_bytes)>(f[14]);
}

}  // namespace

PYBIND11_MODULE(_bpt_torch, m) {
    m.def("bind_library", &bind_library);
    m.def("residual_norm", &residual_norm);
    m.def("gated_feed_forward", &gated_feed_forward);
    m.def("token_states", &token_states);
    m.def("clip_gradients", &clip_gradients);
    m.def("share_memory", [](const Tensor& a, const std::optional<Tensor>& b) { return share_memory(a, b.has_value() ? *b : a); }, py::arg("a"),
          py::arg("b") = py::none());
    m.def("adjust_logits", &adjust_logits);
}
