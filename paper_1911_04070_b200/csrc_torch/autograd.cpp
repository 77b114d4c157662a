// The position-wise operators as PyTorch functions with gradients, in C++ over the C ABI of include/bpt.h: argument checks,
// memory from PyTorch, the current stream, and the autograd nodes.  What layer.residual_norm and layer.gated_feed_forward call.
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

void bind_library(const std::vector<uintptr_t>& f) {
    TORCH_CHECK(f.size() == 7, "seven functions are expected");
    api.res_norm_fwd = reinterpret_cast<decltype(api.res_norm_fwd)>(f[0]);
    api.res_norm_bytes = reinterpret_cast<decltype(api.res_norm_bytes)>(f[1]);
    api.res_norm_bwd = reinterpret_cast<decltype(api.res_norm_bwd)>(f[2]);
    api.few_rows = reinterpret_cast<decltype(api.few_rows)>(f[3]);
    api.gated_ff_bytes = reinterpret_cast<decltype(api.gated_ff_bytes)>(f[4]);
    api.gated_ff_fwd = reinterpret_cast<decltype(api.gated_ff_fwd)>(f[5]);
    api.gated_ff_bwd = reinterpret_cast<decltype(api.gated_ff_bwd)>(f[6]);
}

}  // namespace

PYBIND11_MODULE(_bpt_torch, m) {
    m.def("bind_library", &bind_library);
    m.def("residual_norm", &residual_norm);
    m.def("gated_feed_forward", &gated_feed_forward);
}
