// The operators around the attention of a layer as native autograd functions over the C ABI (include/sna.h): checks of arguments,
// allocations and what is kept for the backward pass.  Nothing is computed here.
#include <c10/core/AutogradState.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/extension.h>

#include "../../include/sna.h"
#include "sna_torch.hpp"

namespace {

using sna_torch::check;
using torch::autograd::AutogradContext;
using torch::autograd::Variable;
using torch::autograd::variable_list;

void* stream_of(const at::Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.device().index()).stream(); }

sna_dtype_t dtype_of(const at::Tensor& t, const char* name) {
    switch (t.scalar_type()) {
        case at::kFloat: return SNA_FLOAT32;
        case at::kBFloat16: return SNA_BFLOAT16;
        case at::kHalf: return SNA_FLOAT16;
        default: TORCH_CHECK_VALUE(false, name, " must be float32, bfloat16 or float16, got ", t.scalar_type());
    }
}

// Forward-mode differentiation: the kernels compute no tangents, and a result without one would pass for a derivative of zero.
void check_no_tangent(const at::Tensor& t, const char* name) {
    TORCH_CHECK(!c10::AutogradState::get_tls_state().get_fw_grad_mode() || !t._fw_grad(0).defined(), name, " carries a tangent: forward-mode differentiation is not supported");
}
void check_cuda(const at::Tensor& t, const char* name, const at::Tensor& first, const char* first_name) {
    TORCH_CHECK_VALUE(t.is_cuda() && t.device() == first.device(), name, " must be a CUDA tensor on the device of ", first_name, " (", first.device(), "), got ", t.device());
    TORCH_CHECK_VALUE(t.layout() == at::kStrided && !t.is_neg(), name, " must be a dense tensor without a pending negation");
    check_no_tangent(t, name);
}
void check_like(const at::Tensor& t, const char* name, const at::Tensor& first, const char* first_name) {
    TORCH_CHECK_VALUE(t.defined(), name, " is missing");
    check_cuda(t, name, first, first_name);
    TORCH_CHECK_VALUE(t.scalar_type() == first.scalar_type(), name, " must be of the type of ", first_name, " (", first.scalar_type(), "), got ", t.scalar_type());
}
void check_once_differentiable(const char* name) {
    // the gradient is computed by kernels that autograd knows nothing of: a graph through it would be silently cut
    TORCH_CHECK(!at::GradMode::is_enabled(), name, " is differentiable once: create_graph is not supported");
}
bool wants_grad(std::initializer_list<const at::Tensor*> tensors) {
    if (!at::GradMode::is_enabled()) return false;
    for (const at::Tensor* t : tensors)
        if (t->defined() && t->requires_grad()) return true;
    return false;
}

at::Tensor or_undefined(const std::optional<at::Tensor>& t) { return t.has_value() ? *t : at::Tensor(); }

// Whether a kernel can read the 5-D tensor in place: contiguous channels, address and strides in multiples of `grain` elements.
bool in_place(const at::Tensor& t, int64_t grain) {
    if (t.size(4) > 1 && t.stride(4) != 1) return false;
    if (reinterpret_cast<uintptr_t>(t.data_ptr()) % (grain * t.element_size()) != 0) return false;
    for (int i = 0; i < 4; ++i)
        if (t.size(i) > 1 && t.stride(i) % grain != 0) return false;
    return true;
}
at::Tensor readable(const at::Tensor& t, int64_t grain) {
    if (in_place(t, grain)) return t;
    const at::Tensor c = t.contiguous();
    return in_place(c, grain) ? c : c.clone();      // (a contiguous view that starts at an odd address)
}
// Memory for a result of the shape of `t`, in the order of its strides where a kernel can write that.
at::Tensor result_like(const at::Tensor& t, int64_t grain) {
    at::Tensor r = at::empty_like(t);
    return in_place(r, grain) ? r : at::empty_like(t, at::MemoryFormat::Contiguous);
}
// What autograd hands over, as the kernels read it.  One row for all points (the gradient of a mean over them) is spread out first: read in place, the blocks of
// a kernel queue for the same few lines (attention's gradient, B = 2, 4 heads of 64, 4096 points, bf16: 199 us instead of 149).
at::Tensor gradient(const at::Tensor& g, const at::Tensor& like) {
    check_no_tangent(g, "the gradient");
    const at::Tensor t = g.to(like.scalar_type()).resolve_neg();
    return (t.size(2) > 1 && t.stride(2) == 0) || (t.size(3) > 1 && t.stride(3) == 0) ? t.contiguous() : t;
}
sna_tensor_t described(const at::Tensor& t) {
    auto stride = [&](int i) { return t.size(i) > 1 ? t.stride(i) : 0; };
    return {t.data_ptr(), stride(0), stride(1), stride(2), stride(3)};
}

// ---- norm and rotation ----------------------------------------------------------------------------------------------------

struct RotatePart {
    at::Tensor x, weight, lat, lon;
};

void check_part(const RotatePart& p, const char* name, const at::Tensor& q) {
    const std::string n(name);
    check_like(p.x, name, q, "q");
    TORCH_CHECK_VALUE(p.x.dim() == 5 && p.x.size(0) == q.size(0) && p.x.size(4) == q.size(4), name, " must be [B, H, nlat, nlon, C] with B = ", q.size(0), " and C = ",
                      q.size(4), ", got ", p.x.sizes());
    for (int i = 0; i < 5; ++i) TORCH_CHECK_VALUE(p.x.size(i) < (1 << 30), name, " is too large: ", p.x.sizes());
    if (p.weight.defined()) {
        check_cuda(p.weight, (n + "_weight").c_str(), q, "q");
        TORCH_CHECK_VALUE(p.weight.scalar_type() == at::kFloat && p.weight.dim() == 1 && p.weight.size(0) == q.size(4), name, "_weight must be float32 of shape [", q.size(4), "]");
    }
    TORCH_CHECK_VALUE(p.lat.defined() == p.lon.defined(), name, "_rotation must be a pair of tables");
    if (!p.lat.defined()) return;
    const at::Tensor* tables[2] = {&p.lat, &p.lon};
    for (int i = 0; i < 2; ++i) {
        const at::Tensor& t = *tables[i];
        check_cuda(t, (n + "_rotation").c_str(), q, "q");
        TORCH_CHECK_VALUE(t.scalar_type() == at::kFloat && t.dim() == 3 && t.size(0) == p.x.size(2 + i) && t.size(2) == 2, name, "_rotation: the table of ",
                          i == 0 ? "latitudes" : "longitudes", " must be float32 of shape [", p.x.size(2 + i), ", pairs, 2], got ", t.sizes());
        TORCH_CHECK_VALUE(t.is_contiguous() && reinterpret_cast<uintptr_t>(t.data_ptr()) % 8 == 0, name, "_rotation must be contiguous and aligned to 8 bytes");
        TORCH_CHECK_VALUE(!t.requires_grad(), name, "_rotation: no gradient of the angles is computed");
        TORCH_CHECK_VALUE(2 * t.size(1) <= q.size(4), name, "_rotation has more pairs than ", q.size(4), " channels");
    }
    TORCH_CHECK_VALUE(2 * (p.lat.size(1) + p.lon.size(1)) <= q.size(4), name, "_rotation has more pairs than ", q.size(4), " channels");
}

sna_rotate_t described(const RotatePart& p) {
    sna_rotate_t r{};
    r.nlat = (int)p.x.size(2); r.nlon = (int)p.x.size(3); r.H = (int)p.x.size(1);
    r.x = described(p.x);
    r.weight = p.weight.defined() ? p.weight.const_data_ptr<float>() : nullptr;
    if (p.lat.defined()) {
        r.lat_table = p.lat.const_data_ptr<float>(); r.lon_table = p.lon.const_data_ptr<float>();
        r.pairs_lat = (int)p.lat.size(1); r.pairs_lon = (int)p.lon.size(1);
    }
    return r;
}

variable_list rotate_forward(RotatePart (&parts)[2], double eps, bool interleaved) {
    const at::Tensor& q = parts[0].x;
    const c10::cuda::CUDAGuard guard(q.device());
    const sna_dtype_t dtype = dtype_of(q, "q");
    variable_list out(2);
    sna_rotate_t described_parts[2];
    for (int i = 0; i < 2; ++i) {
        RotatePart& p = parts[i];
        p.x = readable(p.x, 4);
        if (p.weight.defined()) p.weight = p.weight.contiguous();
        out[i] = result_like(p.x, 4);
        described_parts[i] = described(p);
        described_parts[i].y = described(out[i]);
    }
    check(sna_norm_rotate_forward(described_parts, 2, dtype, (int)q.size(0), (int)q.size(4), (float)eps, interleaved, stream_of(q)));
    return out;
}

class QkNormRotate : public torch::autograd::Function<QkNormRotate> {
public:
    using Optional = std::optional<at::Tensor>;
    static variable_list forward(AutogradContext* ctx, at::Tensor q, at::Tensor k, Optional q_weight, Optional k_weight, Optional q_lat, Optional q_lon, Optional k_lat,
                                 Optional k_lon, double eps, bool interleaved) {
        RotatePart parts[2] = {{q, or_undefined(q_weight), or_undefined(q_lat), or_undefined(q_lon)}, {k, or_undefined(k_weight), or_undefined(k_lat), or_undefined(k_lon)}};
        ctx->saved_data["q_weight"] = parts[0].weight.defined() && parts[0].weight.requires_grad();
        ctx->saved_data["k_weight"] = parts[1].weight.defined() && parts[1].weight.requires_grad();
        variable_list out = rotate_forward(parts, eps, interleaved);
        ctx->save_for_backward({parts[0].x, parts[1].x, parts[0].weight, parts[1].weight, parts[0].lat, parts[0].lon, parts[1].lat, parts[1].lon});
        ctx->saved_data["eps"] = eps;
        ctx->saved_data["interleaved"] = interleaved;
        return out;
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        check_once_differentiable("qk_norm_rotate");
        const auto saved = ctx->get_saved_variables();
        RotatePart parts[2] = {{saved[0], saved[2], saved[4], saved[5]}, {saved[1], saved[3], saved[6], saved[7]}};
        const at::Tensor& q = grads[0];
        const c10::cuda::CUDAGuard guard(q.device());
        variable_list result(10);
        sna_rotate_t described_parts[2];
        at::Tensor dy[2];
        for (int i = 0; i < 2; ++i) {
            RotatePart& p = parts[i];
            // (what hooks on saved tensors return is checked like arguments)
            check_like(p.x, i == 0 ? "q" : "k", q, "the gradient");
            TORCH_CHECK_VALUE(p.x.sizes() == grads[i].sizes(), i == 0 ? "q" : "k", " has shape ", p.x.sizes(), ", expected ", grads[i].sizes());
            check_part(p, i == 0 ? "q" : "k", q);
            p.x = readable(p.x, 4);
            if (p.weight.defined()) p.weight = p.weight.contiguous();
            dy[i] = readable(gradient(grads[i], p.x), 4);
            result[i] = result_like(p.x, 4);
            described_parts[i] = described(p);
            described_parts[i].dy = described(dy[i]);
            described_parts[i].dx = described(result[i]);
            if (p.weight.defined() && ctx->saved_data[i == 0 ? "q_weight" : "k_weight"].toBool()) {
                result[2 + i] = at::empty_like(p.weight);
                described_parts[i].dweight = result[2 + i].data_ptr<float>();
            }
        }
        const int B = (int)q.size(0), C = (int)q.size(4);
        const size_t bytes = result[2].defined() || result[3].defined() ? sna_norm_rotate_workspace_bytes(C) : 0;
        at::Tensor workspace = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
        check(sna_norm_rotate_backward(described_parts, 2, dtype_of(q, "the gradient"), B, C, (float)ctx->saved_data["eps"].toDouble(), ctx->saved_data["interleaved"].toBool(),
                                       bytes ? workspace.data_ptr() : nullptr, bytes, stream_of(q)));
        return result;
    }
};

std::tuple<at::Tensor, at::Tensor> qk_norm_rotate(const at::Tensor& q, const at::Tensor& k, const std::optional<at::Tensor>& q_weight_, const std::optional<at::Tensor>& k_weight_,
                                                  const std::optional<at::Tensor>& q_lat_, const std::optional<at::Tensor>& q_lon_, const std::optional<at::Tensor>& k_lat_,
                                                  const std::optional<at::Tensor>& k_lon_, double eps, bool interleaved) {
    const at::Tensor q_weight = or_undefined(q_weight_), k_weight = or_undefined(k_weight_);
    RotatePart parts[2] = {{q, q_weight, or_undefined(q_lat_), or_undefined(q_lon_)}, {k, k_weight, or_undefined(k_lat_), or_undefined(k_lon_)}};
    TORCH_CHECK_VALUE(q.dim() == 5, "q must be [B, H, nlat, nlon, C], got ", q.sizes());
    TORCH_CHECK_VALUE(q.is_cuda(), "q must be a CUDA tensor");
    check_cuda(q, "q", q, "q");
    dtype_of(q, "q");
    check_part(parts[0], "q", q);
    check_part(parts[1], "k", q);
    variable_list out = wants_grad({&q, &k, &q_weight, &k_weight})
                            ? QkNormRotate::apply(q, k, q_weight_, k_weight_, q_lat_, q_lon_, k_lat_, k_lon_, eps, interleaved)
                            : rotate_forward(parts, eps, interleaved);
    return {out[0], out[1]};
}

// ---- attention ------------------------------------------------------------------------------------------------------------

// Points in one line, 16-byte pieces: the tensor itself if it is so, else a contiguous copy.
bool in_line(const at::Tensor& t) { return in_place(t, 8) && (t.size(2) <= 1 || t.size(3) <= 1 || t.stride(2) == t.size(3) * t.stride(3)); }
at::Tensor attendable(const at::Tensor& t) {
    if (in_line(t)) return t;
    const at::Tensor c = t.contiguous();
    return in_line(c) ? c : c.clone();
}
at::Tensor attention_result_like(const at::Tensor& t) {
    at::Tensor r = at::empty_like(t);
    return in_line(r) ? r : at::empty_like(t, at::MemoryFormat::Contiguous);
}

struct AttentionInputs {
    at::Tensor q, k, v, log_weights;
    double scale;
};

void check_attention(const AttentionInputs& in) {
    const at::Tensor& q = in.q;
    TORCH_CHECK_VALUE(q.dim() == 5, "q must be [B, H, nlat, nlon, C], got ", q.sizes());
    TORCH_CHECK_VALUE(q.is_cuda(), "q must be a CUDA tensor");
    check_cuda(q, "q", q, "q");
    TORCH_CHECK_VALUE(q.scalar_type() == at::kBFloat16 || q.scalar_type() == at::kHalf, "q must be bfloat16 or float16, got ", q.scalar_type());
    check_like(in.k, "k", q, "q");
    check_like(in.v, "v", q, "q");
    TORCH_CHECK_VALUE(in.k.dim() == 5 && in.k.size(0) == q.size(0) && in.k.size(4) == q.size(4), "k must be [B, H, nlat, nlon, C] with B = ", q.size(0), " and C = ", q.size(4),
                      ", got ", in.k.sizes());
    TORCH_CHECK_VALUE(in.v.sizes() == in.k.sizes(), "v has shape ", in.v.sizes(), ", expected ", in.k.sizes());
    for (const at::Tensor* t : {&in.q, &in.k})
        for (int i = 0; i < 5; ++i) TORCH_CHECK_VALUE(t->size(i) < (1 << 30), "a tensor is too large: ", t->sizes());
    TORCH_CHECK_VALUE(in.k.size(1) > 0 ? q.size(1) % in.k.size(1) == 0 : q.size(1) == 0, "q's heads (", q.size(1), ") must be a multiple of k's (", in.k.size(1), ")");
    if (!in.log_weights.defined()) return;
    const at::Tensor& w = in.log_weights;
    check_cuda(w, "log_weights", q, "q");
    const int64_t points = in.k.size(2) * in.k.size(3);
    TORCH_CHECK_VALUE(w.scalar_type() == at::kFloat, "log_weights must be float32, got ", w.scalar_type());
    TORCH_CHECK_VALUE((w.dim() == 1 || (w.dim() == 2 && (w.size(0) == q.size(0) || w.size(0) == 1))) && w.size(-1) == points, "log_weights must be [", points, "] or [", q.size(0), ", ",
                      points, "], got ", w.sizes());
    TORCH_CHECK_VALUE(!w.requires_grad(), "log_weights: no gradient of the weights is computed");
}

// (the inputs become what the kernels read)
void make_readable(AttentionInputs& in) {
    for (at::Tensor* t : {&in.q, &in.k, &in.v}) *t = attendable(*t);
    if (in.log_weights.defined() && in.log_weights.size(-1) > 1 && in.log_weights.stride(-1) != 1) in.log_weights = in.log_weights.contiguous();
}

sna_attention_t described(const AttentionInputs& in) {
    sna_attention_t a{};
    a.B = (int)in.q.size(0); a.Hq = (int)in.q.size(1); a.Hk = (int)in.k.size(1); a.C = (int)in.q.size(4);
    a.nlat_q = (int)in.q.size(2); a.nlon_q = (int)in.q.size(3); a.nlat_k = (int)in.k.size(2); a.nlon_k = (int)in.k.size(3);
    a.q = described(in.q); a.k = described(in.k); a.v = described(in.v);
    if (in.log_weights.defined()) {
        a.log_weights = in.log_weights.const_data_ptr<float>();
        a.log_weights_batch = in.log_weights.dim() == 2 && in.log_weights.size(0) > 1 ? in.log_weights.stride(0) : 0;
    }
    a.scale = (float)in.scale;
    return a;
}

std::tuple<at::Tensor, at::Tensor, at::Tensor> attention_forward(AttentionInputs& in, bool for_backward) {
    const c10::cuda::CUDAGuard guard(in.q.device());
    make_readable(in);
    at::Tensor out = attention_result_like(in.q), lse = at::empty(in.q.sizes().slice(0, 4), in.q.options().dtype(at::kFloat));
    const sna_dtype_t dtype = dtype_of(in.q, "q");
    sna_attention_t a = described(in);
    a.out = described(out);
    at::Tensor rest;
    if (for_backward) {
        rest = attention_result_like(in.q);
        a.out_rest = described(rest);
    }
    a.lse = lse.data_ptr<float>();
    const size_t bytes = sna_attention_forward_workspace_bytes(&a, dtype);
    at::Tensor workspace;
    if (bytes > 0) workspace = at::empty({(int64_t)bytes}, in.q.options().dtype(at::kByte));
    check(sna_attention_forward(&a, dtype, bytes ? workspace.data_ptr() : nullptr, bytes, stream_of(in.q)));
    return {out, lse, rest};
}

class WeightedAttention : public torch::autograd::Function<WeightedAttention> {
public:
    static variable_list forward(AutogradContext* ctx, at::Tensor q, at::Tensor k, at::Tensor v, std::optional<at::Tensor> log_weights, double scale) {
        AttentionInputs in{q, k, v, or_undefined(log_weights), scale};
        auto [out, lse, rest] = attention_forward(in, true);
        ctx->save_for_backward({in.q, in.k, in.v, in.log_weights, out, lse, rest});
        ctx->saved_data["scale"] = scale;
        ctx->mark_non_differentiable({lse});
        return {out, lse};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        check_once_differentiable("weighted_attention");
        const auto saved = ctx->get_saved_variables();
        AttentionInputs in{saved[0], saved[1], saved[2], saved[3], ctx->saved_data["scale"].toDouble()};
        // (what hooks on saved tensors return is checked like arguments)
        check_attention(in);
        const at::Tensor& lse = saved[5];
        for (int i : {4, 6}) {
            check_like(saved[i], "out", in.q, "q");
            TORCH_CHECK_VALUE(saved[i].sizes() == in.q.sizes(), "out has shape ", saved[i].sizes(), ", expected ", in.q.sizes());
        }
        TORCH_CHECK_VALUE(grads[0].sizes() == in.q.sizes() && grads[0].device() == in.q.device(), "the gradient has shape ", grads[0].sizes(), ", expected ", in.q.sizes());
        check_cuda(lse, "lse", in.q, "q");
        TORCH_CHECK_VALUE(lse.scalar_type() == at::kFloat && lse.sizes() == in.q.sizes().slice(0, 4) && lse.is_contiguous(), "lse must be float32 and contiguous, of shape ",
                          in.q.sizes().slice(0, 4));
        const c10::cuda::CUDAGuard guard(in.q.device());
        make_readable(in);
        const at::Tensor out = attendable(saved[4]), rest = attendable(saved[6]), dout = attendable(gradient(grads[0], in.q));
        at::Tensor dq = attention_result_like(in.q), dk = attention_result_like(in.k), dv = attention_result_like(in.v);
        const sna_dtype_t dtype = dtype_of(in.q, "q");
        sna_attention_t a = described(in);
        a.out = described(out); a.out_rest = described(rest); a.dout = described(dout);
        a.dq = described(dq); a.dk = described(dk); a.dv = described(dv);
        a.lse = const_cast<float*>(lse.const_data_ptr<float>());
        const size_t bytes = sna_attention_backward_workspace_bytes(&a, dtype);
        at::Tensor workspace;
        if (bytes > 0) workspace = at::empty({(int64_t)bytes}, in.q.options().dtype(at::kByte));
        check(sna_attention_backward(&a, dtype, bytes ? workspace.data_ptr() : nullptr, bytes, stream_of(in.q)));
        return {dq, dk, dv, Variable(), Variable()};
    }
};

std::tuple<at::Tensor, at::Tensor> weighted_attention(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const std::optional<at::Tensor>& log_weights, double scale) {
    AttentionInputs in{q, k, v, or_undefined(log_weights), scale};
    check_attention(in);
    if (wants_grad({&q, &k, &v})) {
        const variable_list r = WeightedAttention::apply(q, k, v, log_weights, scale);
        return {r[0], r[1]};
    }
    auto [out, lse, rest] = attention_forward(in, false);
    return {out, lse};
}

// ---- dropout --------------------------------------------------------------------------------------------------------------

at::Tensor dropout_into(const at::Tensor& x, const at::Tensor& residual, const at::Tensor& state, double p) {
    const c10::cuda::CUDAGuard guard(x.device());
    at::Tensor out = at::empty_like(x, at::MemoryFormat::Contiguous);
    check(sna_dropout(x.data_ptr(), residual.defined() ? residual.data_ptr() : nullptr, out.data_ptr(), dtype_of(x, "x"), x.numel(), p, state.const_data_ptr<int64_t>(), stream_of(x)));
    return out;
}
void check_state(const at::Tensor& state, const at::Tensor& x) {
    TORCH_CHECK_VALUE(state.defined(), "state is missing");
    check_cuda(state, "state", x, "x");
    TORCH_CHECK_VALUE(state.scalar_type() == at::kLong && state.dim() == 1 && state.size(0) == 2 && state.is_contiguous(), "state must be int64 of shape [2] (seed, offset), contiguous");
}

class ResidualDropout : public torch::autograd::Function<ResidualDropout> {
public:
    static at::Tensor forward(AutogradContext* ctx, at::Tensor x, std::optional<at::Tensor> residual_, at::Tensor state, double p) {
        const at::Tensor residual = or_undefined(residual_);
        ctx->save_for_backward({state});
        ctx->saved_data["p"] = p;
        ctx->saved_data["x"] = x.requires_grad();
        ctx->saved_data["residual"] = residual.defined() && residual.requires_grad();
        return dropout_into(x.contiguous(), residual.defined() ? residual.contiguous() : residual, state, p);
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads) {
        check_once_differentiable("residual_dropout");
        const at::Tensor state = ctx->get_saved_variables()[0];
        check_no_tangent(grads[0], "the gradient");
        const at::Tensor dout = grads[0].resolve_neg();
        check_state(state, dout);
        variable_list result(4);
        if (ctx->saved_data["x"].toBool()) result[0] = dropout_into(dout.contiguous(), at::Tensor(), state, ctx->saved_data["p"].toDouble());
        if (ctx->saved_data["residual"].toBool()) result[1] = dout;
        return result;
    }
};

at::Tensor residual_dropout(const at::Tensor& x, const at::Tensor& state, double p, const std::optional<at::Tensor>& residual_) {
    const at::Tensor residual = or_undefined(residual_);
    TORCH_CHECK_VALUE(x.is_cuda(), "x must be a CUDA tensor");
    check_cuda(x, "x", x, "x");
    dtype_of(x, "x");
    check_state(state, x);
    TORCH_CHECK_VALUE(p >= 0.0 && p < 1.0, "p must be at least 0 and less than 1, got ", p);
    if (residual.defined()) {
        check_like(residual, "residual", x, "x");
        TORCH_CHECK_VALUE(residual.sizes() == x.sizes(), "residual has shape ", residual.sizes(), ", expected ", x.sizes());
    }
    if (wants_grad({&x, &residual})) return ResidualDropout::apply(x, residual_, state, p);
    return dropout_into(x.contiguous(), residual.defined() ? residual.contiguous() : residual, state, p);
}

}  // namespace

namespace sna_torch {
void bind_layer(py::module_& m) {
    m.def("qk_norm_rotate", &qk_norm_rotate, py::call_guard<py::gil_scoped_release>());
    m.def("weighted_attention", &weighted_attention, py::call_guard<py::gil_scoped_release>());
    m.def("residual_dropout", &residual_dropout, py::call_guard<py::gil_scoped_release>());
}
}  // namespace sna_torch
