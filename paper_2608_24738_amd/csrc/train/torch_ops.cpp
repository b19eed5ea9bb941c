// torch_ops.cpp -- the operators around a vocabulary as torch functions with
// gradients: checks of arguments, outputs and workspaces, and the calls of the
// C-ABI (include/tm_train.h) on the current stream.  No arithmetic happens here.
//
// In C++, since small calls are bound by the host and a backward pass runs on
// autograd's own thread, where Python code first waits for the interpreter: a
// forward and backward pass of layer norm took 122 us of host time from Python.
#include <torch/extension.h>

#include <ATen/core/grad_mode.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/custom_function.h>

#include <cmath>
#include <limits>
#include <optional>
#include <tuple>

#include "../../../include/tm_train.h"

namespace {

using at::Tensor;
using std::optional;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

int float_type(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return TM_DTYPE_F32;
        case at::kHalf: return TM_DTYPE_F16;
        case at::kBFloat16: return TM_DTYPE_BF16;
        default: return -1;
    }
}
int whole_type(at::ScalarType t) {
    switch (t) {
        case at::kByte: return TM_DTYPE_U8;
        case at::kInt: return TM_DTYPE_I32;
        case at::kLong: return TM_DTYPE_I64;
        default: return -1;
    }
}

void check_floats(const Tensor &t, const char *what) {
    TORCH_CHECK_TYPE(float_type(t.scalar_type()) >= 0, what, " must be float32, float16 or bfloat16, got ", t.scalar_type());
}
void check_on_gpu(const Tensor &t, const char *what) {
    TORCH_CHECK_VALUE(t.is_cuda(), what, " must be a ROCm (cuda) tensor");
}
void check_beside(const Tensor &t, const char *what, const Tensor &other, const char *which) {
    TORCH_CHECK_VALUE(t.device() == other.device(), what, " must be on ", other.device(), " as ", which, ", got ", t.device());
}
// Whole numbers that name rows of a table, contiguous; bools count as 0 and 1.
Tensor check_tokens(const Tensor &t, const char *what, const Tensor &other, const char *which) {
    check_beside(t, what, other, which);
    const Tensor plain = t.scalar_type() == at::kBool ? t.contiguous().view(at::kByte) : t;
    TORCH_CHECK_TYPE(whole_type(plain.scalar_type()) >= 0, what, " must be uint8, bool, int32 or int64, got ", t.scalar_type());
    return plain.contiguous();
}

// A status of the library as an exception.
void done(int status, const char *name) {
    TORCH_CHECK(status == TM_OK, name, " failed: ", tm_strerror(status), " (status ", status, ")");
}

// A tensor (..., width) as rows whose elements lie side by side, `stride` apart, or a contiguous copy of it.
struct Rows {
    Tensor t;
    int64_t rows, width, stride;
};
Rows rows_of(const Tensor &t) {
    const int64_t dims = t.dim(), width = t.size(-1);
    int64_t extent = 1, step = width;
    bool one = t.stride(-1) == 1 || width == 1;
    for (int64_t a = dims - 2; a >= 0 && one; --a) {
        const int64_t n = t.size(a), st = t.stride(a);
        if (n == 1) continue;
        if (extent == 1)
            step = st;
        else
            one = st == extent * step;
        extent *= n;
    }
    if (t.numel() == 0) return {t, width ? t.numel() / width : 0, width, width};
    if (one && step >= 0) return {t, extent, width, step};
    return {t.contiguous(), t.numel() / width, width, width};
}

struct Call {
    c10::DeviceGuard guard;
    hipStream_t stream;
    explicit Call(const Tensor &t) : guard(t.device()), stream(c10::hip::getCurrentHIPStream(t.device().index()).stream()) {}
};

Tensor floats(at::IntArrayRef shape, const Tensor &like) { return at::empty(shape, like.options().dtype(at::kFloat)); }
Tensor room(size_t bytes, const Tensor &like) {
    return bytes ? at::empty({int64_t(bytes)}, like.options().dtype(at::kByte)) : Tensor();
}
void *at_of(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
float *floats_of(const Tensor &t) { return static_cast<float *>(at_of(t)); }

void once() {
    TORCH_CHECK(!at::GradMode::is_enabled(), "the training operators can be differentiated once only");
}
// What autograd kept, dense: hooks on saved tensors may give it another layout, nothing else.
void unchanged(const Tensor &t, at::ScalarType type, at::IntArrayRef shape, c10::Device device) {
    TORCH_CHECK(t.scalar_type() == type && t.device() == device && t.sizes() == shape,
                "a hook on saved tensors gave back another type, shape or device");
}
Tensor restored(const Tensor &t, at::ScalarType type, at::IntArrayRef shape, c10::Device device) {
    if (!t.defined()) return t;
    unchanged(t, type, shape, device);
    return t.contiguous();
}
bool learns(const Tensor &t) { return t.defined() && t.requires_grad(); }
std::vector<int64_t> with(at::IntArrayRef shape, int64_t last) {
    std::vector<int64_t> out(shape.begin(), shape.end());
    out.push_back(last);
    return out;
}

// ---------------------------------------------------------------------------
// Layer norm.
// ---------------------------------------------------------------------------

std::tuple<Rows, Tensor, Tensor> norm_forward(const Tensor &x, const Tensor &weight, const Tensor &bias, double eps, bool keep) {
    const Tensor out = at::empty(x.sizes(), x.options());
    const Tensor kept = keep ? floats(with(x.sizes().slice(0, x.dim() - 1), 2), x) : Tensor();
    Rows r = rows_of(x);
    const Tensor &param = weight.defined() ? weight : bias;
    const Call call(x);
    done(tm_layer_norm(r.t.data_ptr(), float_type(x.scalar_type()), r.rows, r.width, r.stride, at_of(weight), at_of(bias),
                       param.defined() ? float_type(param.scalar_type()) : 0, eps, out.data_ptr(), floats_of(kept),
                       call.stream),
         "tm_layer_norm");
    return {std::move(r), out, kept};
}

struct LayerNorm : torch::autograd::Function<LayerNorm> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, const optional<Tensor> &weight, const optional<Tensor> &bias,
                          double eps) {
        const Tensor w = weight.value_or(Tensor()), b = bias.value_or(Tensor());
        auto [rows, out, kept] = norm_forward(x, w, b, eps, true);
        ctx->save_for_backward({rows.t, w, kept});
        ctx->saved_data["weight"] = w.defined();
        ctx->saved_data["bias"] = b.defined();
        if (w.defined() || b.defined()) ctx->saved_data["type"] = int64_t((w.defined() ? w : b).scalar_type());
        return out;
    }
    static variable_list backward(AutogradContext *ctx, variable_list ups) {
        once();
        const bool has_w = ctx->saved_data["weight"].toBool(), has_b = ctx->saved_data["bias"].toBool();
        const auto type = has_w || has_b ? at::ScalarType(ctx->saved_data["type"].toInt()) : at::kFloat;
        // the gradients' numbers count the tensors that were given
        const bool wants_x = ctx->needs_input_grad(0), wants_w = has_w && ctx->needs_input_grad(1),
                   wants_b = has_b && ctx->needs_input_grad(has_w ? 2 : 1);
        if (!wants_x && !wants_w && !wants_b) return {Tensor(), Tensor(), Tensor(), Tensor()};
        const variable_list saved = ctx->get_saved_variables();
        const Tensor up = ups[0].contiguous();
        const c10::Device dev = up.device();
        unchanged(saved[0], up.scalar_type(), up.sizes(), dev);
        const Rows r = rows_of(saved[0]);
        const Tensor weight = restored(saved[1], type, {r.width}, dev);
        const Tensor kept = restored(saved[2], at::kFloat, with(up.sizes().slice(0, up.dim() - 1), 2), dev);
        const auto params = up.options().dtype(type);
        const Tensor dx = wants_x ? at::empty(up.sizes(), up.options()) : Tensor();
        const Tensor dw = wants_w ? at::empty({r.width}, params) : Tensor();
        const Tensor db = wants_b ? at::empty({r.width}, params) : Tensor();
        const int dtype = float_type(up.scalar_type());
        const size_t bytes = wants_w || wants_b ? tm_layer_norm_grad_workspace_size(dtype, r.rows, r.width) : 0;
        const Tensor workspace = room(bytes, up);
        const Call call(up);
        done(tm_layer_norm_grad(r.t.data_ptr(), dtype, r.rows, r.width, r.stride, at_of(weight), float_type(type),
                                floats_of(kept), up.data_ptr(), at_of(dx), at_of(dw), at_of(db), at_of(workspace), bytes,
                                call.stream),
             "tm_layer_norm_grad");
        return {dx, dw, db, Tensor()};
    }
};

Tensor layer_norm(const Tensor &x, const optional<Tensor> &weight, const optional<Tensor> &bias, double eps) {
    check_on_gpu(x, "x");
    check_floats(x, "x");
    TORCH_CHECK_VALUE(x.dim() >= 1 && x.size(-1) >= 1, "x must be (..., width), got ", x.sizes());
    Tensor params[2];
    const char *names[2] = {"weight", "bias"};
    for (int i = 0; i < 2; ++i) {
        const optional<Tensor> &p = i ? bias : weight;
        if (!p) continue;
        check_floats(*p, names[i]);
        check_beside(*p, names[i], x, "x");
        TORCH_CHECK_VALUE(p->dim() == 1 && p->size(0) == x.size(-1), names[i], " must be (", x.size(-1), ",), got ", p->sizes());
        params[i] = p->contiguous();
    }
    TORCH_CHECK_TYPE(!weight || !bias || weight->scalar_type() == bias->scalar_type(),
                     "weight and bias must have one type, got ", weight->scalar_type(), " and ", bias->scalar_type());
    TORCH_CHECK_VALUE(float(eps) >= std::numeric_limits<float>::min() && std::isfinite(float(eps)),
                      "eps must be positive and finite, got ", eps);
    if (at::GradMode::is_enabled() && (learns(x) || learns(params[0]) || learns(params[1])))
        return LayerNorm::apply(x, weight ? optional<Tensor>(params[0]) : std::nullopt,
                                bias ? optional<Tensor>(params[1]) : std::nullopt, eps);
    return std::get<1>(norm_forward(x, params[0], params[1], eps, false));
}

// ---------------------------------------------------------------------------
// Rows of a table.
// ---------------------------------------------------------------------------

Tensor embedding_forward(const Tensor &tokens, const Tensor &table, double scale) {
    const Tensor out = at::empty(with(tokens.sizes(), table.size(1)), table.options());
    const Rows r = rows_of(table);
    const Call call(table);
    done(tm_embedding(r.t.data_ptr(), float_type(table.scalar_type()), r.rows, r.width, r.stride, tokens.data_ptr(),
                      whole_type(tokens.scalar_type()), tokens.numel(), scale, out.data_ptr(), call.stream),
         "tm_embedding");
    return out;
}

struct Embedding : torch::autograd::Function<Embedding> {
    static Tensor forward(AutogradContext *ctx, const Tensor &table, const Tensor &tokens, double scale) {
        ctx->save_for_backward({tokens});
        ctx->saved_data["rows"] = table.size(0);
        ctx->saved_data["type"] = int64_t(tokens.scalar_type());
        ctx->saved_data["scale"] = scale;
        return embedding_forward(tokens, table, scale);
    }
    static variable_list backward(AutogradContext *ctx, variable_list ups) {
        once();
        if (!ctx->needs_input_grad(0)) return {Tensor(), Tensor(), Tensor()};
        const Tensor up = ups[0].contiguous();
        const auto type = at::ScalarType(ctx->saved_data["type"].toInt());
        const Tensor tokens = restored(ctx->get_saved_variables()[0], type, up.sizes().slice(0, up.dim() - 1), up.device());
        const int64_t rows = ctx->saved_data["rows"].toInt(), width = up.size(-1);
        const Tensor grad = at::empty({rows, width}, up.options());
        const size_t bytes = tm_embedding_grad_workspace_size(rows, width, tokens.numel());
        const Tensor workspace = room(bytes, up);
        const Call call(up);
        done(tm_embedding_grad(tokens.data_ptr(), whole_type(type), tokens.numel(), up.data_ptr(),
                               float_type(up.scalar_type()), rows, width, ctx->saved_data["scale"].toDouble(),
                               grad.data_ptr(), at_of(workspace), bytes, call.stream),
             "tm_embedding_grad");
        return {grad, Tensor(), Tensor()};
    }
};

Tensor embedding(const Tensor &tokens, const Tensor &table, double scale) {
    check_on_gpu(table, "table");
    check_floats(table, "table");
    TORCH_CHECK_VALUE(table.dim() == 2 && table.size(0) >= 1 && table.size(1) >= 1, "table must be (rows, width), got ",
                      table.sizes());
    const Tensor plain = check_tokens(tokens, "tokens", table, "the table");
    TORCH_CHECK_VALUE(std::isfinite(float(scale)), "scale must be finite, got ", scale);
    if (at::GradMode::is_enabled() && table.requires_grad()) return Embedding::apply(table, plain, scale);
    return embedding_forward(plain, table, scale);
}

// ---------------------------------------------------------------------------
// Log-probabilities from hidden states.
// ---------------------------------------------------------------------------

struct HeadOut {
    Tensor hidden, weight;      // as they were read
    Tensor logp, sums, kept;
};

HeadOut head_forward(const Tensor &hidden, const Tensor &weight, const Tensor &labels, double scale, bool sums, bool keep) {
    HeadOut out;
    const auto shape = hidden.sizes().slice(0, hidden.dim() - 1);
    if (labels.defined()) out.logp = floats(shape, hidden);
    if (sums) out.sums = floats(shape, hidden);
    if (keep) out.kept = floats(with(shape, 2), hidden);
    const Rows h = rows_of(hidden), w = rows_of(weight);
    const int dtype = float_type(hidden.scalar_type());
    const size_t bytes = tm_head_logp_workspace_size(dtype, h.rows, w.rows, h.width, w.t.data_ptr(), w.stride);
    const Tensor workspace = room(bytes, hidden);
    const Call call(hidden);
    done(tm_head_logp(h.t.data_ptr(), dtype, h.rows, w.rows, h.width, h.stride, w.t.data_ptr(), w.stride, at_of(labels),
                      labels.defined() ? whole_type(labels.scalar_type()) : 0, scale, floats_of(out.logp),
                      floats_of(out.sums), floats_of(out.kept), at_of(workspace), bytes, call.stream),
         "tm_head_logp");
    out.hidden = h.t;
    out.weight = w.t;
    return out;
}

struct HeadLogProbs : torch::autograd::Function<HeadLogProbs> {
    static variable_list forward(AutogradContext *ctx, const Tensor &hidden, const Tensor &weight,
                                 const optional<Tensor> &labels, double scale, bool sums) {
        const Tensor y = labels.value_or(Tensor());
        HeadOut out = head_forward(hidden, weight, y, scale, sums, true);
        ctx->set_materialize_grads(false);
        ctx->save_for_backward({out.hidden, out.weight, y, out.kept});
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["type"] = int64_t(hidden.scalar_type());
        ctx->saved_data["shape"] = hidden.sizes();
        ctx->saved_data["classes"] = weight.size(0);
        if (y.defined()) ctx->saved_data["label_type"] = int64_t(y.scalar_type());
        variable_list outs;
        if (y.defined()) outs.push_back(out.logp);
        if (sums) outs.push_back(out.sums);
        return outs;
    }
    static variable_list backward(AutogradContext *ctx, variable_list ups) {
        once();
        const bool wants_h = ctx->needs_input_grad(0), wants_w = ctx->needs_input_grad(1);
        const variable_list none(5);
        if (!wants_h && !wants_w) return none;
        const variable_list saved = ctx->get_saved_variables();
        const bool labelled = ctx->saved_data.count("label_type") > 0;
        Tensor up_logp = labelled ? ups[0] : Tensor(), up_sums = labelled ? (ups.size() > 1 ? ups[1] : Tensor()) : ups[0];
        if (!up_logp.defined() && !up_sums.defined()) return none;
        if (up_logp.defined()) up_logp = up_logp.to(at::kFloat).contiguous();
        if (up_sums.defined()) up_sums = up_sums.to(at::kFloat).contiguous();
        const c10::Device dev = (up_logp.defined() ? up_logp : up_sums).device();
        const auto type = at::ScalarType(ctx->saved_data["type"].toInt());
        const std::vector<int64_t> shape = ctx->saved_data["shape"].toIntVector();
        const int64_t classes = ctx->saved_data["classes"].toInt(), width = shape.back();
        const at::IntArrayRef lead = at::IntArrayRef(shape).slice(0, shape.size() - 1);
        unchanged(saved[0], type, shape, dev);
        unchanged(saved[1], type, {classes, width}, dev);
        const Tensor labels = labelled ? restored(saved[2], at::ScalarType(ctx->saved_data["label_type"].toInt()), lead, dev)
                                       : Tensor();
        const Tensor kept = restored(saved[3], at::kFloat, with(lead, 2), dev);
        const Rows h = rows_of(saved[0]), w = rows_of(saved[1]);
        const Tensor dh = wants_h ? at::empty(shape, h.t.options()) : Tensor();
        const Tensor dw = wants_w ? at::empty({classes, width}, w.t.options()) : Tensor();
        const int dtype = float_type(type);
        const size_t bytes = tm_head_logp_grad_workspace_size(dtype, h.rows, w.rows, width, w.t.data_ptr(), w.stride,
                                                              wants_h, wants_w);
        const Tensor workspace = room(bytes, kept);
        const Call call(kept);
        done(tm_head_logp_grad(h.t.data_ptr(), dtype, h.rows, w.rows, width, h.stride, w.t.data_ptr(), w.stride,
                               at_of(labels), labelled ? whole_type(labels.scalar_type()) : 0,
                               ctx->saved_data["scale"].toDouble(), floats_of(kept), floats_of(up_logp), floats_of(up_sums),
                               at_of(dh), at_of(dw), at_of(workspace), bytes, call.stream),
             "tm_head_logp_grad");
        return {dh, dw, Tensor(), Tensor(), Tensor()};
    }
};

std::tuple<optional<Tensor>, optional<Tensor>> head_log_probs(const Tensor &hidden, const Tensor &weight,
                                                              const optional<Tensor> &labels, double scale, bool sums) {
    check_on_gpu(hidden, "hidden");
    check_floats(hidden, "hidden");
    TORCH_CHECK_VALUE(hidden.dim() >= 1 && weight.dim() == 2 && weight.size(0) >= 1 && weight.size(1) >= 1,
                      "hidden must be (..., width) and weight (classes, width), got ", hidden.sizes(), " and ", weight.sizes());
    TORCH_CHECK_TYPE(weight.scalar_type() == hidden.scalar_type(), "weight must be ", hidden.scalar_type(),
                     " as the hidden states are, got ", weight.scalar_type());
    check_beside(weight, "weight", hidden, "the hidden states");
    TORCH_CHECK_VALUE(weight.size(1) == hidden.size(-1), "hidden states of width ", hidden.size(-1),
                      " do not fit a weight of width ", weight.size(1));
    Tensor y;
    if (labels) {
        y = check_tokens(*labels, "labels", hidden, "the hidden states");
        TORCH_CHECK_VALUE(y.sizes() == hidden.sizes().slice(0, hidden.dim() - 1), "labels of shape ", y.sizes(),
                          " do not fit hidden states of shape ", hidden.sizes());
    }
    TORCH_CHECK_VALUE(float(scale) > std::numeric_limits<float>::min() && std::isfinite(float(scale) * 1.5f),
                      "scale must be positive and finite, got ", scale);
    TORCH_CHECK_VALUE(labels || sums, "nothing to compute: give labels or ask for log_sums");
    Tensor logp, total;
    if (at::GradMode::is_enabled() && (hidden.requires_grad() || weight.requires_grad())) {
        const variable_list outs = HeadLogProbs::apply(hidden, weight, labels ? optional<Tensor>(y) : std::nullopt, scale, sums);
        if (labels) logp = outs[0];
        if (sums) total = outs[labels ? 1 : 0];
    } else {
        const HeadOut out = head_forward(hidden, weight, y, scale, sums, false);
        logp = out.logp;
        total = out.sums;
    }
    return {labels ? optional<Tensor>(logp) : std::nullopt, sums ? optional<Tensor>(total) : std::nullopt};
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
    m.doc() = "The operators around a vocabulary (module training has their documentation).";
    m.def("layer_norm", torch::wrap_pybind_function(&layer_norm));
    m.def("embedding", torch::wrap_pybind_function(&embedding));
    m.def("head_log_probs", torch::wrap_pybind_function(&head_log_probs));
}
