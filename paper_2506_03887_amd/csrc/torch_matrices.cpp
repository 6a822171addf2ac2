// The calls on a model's table and head as torch has them: their checks of tensors, and lookup and loss as nodes of the autograd graph (in C++ as
// the distillation's, whose backward pass does not wait for the interpreter either).
#include <climits>
#include <tuple>

#include "torch_tensors.hpp"

namespace {

bool is_float(const Tensor &t) { return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kHalf || t.scalar_type() == at::kFloat; }
bool is_id(const Tensor &t) { return t.scalar_type() == at::kInt || t.scalar_type() == at::kLong; }
bool is_matrix(const Tensor &t) { return t.dim() == 2 && (t.stride(1) == 1 || t.size(1) <= 1) && t.stride(0) >= 0 && t.size(0) <= INT_MAX && t.size(1) <= INT_MAX; }
Tensor bytes(int64_t n, const Tensor &like) { return at::empty({std::max<int64_t>(n, 1)}, like.options().dtype(at::kByte).requires_grad(false)); }
// (rows that repeat one, as an expanded gradient's do, are laid out)
Tensor rows_of(const Tensor &t) { return t.dim() == 2 && (t.stride(1) == 1 || t.size(1) <= 1) && (t.size(0) <= 1 || t.stride(0) >= t.size(1)) ? t : t.contiguous(); }
// (a tangent would be lost, and the result read as constant)
void refuse_tangents(std::initializer_list<const Tensor *> tensors, const char *call) {
    for (const Tensor *t : tensors) TORCH_CHECK_NOT_IMPLEMENTED(!t->_fw_grad(0).defined(), call, " has no forward-mode derivative");
}
// (written behind autograd's back: its history would stay)
void refuse_history(const MaybeTensor &out) { expect(!out || !at::GradMode::is_enabled() || !out->requires_grad(), "out: not part of an autograd graph"); }
void check_workspace(int64_t need, const char *call) { if (need < 0) expect_ok((int)need, call); }
// In a backward pass, on a thread of the engine's, errors are torch's own.
void check_status(int64_t status, const char *call) { TORCH_CHECK(status >= 0, "pre3 status ", status, ": ", refusal(call)); }

// ---- the table

pre3_embedding embedding(const Tensor *table, const Tensor &ids, at::ScalarType type, int64_t vocab, int64_t dim, double scale) {
    pre3_embedding e{};
    e.table = table ? table->data_ptr() : nullptr;
    e.ids = ids.data_ptr();
    e.table_stride = table ? row_stride(*table) : dim;
    e.type = type_of_logits(type);
    e.id_bytes = (int32_t)ids.element_size();
    e.rows = (int32_t)ids.numel();
    e.vocab = (int32_t)vocab;
    e.dim = (int32_t)dim;
    e.scale = (float)scale;
    return e;
}
Tensor lookup(const Tensor &weight, const Tensor &tokens, double scale, const MaybeTensor &out) {
    const c10::DeviceGuard guard(weight.device());
    std::vector<int64_t> shape(tokens.sizes().begin(), tokens.sizes().end());
    shape.push_back(weight.size(1));
    const Tensor to = out ? *out : at::empty(shape, weight.options().requires_grad(false));
    const pre3_embedding e = embedding(&weight, tokens, weight.scalar_type(), weight.size(0), weight.size(1), scale);
    expect_ok(pre3_embed(&e, to.data_ptr(), weight.size(1), stream_of(weight)), "pre3_embed");
    return to;
}

struct Embed : torch::autograd::Function<Embed> {
    static Tensor forward(AutogradContext *ctx, const Tensor &weight, const Tensor &tokens, double scale) {
        ctx->save_for_backward({tokens});
        ctx->saved_data["vocab"] = weight.size(0);
        ctx->saved_data["scale"] = scale;
        return lookup(weight, tokens, scale, std::nullopt);
    }
    static variable_list backward(AutogradContext *ctx, variable_list upstream) {
        TORCH_CHECK(!at::GradMode::is_enabled(), "embed is differentiable once");              // create_graph=True
        const Tensor tokens = ctx->get_saved_variables()[0];
        const int64_t dim = upstream[0].size(-1), vocab = ctx->saved_data["vocab"].toInt();
        const c10::DeviceGuard guard(upstream[0].device());
        const Tensor rows = rows_of(upstream[0].reshape({-1, dim}));
        const pre3_embedding e = embedding(nullptr, tokens, rows.scalar_type(), vocab, dim, ctx->saved_data["scale"].toDouble());
        const int64_t need = pre3_embed_workspace_bytes(e.rows, e.dim);
        check_status(need, "pre3_embed_workspace_bytes");
        const Tensor workspace = bytes(need, rows), grad = at::empty({vocab, dim}, rows.options().requires_grad(false));
        check_status(pre3_embed_grad(&e, rows.data_ptr(), row_stride(rows), grad.data_ptr(), workspace.data_ptr(), need, stream_of(rows)), "pre3_embed_grad");
        return {grad, Tensor(), Tensor()};
    }
};

Tensor embed(const Tensor &weight, const Tensor &tokens, double scale, const MaybeTensor &out) {
    refuse_tangents({&weight}, "embed");
    refuse_history(out);
    expect(is_matrix(weight) && weight.size(0) > 0 && weight.size(1) > 0 && (weight.size(0) == 1 || weight.stride(0) >= weight.size(1)),
           "weight: [vocab, dim], the second dimension contiguous");
    expect(tokens.is_contiguous() && tokens.numel() <= INT_MAX, "tokens: contiguous");
    expect(on(tokens, weight), "tensors on several devices");
    expect_kind(weight, is_float(weight), "logits");
    expect_kind(tokens, is_id(tokens), "i32 or i64");
    const bool graph = at::GradMode::is_enabled() && weight.requires_grad();
    if (out) {
        expect(!graph, "out: not where a gradient is asked for");
        expect(out->is_contiguous() && out->dim() == tokens.dim() + 1 && out->sizes().slice(0, tokens.dim()) == tokens.sizes() && out->size(-1) == weight.size(1) &&
                   out->scalar_type() == weight.scalar_type() && on(*out, weight),
               "out: [tokens' shape, dim], contiguous, of the weight's type and device");
    }
    if (graph) return Embed::apply(weight, tokens, scale);
    const Tensor to = lookup(weight, tokens, scale, out);
    if (out) written(to);
    return to;
}

// ---- the head's loss

void expect_mask(const MaybeTensor &mask, int64_t rows, int64_t vocab, const Tensor &like) {
    if (!mask) return;
    expect(mask->dim() == 2 && mask->size(0) == rows && mask->size(1) == (vocab + 31) / 32 && mask->is_contiguous() && on(*mask, like),
           "bitmask: [rows, ceil(vocab / 32)], contiguous, on the hidden states' device");
    expect_kind(*mask, is_word(*mask), "u32");
}
void expect_head(const Tensor &hidden, const Tensor &weight, const Tensor &targets, const MaybeTensor &mask) {
    expect(is_matrix(hidden) && hidden.size(1) > 0, "hidden: [rows, dim], the second dimension contiguous");
    expect(is_matrix(weight) && weight.size(0) > 0 && weight.size(1) == hidden.size(1), "weight: [vocab, dim], the second dimension contiguous");
    expect(hidden.size(0) <= 1 || hidden.stride(0) >= hidden.size(1), "hidden: rows that overlap");
    expect(weight.size(0) == 1 || weight.stride(0) >= weight.size(1), "weight: rows that overlap");
    expect(targets.dim() == 1 && targets.size(0) == hidden.size(0) && targets.is_contiguous(), "targets: [rows], contiguous");
    expect(on(weight, hidden) && on(targets, hidden), "tensors on several devices");
    expect_kind(hidden, is_float(hidden), "logits");
    expect(weight.scalar_type() == hidden.scalar_type(), "hidden and weight: of one type");
    expect_kind(targets, is_id(targets), "i32 or i64");
    expect_mask(mask, hidden.size(0), weight.size(0), hidden);
}
pre3_head head_of(const Tensor &hidden, const Tensor &weight, const Tensor &targets, const MaybeTensor &mask) {
    pre3_head h{};
    h.hidden = hidden.data_ptr();
    h.weight = weight.data_ptr();
    h.targets = targets.data_ptr();
    h.bitmask = mask ? static_cast<const uint32_t *>(mask->data_ptr()) : nullptr;
    h.hidden_stride = row_stride(hidden);
    h.weight_stride = row_stride(weight);
    h.type = type_of_logits(hidden.scalar_type());
    h.target_bytes = (int32_t)targets.element_size();
    h.rows = (int32_t)hidden.size(0);
    h.vocab = (int32_t)weight.size(0);
    h.dim = (int32_t)hidden.size(1);
    return h;
}
// The workspace, which has to live until the launch: what the allocator gives away after that, it gives to the same stream.
Tensor workspace_for(pre3_head &h, int64_t need, const Tensor &like) {
    const Tensor workspace = bytes(need, like);
    h.workspace = workspace.data_ptr();
    h.workspace_bytes = need;
    return workspace;
}
// The loss; with `stats` and `kept`, what the backward pass needs.
Tensor head_loss_of(const Tensor &hidden, const Tensor &weight, const Tensor &targets, const MaybeTensor &mask, Tensor *stats, Tensor *kept) {
    const c10::DeviceGuard guard(hidden.device());
    pre3_head h = head_of(hidden, weight, targets, mask);
    const int64_t need = pre3_head_workspace_bytes(&h, stats ? PRE3_HEAD_LOSS : PRE3_HEAD_LOSS_ALONE);
    check_workspace(need, "pre3_head_workspace_bytes");
    const Tensor workspace = workspace_for(h, need, hidden);
    Tensor loss = at::empty({h.rows}, floats(hidden));
    if (stats) *stats = at::empty({h.rows, 2}, floats(hidden));
    if (kept) {
        const int64_t size = pre3_head_kept_bytes(&h);
        check_workspace(size, "pre3_head_kept_bytes");
        *kept = bytes(size, hidden);
        h.kept = size ? kept->data_ptr() : nullptr;
    }
    expect_ok(pre3_head_loss(&h, loss.data_ptr<float>(), stats ? stats->data_ptr<float>() : nullptr, stream_of(hidden)), "pre3_head_loss");
    return loss;
}

struct HeadLoss : torch::autograd::Function<HeadLoss> {
    static Tensor forward(AutogradContext *ctx, const Tensor &hidden, const Tensor &weight, const Tensor &targets, const MaybeTensor &mask) {
        Tensor stats, kept, loss = head_loss_of(hidden, weight, targets, mask, &stats, &kept);
        ctx->save_for_backward({hidden, weight, targets, mask ? *mask : Tensor(), stats, kept});
        return loss;
    }
    static variable_list backward(AutogradContext *ctx, variable_list upstream) {
        TORCH_CHECK(!at::GradMode::is_enabled(), "head_loss is differentiable once");          // create_graph=True
        const variable_list saved = ctx->get_saved_variables();                                // (raises where one of them has been written since)
        const Tensor &hidden = saved[0], &weight = saved[1], up = upstream[0];
        const MaybeTensor mask = saved[3].defined() ? MaybeTensor(saved[3]) : std::nullopt;
        const c10::DeviceGuard guard(hidden.device());
        pre3_head h = head_of(hidden, weight, saved[2], mask);
        h.kept = saved[5].numel() ? saved[5].data_ptr() : nullptr;
        const int64_t need = pre3_head_workspace_bytes(&h, PRE3_HEAD_GRADIENTS);
        check_status(need, "pre3_head_workspace_bytes");
        const Tensor workspace = workspace_for(h, need, hidden);
        Tensor d_hidden, d_weight;
        if (ctx->needs_input_grad(0)) d_hidden = at::empty({h.rows, h.dim}, hidden.options().requires_grad(false));
        if (ctx->needs_input_grad(1)) d_weight = at::empty({h.vocab, h.dim}, weight.options().requires_grad(false));
        check_status(pre3_head_grad(&h, saved[4].data_ptr<float>(), up.data_ptr<float>(), up.stride(0), d_hidden.defined() ? d_hidden.data_ptr() : nullptr, h.dim,
                                    d_weight.defined() ? d_weight.data_ptr() : nullptr, h.dim, stream_of(hidden)),
                     "pre3_head_grad");
        return {d_hidden, d_weight, Tensor(), Tensor()};
    }
};

Tensor head_loss(const Tensor &hidden, const Tensor &weight, const Tensor &targets, const MaybeTensor &mask) {
    refuse_tangents({&hidden, &weight}, "head_loss");
    expect_head(hidden, weight, targets, mask);
    if (at::GradMode::is_enabled() && (hidden.requires_grad() || weight.requires_grad())) return HeadLoss::apply(hidden, weight, targets, mask);
    return head_loss_of(hidden, weight, targets, mask, nullptr, nullptr);
}

std::tuple<Tensor, Tensor, Tensor> head_loss_grad(const Tensor &of_hidden, const Tensor &of_weight, const Tensor &targets, const MaybeTensor &mask, const MaybeTensor &row_weight) {
    refuse_tangents({&of_hidden, &of_weight, row_weight ? &*row_weight : &of_weight}, "head_loss_grad");
    const Tensor hidden = of_hidden.detach(), weight = of_weight.detach();
    expect_head(hidden, weight, targets, mask);
    if (row_weight) {
        expect(row_weight->dim() == 1 && row_weight->size(0) == hidden.size(0) && on(*row_weight, hidden), "row_weight: [rows], on the hidden states' device");
        expect_kind(*row_weight, row_weight->scalar_type() == at::kFloat, "f32");
    }
    const c10::DeviceGuard guard(hidden.device());
    pre3_head h = head_of(hidden, weight, targets, mask);
    const int64_t need = pre3_head_workspace_bytes(&h, PRE3_HEAD_GRADIENTS);
    check_workspace(need, "pre3_head_workspace_bytes");
    const Tensor workspace = workspace_for(h, need, hidden), loss = at::empty({h.rows}, floats(hidden)), d_hidden = at::empty({h.rows, h.dim}, hidden.options()),
                 d_weight = at::empty({h.vocab, h.dim}, weight.options());
    expect_ok(pre3_head_loss_grad(&h, row_weight ? row_weight->data_ptr<float>() : nullptr, row_weight ? row_weight->stride(0) : 0, loss.data_ptr<float>(), d_hidden.data_ptr(), h.dim,
                                  d_weight.data_ptr(), h.dim, stream_of(hidden)),
              "pre3_head_loss_grad");
    return {loss, d_hidden, d_weight};
}

// ---- the head in 8 bits

std::tuple<Tensor, Tensor> quantise_rows(const Tensor &of) {
    refuse_tangents({&of}, "quantise_rows");
    const Tensor x = of.detach();
    expect(is_matrix(x) && x.size(1) > 0 && (x.size(0) <= 1 || x.stride(0) >= x.size(1)), "x: [rows, dim], the second dimension contiguous");
    expect_kind(x, is_float(x), "logits");
    const c10::DeviceGuard guard(x.device());
    const int64_t rows = x.size(0), dim = x.size(1), stride = (dim + 15) / 16 * 16;
    const Tensor out = at::empty({rows, stride}, x.options().dtype(at::kChar)), scale = at::empty({rows}, floats(x));
    expect_ok(pre3_quantise_rows(x.data_ptr(), type_of_logits(x.scalar_type()), row_stride(x), (int32_t)rows, (int32_t)dim, static_cast<int8_t *>(out.data_ptr()), stride,
                                 scale.data_ptr<float>(), stream_of(x)),
              "pre3_quantise_rows");
    return {out.narrow(1, 0, dim), scale};
}

Tensor head_logits(const Tensor &of, const Tensor &weight, const Tensor &scale, const MaybeTensor &mask, const MaybeTensor &out) {
    refuse_tangents({&of, &scale}, "head_logits");
    refuse_history(out);
    const Tensor hidden = of.detach();
    expect(is_matrix(hidden) && hidden.size(1) > 0 && (hidden.size(0) <= 1 || hidden.stride(0) >= hidden.size(1)), "hidden: [rows, dim], the second dimension contiguous");
    expect(is_matrix(weight) && weight.size(0) > 0 && weight.size(1) == hidden.size(1), "weight: [vocab, dim], the second dimension contiguous");
    const int64_t rows = hidden.size(0), dim = hidden.size(1), vocab = weight.size(0), whole = (dim + 15) / 16 * 16;
    // a single row's stride may be anything
    const int64_t stride = vocab > 1 ? weight.stride(0) : whole;
    expect(stride >= whole && stride % 16 == 0, "weight: rows at 16-byte boundaries, as quantise_rows lays them out");
    expect(scale.dim() == 1 && scale.size(0) == vocab && scale.is_contiguous(), "scale: [vocab], contiguous");
    expect(on(weight, hidden) && on(scale, hidden), "tensors on several devices");
    expect_kind(hidden, is_float(hidden), "logits");
    expect_kind(weight, weight.scalar_type() == at::kChar, "i8");
    expect_kind(scale, scale.scalar_type() == at::kFloat, "f32");
    expect(reinterpret_cast<uintptr_t>(weight.data_ptr()) % 16 == 0 && weight.storage_offset() + (vocab - 1) * stride + whole <= (int64_t)weight.storage().nbytes(),
           "weight: rows at 16-byte boundaries, as quantise_rows lays them out");
    expect_mask(mask, rows, vocab, hidden);
    if (out)
        expect(out->dim() == 2 && out->size(0) == rows && out->size(1) == vocab && out->scalar_type() == hidden.scalar_type() && on(*out, hidden) && (out->stride(1) == 1 || vocab == 1) &&
                   (rows <= 1 || out->stride(0) >= vocab),
               "out: [rows, vocab] of the hidden states' type and device, the second dimension contiguous");
    const c10::DeviceGuard guard(hidden.device());
    pre3_head8 h{};
    h.hidden = hidden.data_ptr();
    h.weight = static_cast<const int8_t *>(weight.data_ptr());
    h.weight_scale = scale.data_ptr<float>();
    h.bitmask = mask ? static_cast<const uint32_t *>(mask->data_ptr()) : nullptr;
    h.hidden_stride = row_stride(hidden);
    h.weight_stride = stride;
    h.type = type_of_logits(hidden.scalar_type());
    h.rows = (int32_t)rows;
    h.vocab = (int32_t)vocab;
    h.dim = (int32_t)dim;
    const int64_t need = pre3_head8_workspace_bytes(h.rows, h.dim);
    check_workspace(need, "pre3_head8_workspace_bytes");
    const Tensor workspace = bytes(need, hidden), to = out ? *out : at::empty({rows, vocab}, hidden.options());
    h.workspace = workspace.data_ptr();
    h.workspace_bytes = need;
    expect_ok(pre3_head8_logits(&h, to.data_ptr(), row_stride(to), stream_of(hidden)), "pre3_head8_logits");
    if (out) written(to);
    return to;
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
    m.def("embed", &embed);
    m.def("head_loss", &head_loss);
    m.def("head_loss_grad", &head_loss_grad);
    m.def("quantise_rows", &quantise_rows);
    m.def("head_logits", &head_logits);
    m.def("raise_as", [](pybind11::object error) { pre3_error = error.release().ptr(); });
}
