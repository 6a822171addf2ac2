// C ABI of the calls on the model's table and head (declared in include/pre3.h): argument checks and launches.
#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "../../include/pre3.h"
#include "launch.hpp"

using namespace pre3;

namespace {

bool is_type(int32_t type) { return type == kLogitBf16 || type == kLogitF16 || type == kLogitF32; }
bool is_aligned(const void *p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
uintptr_t bytes_of(int32_t type) { return type == kLogitF32 ? 4 : 2; }
bool id_width(int32_t bytes) { return bytes == 4 || bytes == 8; }
int status_of(hipError_t e) { return e == hipSuccess ? PRE3_OK : PRE3_E_HIP; }

// A workspace's address and size.
bool holds(const void *workspace, int64_t has, size_t needs, uintptr_t alignment) { return workspace && is_aligned(workspace, alignment) && has >= (int64_t)needs; }

int check(const pre3_embedding *e, bool table) {
    if (!e || e->rows < 0 || e->vocab < 1 || e->dim < 1 || !is_type(e->type) || !id_width(e->id_bytes)) return PRE3_E_BADARG;
    if (e->rows > kEmbedMostRows || e->vocab > kEmbedMostVocab || e->dim > kHeadMostDim) return PRE3_E_LIMIT;
    if (table && e->table_stride < e->dim) return PRE3_E_BADARG;
    if (e->rows == 0) return PRE3_OK;
    if (!e->ids || !is_aligned(e->ids, e->id_bytes)) return PRE3_E_BADARG;
    if (table && (!e->table || !is_aligned(e->table, bytes_of(e->type)))) return PRE3_E_BADARG;
    return PRE3_OK;
}
EmbedRows rows_of(const pre3_embedding *e) {
    return {e->table, e->ids, static_cast<LogitType>(e->type), e->id_bytes, e->rows, e->vocab, e->dim, e->table_stride, e->scale};
}

int check(const pre3_head *h) {
    if (!h || h->rows < 0 || h->vocab < 1 || h->dim < 1 || !is_type(h->type) || !id_width(h->target_bytes)) return PRE3_E_BADARG;
    if (h->rows > kHeadMostRows || h->vocab > kHeadMostVocab || h->dim > kHeadMostDim || (int64_t)h->rows * h->dim > kHeadMostHidden) return PRE3_E_LIMIT;
    if (h->hidden_stride < h->dim || h->weight_stride < h->dim) return PRE3_E_BADARG;
    if (h->rows == 0) return PRE3_OK;
    const uintptr_t size = bytes_of(h->type);
    if (!h->hidden || !h->weight || !h->targets || !is_aligned(h->hidden, size) || !is_aligned(h->weight, size) || !is_aligned(h->targets, h->target_bytes) ||
        !is_aligned(h->bitmask, 4) || !is_aligned(h->kept, 16))
        return PRE3_E_BADARG;
    return PRE3_OK;
}
HeadRows rows_of(const pre3_head *h) {
    return {h->hidden, h->weight, h->targets, static_cast<LogitType>(h->type), h->target_bytes, h->rows, h->vocab, h->dim, h->hidden_stride, h->weight_stride, h->bitmask,
            static_cast<float *>(h->kept)};
}
// forward: the loss is wanted; backward: the gradients that are not null.
int run(const pre3_head *h, bool forward, bool backward, float *loss, float *stats, const float *row_weight, int64_t weight_stride, void *grad_hidden, int64_t grad_hidden_stride,
        void *grad_weight, int64_t grad_weight_stride, pre3_stream stream) {
    const int bad = check(h);
    if (bad) return bad;
    const uintptr_t size = bytes_of(h->type);
    if (backward) {
        if (weight_stride < 0 || (grad_hidden && (grad_hidden_stride < h->dim || !is_aligned(grad_hidden, size))) ||
            (grad_weight && (grad_weight_stride < h->dim || !is_aligned(grad_weight, size))) || !is_aligned(row_weight, 4))
            return PRE3_E_BADARG;
        if (!grad_hidden && !grad_weight) backward = false;
    }
    if (h->rows == 0) return backward && grad_weight ? status_of(launch_zero_rows(grad_weight, static_cast<LogitType>(h->type), h->vocab, h->dim, grad_weight_stride, static_cast<hipStream_t>(stream)))
                                                     : PRE3_OK;
    if ((forward && !loss) || !is_aligned(loss, 4) || !is_aligned(stats, 8) || (!forward && !stats)) return PRE3_E_BADARG;
    if (!forward && !backward) return PRE3_OK;
    HeadRows rows = rows_of(h);
    if (forward && backward) rows.kept = nullptr;                         // (nothing is left to another call)
    if (!holds(h->workspace, h->workspace_bytes, head_call_bytes(rows, backward, !backward && head_is_alone(rows, forward, stats)), 256)) return PRE3_E_BADARG;
    return status_of(launch_head(rows, forward, backward, loss, stats, row_weight, weight_stride, grad_hidden, grad_hidden_stride, grad_weight, grad_weight_stride, h->workspace,
                                 static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int pre3_embed(const pre3_embedding *e, void *out, int64_t out_stride, pre3_stream stream) {
    const int bad = check(e, true);
    if (bad) return bad;
    if (out_stride < e->dim) return PRE3_E_BADARG;
    if (e->rows == 0) return PRE3_OK;
    if (!out || !is_aligned(out, bytes_of(e->type))) return PRE3_E_BADARG;
    return status_of(launch_embed(rows_of(e), out, out_stride, static_cast<hipStream_t>(stream)));
}

int64_t pre3_embed_workspace_bytes(int32_t rows, int32_t dim) {
    return rows < 0 || dim < 1 || rows > kEmbedMostRows || dim > kHeadMostDim ? PRE3_E_BADARG : (int64_t)embed_workspace_bytes(rows, dim);
}

int pre3_embed_grad(const pre3_embedding *e, const void *rows_grad, int64_t rows_stride, void *grad, void *workspace, int64_t workspace_bytes, pre3_stream stream) {
    const int bad = check(e, false);
    if (bad) return bad;
    if ((int64_t)e->vocab * e->dim * (int64_t)bytes_of(e->type) > kEmbedMostGradBytes) return PRE3_E_LIMIT;
    if (!grad || !is_aligned(grad, bytes_of(e->type)) || rows_stride < e->dim) return PRE3_E_BADARG;
    if (e->rows > 0 && (!rows_grad || !is_aligned(rows_grad, bytes_of(e->type)) || !holds(workspace, workspace_bytes, embed_workspace_bytes(e->rows, e->dim), 16))) return PRE3_E_BADARG;
    return status_of(launch_embed_grad(rows_of(e), rows_grad, rows_stride, grad, workspace, static_cast<hipStream_t>(stream)));
}

int64_t pre3_head_workspace_bytes(const pre3_head *h, int32_t calls) {
    const int bad = check(h);
    if (bad) return bad;
    return h->rows == 0 ? 0 : (int64_t)head_workspace_bytes(rows_of(h), calls == PRE3_HEAD_LOSS_ALONE ? HeadCalls::kLossAlone : calls == PRE3_HEAD_LOSS ? HeadCalls::kLoss : HeadCalls::kAll);
}

int64_t pre3_head_kept_bytes(const pre3_head *h) {
    const int bad = check(h);
    if (bad) return bad;
    return h->rows == 0 ? 0 : (int64_t)head_kept_bytes(rows_of(h));
}

int pre3_head_loss(const pre3_head *h, float *loss, float *stats, pre3_stream stream) {
    return run(h, true, false, loss, stats, nullptr, 0, nullptr, 0, nullptr, 0, stream);
}

int pre3_head_grad(const pre3_head *h, const float *stats, const float *row_weight, int64_t weight_stride, void *grad_hidden, int64_t grad_hidden_stride, void *grad_weight,
                   int64_t grad_weight_stride, pre3_stream stream) {
    return run(h, false, true, nullptr, const_cast<float *>(stats), row_weight, weight_stride, grad_hidden, grad_hidden_stride, grad_weight, grad_weight_stride, stream);
}

int pre3_head_loss_grad(const pre3_head *h, const float *row_weight, int64_t weight_stride, float *loss, void *grad_hidden, int64_t grad_hidden_stride, void *grad_weight,
                        int64_t grad_weight_stride, pre3_stream stream) {
    return run(h, true, true, loss, nullptr, row_weight, weight_stride, grad_hidden, grad_hidden_stride, grad_weight, grad_weight_stride, stream);
}

int pre3_quantise_rows(const void *x, int32_t type, int64_t x_stride, int32_t rows, int32_t dim, int8_t *out, int64_t out_stride, float *scale, pre3_stream stream) {
    if (rows < 0 || dim < 1 || !is_type(type) || x_stride < dim || out_stride < dim || out_stride % 16 != 0) return PRE3_E_BADARG;
    if (rows > kEmbedMostVocab || dim > kHeadMostDim) return PRE3_E_LIMIT;
    if (rows == 0) return PRE3_OK;
    if (!x || !out || !scale || !is_aligned(x, bytes_of(type)) || !is_aligned(out, 16) || !is_aligned(scale, 4)) return PRE3_E_BADARG;
    return status_of(launch_quantise(x, static_cast<LogitType>(type), x_stride, rows, dim, out, out_stride, scale, static_cast<hipStream_t>(stream)));
}

int64_t pre3_head8_workspace_bytes(int32_t rows, int32_t dim) {
    return rows < 0 || dim < 1 || rows > kHeadMostRows || dim > kHeadMostDim ? PRE3_E_BADARG : (int64_t)head8_workspace_bytes(rows, dim);
}

int pre3_head8_logits(const pre3_head8 *h, void *logits, int64_t logits_stride, pre3_stream stream) {
    if (!h || h->rows < 0 || h->vocab < 1 || h->dim < 1 || !is_type(h->type)) return PRE3_E_BADARG;
    if (h->rows > kHeadMostRows || h->vocab > kHeadMostVocab || h->dim > kHeadMostDim) return PRE3_E_LIMIT;
    if (h->hidden_stride < h->dim || h->weight_stride < h->dim || h->weight_stride % 16 != 0 || h->weight_stride >= 1 << 23 || logits_stride < h->vocab) return PRE3_E_BADARG;
    if (h->rows == 0) return PRE3_OK;
    const uintptr_t size = bytes_of(h->type);
    if (!h->hidden || !h->weight || !h->weight_scale || !logits || !is_aligned(h->hidden, size) || !is_aligned(logits, size) || !is_aligned(h->weight, 16) ||
        !is_aligned(h->weight_scale, 4) || !is_aligned(h->bitmask, 4) || !holds(h->workspace, h->workspace_bytes, head8_workspace_bytes(h->rows, h->dim), 16))
        return PRE3_E_BADARG;
    const Head8Rows rows{h->hidden, h->weight, h->weight_scale, h->bitmask, static_cast<LogitType>(h->type), h->rows, h->vocab, h->dim, h->hidden_stride, h->weight_stride};
    return status_of(launch_head8(rows, logits, logits_stride, h->workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
