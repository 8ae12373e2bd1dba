// The C ABI of libsurel, continued: the operators of a model behind walks and joined sets.  See
// include/surel.h for the contract of every entry point.
#include "../../include/surel.h"

#include <hip/hip_runtime.h>

#include <math.h>

#include "attention.h"
#include "context.h"
#include "kernels.h"
#include "loss.h"

namespace {

constexpr int64_t kMostBlocks = 0x7FFFFFFF;   // workgroups of one launch
constexpr float kLeastGradScale = 0x1p-100f;  // products of the gradients start from lse / scale, in 32 bits

bool misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// A stride between `count` rows or heads, and what the kernels get for it: one that leads nowhere may be any.
bool bad_stride(int64_t elements, int64_t count) {
    return elements < 0 || (count > 1 && (elements > SUREL_MAX_STRIDE || elements % 8 != 0));
}
uint32_t stride_bytes(int64_t elements, int64_t count) { return count > 1 ? (uint32_t)(2 * elements) : 0; }

// Checks what an attention call was given, and says it in the kernels' words.
int attention_args(const surel_ctx* ctx, const surel_attention_args* x, float least_scale, surel::AttentionArgs* a) {
    if (!x) return SUREL_E_NULL;
    if (x->type != SUREL_BF16 && x->type != SUREL_FP16) return SUREL_E_RANGE;
    if (x->n_seqs < 0 || x->n_seqs > SUREL_MAX_ROWS || x->n_q < 0 || x->n_q > SUREL_MAX_ROWS || x->n_k < 0 ||
        x->n_k > SUREL_MAX_ROWS)
        return SUREL_E_RANGE;
    if (x->dim < 8 || x->dim > SUREL_MAX_HEAD_DIM || x->dim % 8 != 0) return SUREL_E_RANGE;
    if (x->heads < 1 || x->heads > 65535 || x->kv_heads < 1 || x->heads % x->kv_heads != 0) return SUREL_E_RANGE;
    if (bad_stride(x->q_row, x->n_q) || bad_stride(x->q_head, x->heads) || bad_stride(x->k_row, x->n_k) ||
        bad_stride(x->k_head, x->kv_heads) || bad_stride(x->v_row, x->n_k) || bad_stride(x->v_head, x->kv_heads))
        return SUREL_E_RANGE;
    if (!(x->scale > 0.f) || x->scale < least_scale || !isfinite(x->scale)) return SUREL_E_RANGE;
    if (x->causal != 0 && x->causal != 1) return SUREL_E_RANGE;
    if ((x->d_bias == nullptr) != (x->d_bucket == nullptr)) return SUREL_E_NULL;
    if (x->d_bias && (x->n_buckets < 1 || x->n_buckets > 2 * SUREL_MAX_REACH + 1 || x->reach < 0 ||
                      x->reach > SUREL_MAX_REACH))
        return SUREL_E_RANGE;
    if (x->n_seqs > 0 && (!x->d_q_off || !x->d_k_off)) return SUREL_E_NULL;
    if (x->n_q > 0 && !x->d_q) return SUREL_E_NULL;
    if (x->n_k > 0 && (!x->d_k || !x->d_v)) return SUREL_E_NULL;
    if (misaligned16(x->d_q) || misaligned16(x->d_k) || misaligned16(x->d_v)) return SUREL_E_RANGE;
    if (x->n_seqs == 0 && (x->n_q > 0 || x->n_k > 0)) return SUREL_E_RANGE;
    if (!ctx) return SUREL_E_CTX;
    a->q = static_cast<const char*>(x->d_q);
    a->k = static_cast<const char*>(x->d_k);
    a->v = static_cast<const char*>(x->d_v);
    a->q_row = stride_bytes(x->q_row, x->n_q), a->q_head = stride_bytes(x->q_head, x->heads);
    a->k_row = stride_bytes(x->k_row, x->n_k), a->k_head = stride_bytes(x->k_head, x->kv_heads);
    a->v_row = stride_bytes(x->v_row, x->n_k), a->v_head = stride_bytes(x->v_head, x->kv_heads);
    a->q_off = x->d_q_off, a->k_off = x->d_k_off;
    a->n_seqs = (int32_t)x->n_seqs, a->n_q = (int32_t)x->n_q, a->n_k = (int32_t)x->n_k;
    a->heads = x->heads, a->kv_heads = x->kv_heads, a->dim = x->dim;
    a->causal = x->causal;
    a->scale = x->scale;
    a->bias = x->d_bias, a->bucket = x->d_bucket;
    a->n_buckets = x->d_bias ? x->n_buckets : 0;
    a->reach = x->d_bias ? x->reach : 0;
    a->err = ctx->d_err;
    return SUREL_OK;
}

int loss_args(const surel_ctx* ctx, int32_t type, const void* d_h, const void* d_w, const int32_t* d_labels,
              int64_t n_rows, int32_t n_classes, int32_t dim, surel::LossArgs* a) {
    if (type != SUREL_BF16 && type != SUREL_FP16) return SUREL_E_RANGE;
    if (n_rows < 0 || n_rows > SUREL_MAX_ROWS || n_classes < 1 || n_classes > SUREL_MAX_NODES) return SUREL_E_RANGE;
    if (dim < 8 || dim > SUREL_MAX_CLASS_DIM || dim % 8 != 0) return SUREL_E_RANGE;
    if (!d_w || (n_rows > 0 && (!d_h || !d_labels))) return SUREL_E_NULL;
    if (misaligned16(d_h) || misaligned16(d_w)) return SUREL_E_RANGE;
    if (!ctx) return SUREL_E_CTX;
    a->h = static_cast<const char*>(d_h);
    a->w = static_cast<const char*>(d_w);
    a->labels = d_labels;
    a->n_rows = (int32_t)n_rows;
    a->n_classes = n_classes;
    a->dim = dim;
    a->err = ctx->d_err;
    return SUREL_OK;
}

}  // namespace

extern "C" {

int surel_attention(surel_ctx* ctx, const surel_attention_args* args, void* d_out, float* d_lse) {
    surel::AttentionArgs a;
    if (int rc = attention_args(ctx, args, 0.f, &a)) return rc;
    if (a.n_q > 0 && (!d_out || !d_lse)) return SUREL_E_NULL;
    if (misaligned16(d_out)) return SUREL_E_RANGE;
    if (a.n_q == 0) return SUREL_OK;
    if (surel::attention_blocks(ctx->n_cu, a) > kMostBlocks) return SUREL_E_RANGE;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SUREL_E_HIP;
    if (int rc = grow_buffer(ctx, &ctx->d_model, &ctx->model_bytes, surel::attention_scratch_bytes(ctx->n_cu, a)))
        return rc;
    KernelSpan span(ctx, SUREL_K_ATTENTION);
    if (surel::launch_attention(ctx->stream, ctx->n_cu, a, args->type == SUREL_FP16, d_out, d_lse, ctx->d_model) !=
        hipSuccess)
        return SUREL_E_HIP;
    return SUREL_OK;
}

int surel_attention_grad(surel_ctx* ctx, const surel_attention_args* args, const void* d_dout, const void* d_out,
                         const float* d_lse, void* d_dq, void* d_dk, void* d_dv, void* d_dbias) {
    surel::AttentionArgs a;
    if (int rc = attention_args(ctx, args, kLeastGradScale, &a)) return rc;
    if (a.n_q > 0 && (!d_dout || !d_out || !d_lse || !d_dq)) return SUREL_E_NULL;
    if (a.n_k > 0 && (!d_dk || !d_dv)) return SUREL_E_NULL;
    if ((a.bias == nullptr) != (d_dbias == nullptr)) return SUREL_E_NULL;
    if (misaligned16(d_dout) || misaligned16(d_out) || misaligned16(d_dq) || misaligned16(d_dk) || misaligned16(d_dv))
        return SUREL_E_RANGE;
    if (a.n_q > 0 && a.n_k > 0 && surel::attention_grad_blocks(ctx->n_cu, a) > kMostBlocks) return SUREL_E_RANGE;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SUREL_E_HIP;
    if (a.n_q == 0 || a.n_k == 0) {   // nothing meets anything
        hipError_t rc = surel::launch_zero(ctx->stream, d_dq, (int64_t)a.n_q * a.heads * a.dim);
        if (rc == hipSuccess) rc = surel::launch_zero(ctx->stream, d_dk, (int64_t)a.n_k * a.kv_heads * a.dim);
        if (rc == hipSuccess) rc = surel::launch_zero(ctx->stream, d_dv, (int64_t)a.n_k * a.kv_heads * a.dim);
        if (rc == hipSuccess) rc = surel::launch_zero(ctx->stream, d_dbias, (int64_t)a.n_buckets * a.heads);
        return rc == hipSuccess ? SUREL_OK : SUREL_E_HIP;
    }
    if (int rc = grow_buffer(ctx, &ctx->d_model, &ctx->model_bytes, surel::attention_grad_scratch_bytes(ctx->n_cu, a, args->type == SUREL_FP16)))
        return rc;
    KernelSpan span(ctx, SUREL_K_ATTENTION_GRAD);
    if (surel::launch_attention_grad(ctx->stream, ctx->n_cu, a, args->type == SUREL_FP16, d_dout, d_out, d_lse, d_dq, d_dk, d_dv,
                                     d_dbias, ctx->d_model) != hipSuccess)
        return SUREL_E_HIP;
    return SUREL_OK;
}

int surel_softmax_loss(surel_ctx* ctx, int32_t type, const void* d_h, const void* d_w, const int32_t* d_labels,
                       int64_t n_rows, int32_t n_classes, int32_t dim, float* d_loss, float* d_lse) {
    surel::LossArgs a;
    if (int rc = loss_args(ctx, type, d_h, d_w, d_labels, n_rows, n_classes, dim, &a)) return rc;
    if (n_rows > 0 && (!d_loss || !d_lse)) return SUREL_E_NULL;
    if (n_rows == 0) return SUREL_OK;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SUREL_E_HIP;
    if (int rc = grow_buffer(ctx, &ctx->d_model, &ctx->model_bytes, surel::loss_scratch_bytes(ctx->n_cu, a))) return rc;
    KernelSpan span(ctx, SUREL_K_LOSS);
    if (surel::launch_loss(ctx->stream, ctx->n_cu, a, type == SUREL_FP16, d_loss, d_lse, ctx->d_model, ctx->d_turns) !=
        hipSuccess)
        return SUREL_E_HIP;
    return SUREL_OK;
}

int surel_softmax_loss_grad(surel_ctx* ctx, int32_t type, const float* d_dloss, const void* d_h, const void* d_w,
                            const int32_t* d_labels, const float* d_lse, int64_t n_rows, int32_t n_classes, int32_t dim,
                            void* d_dh, void* d_dw) {
    surel::LossArgs a;
    if (int rc = loss_args(ctx, type, d_h, d_w, d_labels, n_rows, n_classes, dim, &a)) return rc;
    if (!d_dw || (n_rows > 0 && (!d_dloss || !d_lse || !d_dh))) return SUREL_E_NULL;
    if (misaligned16(d_dh) || misaligned16(d_dw)) return SUREL_E_RANGE;
    DeviceGuard guard(ctx->device);
    if (!guard.ok) return SUREL_E_HIP;
    if (n_rows == 0)
        return surel::launch_zero(ctx->stream, d_dw, (int64_t)n_classes * dim) == hipSuccess ? SUREL_OK : SUREL_E_HIP;
    if (int rc = grow_buffer(ctx, &ctx->d_model, &ctx->model_bytes, surel::loss_grad_scratch_bytes(ctx->n_cu, a))) return rc;
    KernelSpan span(ctx, SUREL_K_LOSS_GRAD);
    if (surel::launch_loss_grad(ctx->stream, ctx->n_cu, a, type == SUREL_FP16, d_dloss, d_lse, d_dh, d_dw, ctx->d_model) !=
        hipSuccess)
        return SUREL_E_HIP;
    return SUREL_OK;
}

}  // extern "C"
