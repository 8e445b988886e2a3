// Losses of a layer's output: log probabilities with entropy and top alternatives, distillation from a teacher's top logits, and their gradients.
#include "mg_loss_launch.cuh"
#include "mg_loss_plan.cuh"

namespace {

using namespace mgloss;

float2* row_sums_of(const mg_logits* z) { return reinterpret_cast<float2*>(z->row_sums); }

TeacherArgs teacher_args(const mg_teacher* t) { return {t->ids, t->values, t->lse, t->ids_stride, t->values_stride, t->ids_are_i64, t->dtype, t->entries}; }

// forward passes of both operators; `t`: distillation
int run_forward(mg_ctx* ctx, const mg_logits* z, const ScoreArgs& a, const mg_teacher* teacher, float* loss, cudaStream_t st) {
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const ForwardPlan p = plan_forward(z, a.top, !teacher, ctx->n_sms);
    const ForwardLaunch l{z->dtype, whole_vectors(z->x, z->stride, z->rows, z->classes, z->dtype), p.nv, p.lanes, p.parts_log2, p.threads, p.blocks};
    if (teacher) launch_distill(l, a, teacher_args(teacher), loss, st);
    else launch_scores(l, a, st);
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

int run_backward(mg_ctx* ctx, const mg_logits* z, const GradArgs& a, bool distill, cudaStream_t st) {
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    GradPlan p = plan_grad(z, distill ? a.teacher.entries : 0, ctx->n_sms);
    if (!distill && (p.flat_rows = flat_rows(z, a.d, a.d_stride, ctx->n_sms))) p.blocks = (z->rows + p.flat_rows - 1) / p.flat_rows;
    const bool same = same_phase(z->x, z->stride, a.d, a.d_stride, z->rows, z->dtype);
    const GradLaunch l{z->dtype, same, same && whole_vectors(z->x, z->stride, z->rows, z->classes, z->dtype) && whole_vectors(a.d, a.d_stride, z->rows, z->classes, z->dtype), p.lanes, p.chunks, p.piece, p.blocks, p.flat_rows};
    if (distill) launch_distill_grad(l, a, st);
    else launch_scores_grad(l, a, st);
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

}  // namespace

extern "C" int mg_log_probs(mg_ctx* ctx, const mg_logits* z, const void* labels, int labels_are_i64, int32_t top, float* log_prob, float* entropy, float* lse,
                            int32_t* top_ids, float* top_log_probs, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_log_probs(ctx, z, labels, labels_are_i64, top, log_prob, entropy, lse, top_ids, top_log_probs)) return rc;
    if (z->rows == 0) return MG_OK;
    const ScoreArgs a{z->x, z->stride, z->rows, z->classes, z->scale, z->scale * kLog2e, labels, labels_are_i64, top_ids || top_log_probs ? top : 0, log_prob, entropy, lse, top_ids, top_log_probs, row_sums_of(z)};
    return run_forward(ctx, z, a, nullptr, nullptr, (cudaStream_t)stream);
}

extern "C" int mg_log_probs_backward(mg_ctx* ctx, const mg_logits* z, const float* lse, const void* labels, int labels_are_i64, const float* d_log_prob,
                                     const float* entropy, const float* d_entropy, const float* d_lse, void* d_x, int64_t d_x_stride, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_log_probs_backward(ctx, z, lse, labels, labels_are_i64, d_log_prob, entropy, d_entropy, d_lse, d_x, d_x_stride)) return rc;
    if (z->rows == 0) return MG_OK;
    const GradArgs a{z->x, z->stride, z->rows, z->classes, z->scale, d_x, d_x_stride, lse, labels, labels_are_i64, d_log_prob, entropy, d_entropy, d_lse, {}, nullptr, row_sums_of(z)};
    return run_backward(ctx, z, a, false, (cudaStream_t)stream);
}

extern "C" int mg_distill(mg_ctx* ctx, const mg_logits* z, const mg_teacher* teacher, float* loss, float* lse, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_distill(ctx, z, teacher, loss, lse)) return rc;
    if (z->rows == 0) return MG_OK;
    const ScoreArgs a{z->x, z->stride, z->rows, z->classes, z->scale, z->scale * kLog2e, nullptr, 0, 0, nullptr, nullptr, lse, nullptr, nullptr, row_sums_of(z)};
    return run_forward(ctx, z, a, teacher, loss, (cudaStream_t)stream);
}

extern "C" int mg_distill_backward(mg_ctx* ctx, const mg_logits* z, const float* lse, const mg_teacher* teacher, const float* d_loss, void* d_x,
                                   int64_t d_x_stride, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_distill_backward(ctx, z, lse, teacher, d_loss, d_x, d_x_stride)) return rc;
    if (z->rows == 0) return MG_OK;
    const GradArgs a{z->x, z->stride, z->rows, z->classes, z->scale, d_x, d_x_stride, lse, nullptr, 0, nullptr, nullptr, nullptr, nullptr, teacher_args(teacher), d_loss, row_sums_of(z)};
    return run_backward(ctx, z, a, true, (cudaStream_t)stream);
}
