// Losses of a layer's output: log probabilities with entropy and top alternatives, distillation from a teacher's top logits, and their gradients.
#include "mg_loss_grad.cuh"
#include "mg_loss_plan.cuh"

namespace {

using namespace mgloss;

TeacherArgs teacher_args(const mg_teacher* t) { return {t->ids, t->values, t->lse, t->ids_stride, t->values_stride, t->ids_are_i64, t->dtype, t->entries}; }

int pow2_up(int64_t v) { int p = 1; while (p < v) p *= 2; return p; }

// rows that begin and end with a 16-byte vector each
bool whole_vectors(const void* p, int64_t stride, int64_t rows, int32_t classes, int dtype) {
    const int64_t vec = 16 / elem_size(dtype);
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && classes % vec == 0 && (rows <= 1 || stride % vec == 0);
}
// two matrices whose rows begin equally far from one
bool same_phase(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t rows, int dtype) {
    const int64_t vec = 16 / elem_size(dtype);
    return (reinterpret_cast<uintptr_t>(a) - reinterpret_cast<uintptr_t>(b)) % 16 == 0 && (rows <= 1 || (a_stride - b_stride) % vec == 0);
}

constexpr int kHeldValues = 32;   // of a narrow row, to a lane

// lanes to a narrow row, and values to a lane (8, 16 or 32)
struct RowShapeOf { int lanes, values; };
RowShapeOf row_shape(int32_t classes, int dtype, bool edges) {
    const int vec = 16 / elem_size(dtype), least = edges && vec == 8 ? 16 : 8;   // (an edge to a lane)
    const int64_t vecs = std::max<int64_t>(1, classes / vec);
    for (int values : {8, 16})
        for (int lanes = least; lanes <= 32; lanes *= 2)
            if (vecs * vec <= (int64_t)lanes * values && (values == 16 || lanes == least)) return {lanes, values};
    return {32, kHeldValues};
}
bool narrow(int32_t classes) { return classes <= 32 * kHeldValues; }

template <typename T, bool EDGES>
void launch_rows_of(const ScoreArgs& a, const TeacherArgs* t, float* loss, const RowShapeOf& s, int grid, cudaStream_t st) {
    constexpr int VEC = 16 / sizeof(T);
    if (t) {
        if (s.values == 8) k_distill_rows<T, 8 / VEC, EDGES><<<grid, mgloss::kRowThreads, 0, st>>>(a, *t, loss, s.lanes);
        else if (s.values == 16) k_distill_rows<T, 16 / VEC, EDGES><<<grid, mgloss::kRowThreads, 0, st>>>(a, *t, loss, s.lanes);
        else k_distill_rows<T, 32 / VEC, EDGES><<<grid, mgloss::kRowThreads, 0, st>>>(a, *t, loss, s.lanes);
    } else {
        if (s.values == 8) k_scores_rows<T, 8 / VEC, EDGES><<<grid, mgloss::kRowThreads, 0, st>>>(a, s.lanes);
        else if (s.values == 16) k_scores_rows<T, 16 / VEC, EDGES><<<grid, mgloss::kRowThreads, 0, st>>>(a, s.lanes);
        else k_scores_rows<T, 32 / VEC, EDGES><<<grid, mgloss::kRowThreads, 0, st>>>(a, s.lanes);
    }
}

template <typename K, typename... A>
void launch_cluster(K kernel, int64_t blocks, int parts, cudaStream_t st, A... args) {
    if (parts > 8) cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)parts; attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t how = {};
    how.gridDim = dim3((unsigned)blocks); how.blockDim = dim3(kWideThreads); how.stream = st;
    how.attrs = &attr; how.numAttrs = parts > 1 ? 1 : 0;
    cudaLaunchKernelEx(&how, kernel, args...);   // (an error is found by cudaGetLastError)
}

// how many blocks share a wide row: as many as there is room for on the GPU, a segment of registers to each at least
int wide_parts(int64_t rows, int32_t classes, int dtype, int n_sms) {
    const int64_t segment = (int64_t)kWideThreads * kWideVecs * 16 / elem_size(dtype) / 2;
    int parts = 1;
    while (parts < 16 && rows * parts * 2 <= 4 * n_sms && classes / (parts * 2) >= segment / 2) parts *= 2;
    return parts;
}

// both forward directions; `t`: distillation
int run_forward(mg_ctx* ctx, const mg_logits* z, const ScoreArgs& a, const TeacherArgs* t, float* loss, cudaStream_t st) {
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const bool edges = !whole_vectors(z->x, z->stride, z->rows, z->classes, z->dtype);
    if (narrow(z->classes)) {
        const RowShapeOf s = row_shape(z->classes, z->dtype, edges);
        const int groups = mgloss::kRowThreads / s.lanes;
        const int grid = (int)std::min<int64_t>((z->rows + groups - 1) / groups, mg_grid(ctx, 64));
        MG_BY_TYPE(z->dtype, (edges ? launch_rows_of<T, true>(a, t, loss, s, grid, st) : launch_rows_of<T, false>(a, t, loss, s, grid, st)));
    } else {
        const int parts = wide_parts(z->rows, z->classes, z->dtype, ctx->n_sms);
        const int64_t blocks = z->rows * parts;
        if (t) MG_BY_TYPE(z->dtype, (edges ? launch_cluster(k_distill_wide<T, true>, blocks, parts, st, a, *t, loss, parts) : launch_cluster(k_distill_wide<T, false>, blocks, parts, st, a, *t, loss, parts)));
        else MG_BY_TYPE(z->dtype, (edges ? launch_cluster(k_scores_wide<T, true>, blocks, parts, st, a, parts) : launch_cluster(k_scores_wide<T, false>, blocks, parts, st, a, parts)));
    }
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

// pieces of a row's gradient: about four to each block that the GPU holds
int grad_chunks(int64_t rows, int32_t classes, int dtype, int n_sms) {
    const int64_t vecs = classes / (16 / elem_size(dtype)), least = (int64_t)kGradThreads * kGradBatch;
    const int64_t most = std::max<int64_t>(1, vecs / least), want = (32ll * n_sms + rows - 1) / rows;
    return (int)std::min({most, std::max<int64_t>(want, vecs / (4 * least)), (int64_t)((1ll << 31) - 1) / rows});
}

}  // namespace

extern "C" int mg_log_probs(mg_ctx* ctx, const mg_logits* z, const void* labels, int labels_are_i64, int32_t top, float* log_prob, float* entropy, float* lse,
                            int32_t* top_ids, float* top_log_probs, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_log_probs(ctx, z, labels, labels_are_i64, top, log_prob, entropy, lse, top_ids, top_log_probs)) return rc;
    if (z->rows == 0) return MG_OK;
    const ScoreArgs a{z->x, z->stride, z->rows, z->classes, z->scale, z->scale * kLog2e, labels, labels_are_i64, top_ids || top_log_probs ? top : 0, log_prob, entropy, lse, top_ids, top_log_probs};
    return run_forward(ctx, z, a, nullptr, nullptr, (cudaStream_t)stream);
}

extern "C" int mg_log_probs_backward(mg_ctx* ctx, const mg_logits* z, const float* lse, const void* labels, int labels_are_i64, const float* d_log_prob,
                                     const float* entropy, const float* d_entropy, const float* d_lse, void* d_x, int64_t d_x_stride, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_log_probs_backward(ctx, z, lse, labels, labels_are_i64, d_log_prob, entropy, d_entropy, d_lse, d_x, d_x_stride)) return rc;
    if (z->rows == 0) return MG_OK;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const GradArgs a{z->x, z->stride, z->rows, z->classes, z->scale, d_x, d_x_stride, lse, labels, labels_are_i64, d_log_prob, entropy, d_entropy, d_lse, {}, nullptr};
    const bool same = same_phase(z->x, z->stride, d_x, d_x_stride, z->rows, z->dtype);
    const int vec = 16 / elem_size(z->dtype), lanes = std::min(kGradThreads, std::max(8, pow2_up((z->classes / vec + kGradBatch - 1) / kGradBatch)));
    const int chunks = lanes == kGradThreads ? grad_chunks(z->rows, z->classes, z->dtype, ctx->n_sms) : 1, groups = kGradThreads / lanes;
    const int grid = (int)std::min<int64_t>((z->rows * chunks + groups - 1) / groups, (1ll << 31) - 1);
    const cudaStream_t st = (cudaStream_t)stream;
    MG_BY_TYPE(z->dtype, (same ? k_scores_grad<T, true><<<grid, kGradThreads, 0, st>>>(a, lanes, chunks) : k_scores_grad<T, false><<<grid, kGradThreads, 0, st>>>(a, lanes, chunks)));
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

extern "C" int mg_distill(mg_ctx* ctx, const mg_logits* z, const mg_teacher* teacher, float* loss, float* lse, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_distill(ctx, z, teacher, loss, lse)) return rc;
    if (z->rows == 0) return MG_OK;
    const ScoreArgs a{z->x, z->stride, z->rows, z->classes, z->scale, z->scale * kLog2e, nullptr, 0, 0, nullptr, nullptr, lse, nullptr, nullptr};
    const TeacherArgs t = teacher_args(teacher);
    return run_forward(ctx, z, a, &t, loss, (cudaStream_t)stream);
}

extern "C" int mg_distill_backward(mg_ctx* ctx, const mg_logits* z, const float* lse, const mg_teacher* teacher, const float* d_loss, void* d_x,
                                   int64_t d_x_stride, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_distill_backward(ctx, z, lse, teacher, d_loss, d_x, d_x_stride)) return rc;
    if (z->rows == 0) return MG_OK;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const GradArgs a{z->x, z->stride, z->rows, z->classes, z->scale, d_x, d_x_stride, lse, nullptr, 0, nullptr, nullptr, nullptr, nullptr, teacher_args(teacher), d_loss};
    const bool same = same_phase(z->x, z->stride, d_x, d_x_stride, z->rows, z->dtype);
    const cudaStream_t st = (cudaStream_t)stream;
    const int vec = 16 / elem_size(z->dtype);
    const int lanes = std::max({8, pow2_up((z->classes / vec + kGradBatch - 1) / kGradBatch), pow2_up((teacher->entries + kTeacherRoom - 1) / kTeacherRoom)});
    if (lanes <= 32) {
        const int groups = kGradThreads / lanes;
        const int grid = (int)std::min<int64_t>((z->rows + groups - 1) / groups, mg_grid(ctx, 64));
        MG_BY_TYPE(z->dtype, (same ? k_distill_grad_rows<T, true><<<grid, kGradThreads, 0, st>>>(a, lanes) : k_distill_grad_rows<T, false><<<grid, kGradThreads, 0, st>>>(a, lanes)));
    } else {
        const int chunks = grad_chunks(z->rows, z->classes, z->dtype, ctx->n_sms);
        MG_BY_TYPE(z->dtype, (same ? k_distill_grad<T, true><<<(unsigned)(z->rows * chunks), kGradThreads, 0, st>>>(a, chunks) : k_distill_grad<T, false><<<(unsigned)(z->rows * chunks), kGradThreads, 0, st>>>(a, chunks)));
    }
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}
