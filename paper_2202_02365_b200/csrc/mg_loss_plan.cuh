// Host side of the losses: checks of arguments, and how a call is cut into work.  No CUDA calls.
#pragma once

#include <math.h>

#include <algorithm>

#include "mg_call.cuh"

namespace {

inline int check_floats(mg_ctx* ctx, std::initializer_list<const void*> all) {
    for (const void* p : all)
        if (reinterpret_cast<uintptr_t>(p) % 4) return mg_fail(ctx, MG_ERR_ARG, "values by row must be 4-byte aligned");
    return MG_OK;
}

inline int check_logits(mg_ctx* ctx, const mg_logits* z) {
    if (!z) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    if (!known_dtype(z->dtype)) return mg_fail(ctx, MG_ERR_ARG, "unknown dtype");
    if (z->rows < 0 || z->rows >= 1ll << 31) return mg_fail(ctx, MG_ERR_ARG, "the number of rows must be in [0, 2^31)");
    if (z->classes < 1 || z->classes > 1 << 28) return mg_fail(ctx, MG_ERR_ARG, "the number of classes must be in [1, 2^28]");
    if (!(z->scale > 0.f) || isinf(z->scale)) return mg_fail(ctx, MG_ERR_ARG, "the scale must be positive and finite");
    if (reinterpret_cast<uintptr_t>(z->row_sums) % 8) return mg_fail(ctx, MG_ERR_ARG, "row_sums must be 8-byte aligned");
    return check_matrix(ctx, "the logits", z->x, z->stride, z->dtype, z->rows, z->classes, false);
}

inline int check_labels(mg_ctx* ctx, const void* labels, int labels_are_i64) {
    if (reinterpret_cast<uintptr_t>(labels) % (labels_are_i64 ? 8 : 4)) return mg_fail(ctx, MG_ERR_ARG, "the labels are not aligned to their elements");
    return MG_OK;
}

inline int check_gradient(mg_ctx* ctx, const mg_logits* z, const float* lse, const void* d_x, int64_t d_x_stride) {
    if (z->rows > 0 && !lse && !z->row_sums) return mg_fail(ctx, MG_ERR_ARG, "null lse");
    if (int rc = check_matrix(ctx, "d_x", d_x, d_x_stride, z->dtype, z->rows, z->classes, true)) return rc;
    return check_apart(ctx, "the logits", z->x, z->stride, d_x, d_x_stride, z->dtype, z->rows, z->classes);
}

inline int check_log_probs(mg_ctx* ctx, const mg_logits* z, const void* labels, int labels_are_i64, int32_t top, const float* log_prob, const float* entropy, const float* lse,
                           const int32_t* top_ids, const float* top_log_probs) {
    if (int rc = check_logits(ctx, z)) return rc;
    if (int rc = check_labels(ctx, labels, labels_are_i64)) return rc;
    if (z->rows > 0 && log_prob && !labels) return mg_fail(ctx, MG_ERR_ARG, "log probabilities of labels want labels");
    if (top < 0 || top > MG_MAX_TOP || top > z->classes) return mg_fail(ctx, MG_ERR_ARG, "top must be in [0, %d], and no more than there are classes", MG_MAX_TOP);
    return check_floats(ctx, {log_prob, entropy, lse, top_ids, top_log_probs});
}

inline int check_log_probs_backward(mg_ctx* ctx, const mg_logits* z, const float* lse, const void* labels, int labels_are_i64, const float* d_log_prob, const float* entropy,
                                    const float* d_entropy, const float* d_lse, const void* d_x, int64_t d_x_stride) {
    if (int rc = check_logits(ctx, z)) return rc;
    if (int rc = check_labels(ctx, labels, labels_are_i64)) return rc;
    if (z->rows > 0 && d_log_prob && !labels) return mg_fail(ctx, MG_ERR_ARG, "log probabilities of labels want labels");
    if (z->rows > 0 && d_entropy && !entropy) return mg_fail(ctx, MG_ERR_ARG, "the entropy's gradient wants the entropy");
    if (int rc = check_floats(ctx, {lse, d_log_prob, entropy, d_entropy, d_lse})) return rc;
    return check_gradient(ctx, z, lse, d_x, d_x_stride);
}

inline int check_teacher(mg_ctx* ctx, const mg_logits* z, const mg_teacher* t) {
    if (!t) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    if (!known_dtype(t->dtype)) return mg_fail(ctx, MG_ERR_ARG, "unknown dtype");
    if (t->entries < 1 || t->entries > MG_MAX_TEACHER) return mg_fail(ctx, MG_ERR_ARG, "the teacher's entries must be in [1, %d]", MG_MAX_TEACHER);
    if (int rc = check_matrix(ctx, "the teacher's values", t->values, t->values_stride, t->dtype, z->rows, t->entries, false)) return rc;
    if (z->rows > 0 && !t->ids) return mg_fail(ctx, MG_ERR_ARG, "null classes of the teacher's");
    if (reinterpret_cast<uintptr_t>(t->ids) % (t->ids_are_i64 ? 8 : 4)) return mg_fail(ctx, MG_ERR_ARG, "the teacher's classes are not aligned to their elements");
    if (z->rows > 1 && (t->ids_stride < 0 || t->ids_stride > 1ll << 28)) return mg_fail(ctx, MG_ERR_ARG, "the rows of the teacher's classes must be 0 to 2^28 elements apart");
    return check_floats(ctx, {t->lse});
}

inline int check_distill(mg_ctx* ctx, const mg_logits* z, const mg_teacher* t, const float* loss, const float* lse) {
    if (int rc = check_logits(ctx, z)) return rc;
    if (int rc = check_teacher(ctx, z, t)) return rc;
    if (z->rows > 0 && !loss) return mg_fail(ctx, MG_ERR_ARG, "null loss");
    return check_floats(ctx, {loss, lse});
}

inline int check_distill_backward(mg_ctx* ctx, const mg_logits* z, const float* lse, const mg_teacher* t, const float* d_loss, const void* d_x, int64_t d_x_stride) {
    if (int rc = check_logits(ctx, z)) return rc;
    if (int rc = check_teacher(ctx, z, t)) return rc;
    if (z->rows > 0 && !d_loss) return mg_fail(ctx, MG_ERR_ARG, "null gradient of the loss");
    if (int rc = check_floats(ctx, {lse, d_loss})) return rc;
    return check_gradient(ctx, z, lse, d_x, d_x_stride);
}

// ---- how a call is cut ------------------------------------------------------------------

// rows that begin and end with a 16-byte vector each
inline bool whole_vectors(const void* p, int64_t stride, int64_t rows, int32_t classes, int dtype) {
    const int64_t vec = 16 / elem_size(dtype);
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && classes % vec == 0 && (rows <= 1 || stride % vec == 0);
}
// two matrices whose rows begin equally far from one
inline bool same_phase(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t rows, int dtype) {
    const int64_t vec = 16 / elem_size(dtype);
    return (reinterpret_cast<uintptr_t>(a) - reinterpret_cast<uintptr_t>(b)) % 16 == 0 && (rows <= 1 || (a_stride - b_stride) % vec == 0);
}

constexpr int kPlanRowThreads = 256, kPlanHeld = 32;   // of the narrow kernels; values of a row to a lane
constexpr int kPlanWideThreads = 128, kPlanWideLeast = 64, kPlanWideMost = 1024;

struct ForwardPlan { int nv = 0, lanes = 0, parts = 1, parts_log2 = 0, threads = 0; int64_t blocks = 0; };

// Rows that 32 lanes hold in registers are narrow (however they lie to the vectors): 8, 16 or 32 lanes to a row, as few as hold it and are as many as best classes are asked for.
// Wide rows: a block of 128 threads goes along one, or of 64 where these have 16 rounds or fewer.  Both sides, 64 / 128 threads, us: 20,000 fp32 rows of 2,000 with five best 66 / 87, 30,000
// bf16 rows of 5,000 with ten 122 / 150, 10,000 fp32 rows of 8,000 89 / 75, 5,000 of 16,000 91 / 67; by 256 threads 137, -, -, 73, and 4,096 bf16 rows of 50,257 without best classes 81
// for 74.  A cluster of up to 16 blocks where rows are fewer than the GPU holds blocks (eight to a multiprocessor), 512 vectors to each at least; where all of these leave room, of
// 1,024 threads each.
// (thread_rows: there is a kernel that takes rows of up to 32 classes by a thread each.  From 256 rows to a multiprocessor on: 37,900 fp32
// rows of 20 with five best 6.5 us, by lanes 10.0; 9,500 of them 6.5 and 4.4, since a thread's chain of loads and steps is then all there is.)
inline ForwardPlan plan_forward(const mg_logits* z, int32_t top, bool thread_rows, int n_sms) {
    ForwardPlan p;
    if (thread_rows && z->classes <= 32 && z->rows >= 256ll * n_sms) {
        p.lanes = 1; p.nv = 1; p.threads = kPlanRowThreads;
        p.blocks = (z->rows + kPlanRowThreads - 1) / kPlanRowThreads;
        return p;
    }
    const int64_t vec = 16 / elem_size(z->dtype), covered = (z->classes + vec - 1 + vec - 1) / vec, held = kPlanHeld / vec;
    if (covered <= 32 * held) {
        static_assert(MG_MAX_TOP <= 32, "a lane at least to each of the best classes");
        p.lanes = 8;
        while (p.lanes < 32 && (covered > p.lanes * held || top > p.lanes)) p.lanes *= 2;
        p.nv = (int)((covered + p.lanes - 1) / p.lanes);
        p.threads = kPlanRowThreads;
        const int64_t groups = kPlanRowThreads / p.lanes;
        p.blocks = std::min<int64_t>((z->rows + groups - 1) / groups, (int64_t)n_sms * 64);
        return p;
    }
    while (p.parts < 16 && z->rows * p.parts * 2 <= 8ll * n_sms && z->classes / (p.parts * 2) >= 512 * vec) { p.parts *= 2; ++p.parts_log2; }
    p.threads = z->rows * p.parts <= n_sms && z->classes / p.parts > 4096 * vec ? kPlanWideMost : p.parts == 1 && z->classes <= 16 * kPlanWideLeast * vec ? kPlanWideLeast : kPlanWideThreads;
    p.blocks = z->rows * p.parts;
    return p;
}

constexpr int kPlanGradThreads = 256, kPlanGradBatch = 4, kPlanTeacherRoom = 8;

struct GradPlan { int lanes = 0, chunks = 1; int32_t piece = 0; int64_t blocks = 0; int flat_rows = 0; };

// Rows that lie one behind the other from a vector's beginning on, in both matrices: a block takes as many as have 2,048 vectors (8 at least, a multiple of 8, so that every block begins
// with one; 256 at most), fewer where two blocks to a multiprocessor would not come about.  Rows of up to 2,048 values of two bytes: beyond, they are taken one by one.
inline int flat_rows(const mg_logits* z, const void* d, int64_t d_stride, int n_sms) {
    const int64_t vec = 16 / elem_size(z->dtype);
    if (z->classes < vec || z->classes > 256 * vec || (z->rows > 1 && (z->stride != z->classes || d_stride != z->classes))) return 0;
    if (reinterpret_cast<uintptr_t>(z->x) % 16 || reinterpret_cast<uintptr_t>(d) % 16) return 0;
    const int64_t full = 2048 * vec / z->classes / 8 * 8, few = (z->rows + 2 * n_sms - 1) / (2 * n_sms);
    return (int)std::max<int64_t>(8, std::min<int64_t>({full, (few + 7) / 8 * 8, 256}));
}

// Gradients: threads to a row, so that each has up to eight vectors; a block goes along rows that are longer, or along a piece of one.  Of a teacher's pairs the narrow
// kernel takes eight for each lane.
inline GradPlan plan_grad(const mg_logits* z, int32_t entries, int n_sms) {
    GradPlan p;
    const int64_t vec = 16 / elem_size(z->dtype), covered = (z->classes + 2 * (vec - 1)) / vec;
    p.lanes = 4;
    while (p.lanes < kPlanGradThreads && covered > 8 * p.lanes) p.lanes *= 2;
    if (entries) p.lanes = p.lanes <= 8 && entries <= 8 * kPlanTeacherRoom ? 8 : p.lanes <= 32 && entries <= 32 * kPlanTeacherRoom ? 32 : kPlanGradThreads;
    if (p.lanes == kPlanGradThreads) {
        // pieces of four batches, or as few as give every multiprocessor 32 blocks
        const int64_t batch = (int64_t)kPlanGradThreads * kPlanGradBatch, most = std::max<int64_t>(1, covered / batch), want = (32ll * n_sms + z->rows - 1) / std::max<int64_t>(z->rows, 1);
        p.chunks = (int)std::min({most, std::max(want, covered / (4 * batch)), ((int64_t)(1ll << 31) - 1) / std::max<int64_t>(z->rows, 1)});
        p.chunks = std::max(p.chunks, 1);
        p.piece = (int32_t)((covered + p.chunks - 1) / p.chunks);
        p.blocks = z->rows * p.chunks;
    } else {
        const int64_t groups = kPlanGradThreads / p.lanes;
        p.blocks = (z->rows + groups - 1) / groups;
        if (entries) p.blocks = std::min<int64_t>(p.blocks, (int64_t)n_sms * 64);
    }
    return p;
}

}  // namespace
