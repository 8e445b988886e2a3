// Host side of the rows by id: checks of arguments, workspaces.  No CUDA calls.
#pragma once

#include <math.h>

#include <algorithm>

#include "mg_call.cuh"

namespace {

constexpr int kPlanBits = 8, kPlanBins = 1 << kPlanBits, kPlanThreads = 256, kPlanSmall = 1024;   // of the sort; ids that one block sorts

inline size_t rows_align(size_t bytes) { return (bytes + 15) / 16 * 16; }

// the first and the last byte of a matrix lie before or behind another's
inline bool lie_apart(const void* a, int64_t a_stride, int a_dtype, int64_t a_rows, const void* b, int64_t b_stride, int b_dtype, int64_t b_rows, int32_t dim) {
    if (a_rows <= 0 || b_rows <= 0) return true;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    const uintptr_t a1 = a0 + (uintptr_t)(((a_rows - 1) * a_stride + dim) * elem_size(a_dtype)), b1 = b0 + (uintptr_t)(((b_rows - 1) * b_stride + dim) * elem_size(b_dtype));
    return a1 <= b0 || b1 <= a0;
}

inline int check_ids(mg_ctx* ctx, const void* ids, int ids_are_i64, int64_t n, int64_t n_rows) {
    if (n < 0 || n >= (1ll << 31) - 1) return mg_fail(ctx, MG_ERR_ARG, "the number of ids must be in [0, 2^31 - 2]");
    if (n_rows < 0 || n_rows >= (1ll << 31) - 1) return mg_fail(ctx, MG_ERR_ARG, "the number of rows must be in [0, 2^31 - 2]");
    if (n > 0 && !ids) return mg_fail(ctx, MG_ERR_ARG, "null ids");
    if (reinterpret_cast<uintptr_t>(ids) % (ids_are_i64 ? 8 : 4)) return mg_fail(ctx, MG_ERR_ARG, "the ids are not aligned to their elements");
    return MG_OK;
}

inline int check_lookup(mg_ctx* ctx, const void* table, int64_t table_stride, int table_dtype, int64_t n_rows, int32_t dim, const void* ids, int ids_are_i64,
                        int64_t n, float scale, const void* y, int64_t y_stride, int y_dtype) {
    if (!known_dtype(table_dtype) || !known_dtype(y_dtype)) return mg_fail(ctx, MG_ERR_ARG, "unknown dtype");
    if (dim < 1 || dim > 1 << 22) return mg_fail(ctx, MG_ERR_ARG, "the width of a row must be in [1, 2^22]");
    if (!isfinite(scale)) return mg_fail(ctx, MG_ERR_ARG, "the scale must be finite");
    if (int rc = check_ids(ctx, ids, ids_are_i64, n, n_rows)) return rc;
    if (int rc = check_matrix(ctx, "the table", table, table_stride, table_dtype, n_rows, dim, false)) return rc;
    if (int rc = check_matrix(ctx, "y", y, y_stride, y_dtype, n, dim, true)) return rc;
    if (!lie_apart(table, table_stride, table_dtype, n_rows, y, y_stride, y_dtype, n, dim)) return mg_fail(ctx, MG_ERR_ARG, "the output overlaps the table");
    return MG_OK;
}

// ---- groups of equal ids -----------------------------------------------------------------

struct GroupPlan {
    int passes = 0, bits = 0;   // of so many bits each
    int per = 4;                // ids to a thread
    int64_t tiles = 0;
    size_t cleared = 0, at_states = 0, at_chain = 0, at_keys[2] = {0, 0}, at_order = 0, bytes = 0;
};
constexpr size_t kSortSharedBytes = 4 * (4 * kPlanBins + 8);

// keys are 0 .. n_rows; n_rows stands for an id that is no row
inline GroupPlan plan_groups(int64_t n, int64_t n_rows, int n_sms = 148) {
    GroupPlan p;
    if (n <= kPlanSmall) return p;   // (one block, no workspace)
    int bits = 1;
    while (bits < 31 && n_rows >> bits) ++bits;
    p.passes = (bits + kPlanBits - 1) / kPlanBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    // (all kernels of 50,000 ids 22 us with four to a thread, 23 with eight; of 150,001 38 and 35; of 543,000 75 and 55, with sixteen 58; of a million 90, 84 and 82)
    p.per = n < 100'000 ? 4 : 8;
    p.tiles = (n + kPlanThreads * p.per - 1) / (kPlanThreads * p.per);
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t was = at; at += rows_align(bytes); return was; };
    take(kSortSharedBytes);
    p.at_states = take(8 * (size_t)(p.passes * p.tiles) * kPlanBins);
    p.at_chain = take(8 * (size_t)std::max<int64_t>(p.tiles, 1));
    p.cleared = at;
    p.at_keys[0] = take(4 * (size_t)n);
    p.at_keys[1] = take(4 * (size_t)n);
    p.at_order = take(4 * (size_t)n);
    p.bytes = at;
    return p;
}

inline int check_groups(mg_ctx* ctx, const void* ids, int ids_are_i64, int64_t n, int64_t n_rows, const void* order, const void* group_of, const void* group_ids,
                        const void* starts, const void* n_groups, const void* workspace, size_t workspace_bytes) {
    if (int rc = check_ids(ctx, ids, ids_are_i64, n, n_rows)) return rc;
    if ((n > 0 && (!order || !group_of)) || (n > 0 && n_rows > 0 && !group_ids) || !starts || !n_groups) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    if (reinterpret_cast<uintptr_t>(group_ids) % (ids_are_i64 ? 8 : 4)) return mg_fail(ctx, MG_ERR_ARG, "the groups' ids are not aligned to their elements");
    for (const void* p : {order, group_of, starts, n_groups})
        if (reinterpret_cast<uintptr_t>(p) % 4) return mg_fail(ctx, MG_ERR_ARG, "order, group_of, starts and n_groups must be 4-byte aligned");
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return mg_fail(ctx, MG_ERR_ARG, "the workspace must be 16-byte aligned");
    const size_t need = plan_groups(n, n_rows, ctx->n_sms).bytes;
    if (workspace_bytes < need || (!workspace && need)) return mg_fail(ctx, MG_ERR_CAPACITY, "the workspace is smaller than mg_id_groups_workspace says");
    return MG_OK;
}

// ---- sums by group -----------------------------------------------------------------------

struct SumPlan {
    int32_t chunk = 1, chunks = 0, pitch = 0;
    size_t at_begun = 0, bytes = 0;
};

// Places to a chunk: two times the 768 threads that a multiprocessor holds are to have one, of 16 places at least, and no id is to leave more than 8,192 shares.  (Threads as for
// accesses of 16 bytes, of two-byte types where rows are wide.)
inline SumPlan plan_sums(int64_t n, int64_t n_rows, int32_t dim, int n_sms = 148) {
    SumPlan p;
    p.pitch = (dim + 7) / 8 * 8;
    if (n == 0 || n_rows == 0) return p;
    const int64_t lanes = dim >= 256 ? (dim + 255) / 256 * 32 : dim > 64 ? 32 : dim > 32 ? 16 : dim > 16 ? 8 : 4;
    const int64_t threads = (int64_t)n_sms * 1536;
    p.chunk = (int32_t)std::min<int64_t>(std::max<int64_t>({(n * lanes + threads - 1) / threads, (n + 8191) / 8192, 16}), std::max<int64_t>(n, 16));   // (no more than there are: n lanes / threads may pass 32 bits)
    p.chunks = (int32_t)((n + p.chunk - 1) / p.chunk);
    p.at_begun = rows_align(8 * (size_t)p.chunks * p.pitch);
    p.bytes = p.at_begun + rows_align(4 * (size_t)p.chunks);
    return p;
}
inline size_t sums_workspace(int64_t n, int64_t n_rows, int32_t dim, int n_sms = 148) { return plan_sums(n, n_rows, dim, n_sms).bytes; }

inline int check_sums(mg_ctx* ctx, const void* d_y, int64_t d_y_stride, int d_y_dtype, int64_t n, int64_t n_rows, int32_t dim, float scale, const void* order,
                      const void* group_of, const void* group_ids, int ids_are_i64, const void* starts, const void* n_groups, int into, const void* out, int64_t out_stride, int out_dtype,
                      const void* workspace, size_t workspace_bytes) {
    if (!known_dtype(d_y_dtype) || !known_dtype(out_dtype)) return mg_fail(ctx, MG_ERR_ARG, "unknown dtype");
    if (dim < 1 || dim > 1 << 22) return mg_fail(ctx, MG_ERR_ARG, "the width of a row must be in [1, 2^22]");
    if (!isfinite(scale)) return mg_fail(ctx, MG_ERR_ARG, "the scale must be finite");
    if (into != MG_ROWS_TABLE && into != MG_ROWS_ADD && into != MG_ROWS_COMPACT) return mg_fail(ctx, MG_ERR_ARG, "unknown place for the sums");
    if (n < 0 || n >= (1ll << 31) - 1 || n_rows < 0 || n_rows >= (1ll << 31) - 1) return mg_fail(ctx, MG_ERR_ARG, "the numbers of ids and of rows must be in [0, 2^31 - 2]");
    if ((n > 0 && (!order || !group_of)) || (n > 0 && n_rows > 0 && !group_ids) || !starts || !n_groups) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    if (reinterpret_cast<uintptr_t>(group_ids) % (ids_are_i64 ? 8 : 4)) return mg_fail(ctx, MG_ERR_ARG, "the groups' ids are not aligned to their elements");
    for (const void* p : {order, group_of, starts, n_groups})
        if (reinterpret_cast<uintptr_t>(p) % 4) return mg_fail(ctx, MG_ERR_ARG, "order, group_of, starts and n_groups must be 4-byte aligned");
    const int64_t out_rows = into == MG_ROWS_COMPACT ? std::min(n, n_rows) : n_rows;
    if (int rc = check_matrix(ctx, "d_y", d_y, d_y_stride, d_y_dtype, n, dim, false)) return rc;
    if (int rc = check_matrix(ctx, "the output", out, out_stride, out_dtype, out_rows, dim, true)) return rc;
    if (!lie_apart(d_y, d_y_stride, d_y_dtype, n, out, out_stride, out_dtype, out_rows, dim)) return mg_fail(ctx, MG_ERR_ARG, "the output overlaps d_y");
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return mg_fail(ctx, MG_ERR_ARG, "the workspace must be 16-byte aligned");
    const size_t need = sums_workspace(n, n_rows, dim, ctx->n_sms);
    if (workspace_bytes < need || (!workspace && need)) return mg_fail(ctx, MG_ERR_CAPACITY, "the workspace is smaller than mg_embedding_backward_workspace says");
    return MG_OK;
}

}  // namespace
