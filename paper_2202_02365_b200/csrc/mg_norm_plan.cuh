// Host side of dropout and of group norm: checks of arguments, and how a call is cut into work.  No CUDA calls.
#pragma once

#include <math.h>

#include <algorithm>

#include "mg_internal.cuh"
#include "mg_norm.cuh"

namespace {

int elem_size(int dtype) { return dtype == MG_DTYPE_F32 ? 4 : 2; }

int check_dropout(mg_ctx* ctx, const mg_dropout_spec* s, DropArgs* d) {
    *d = DropArgs();
    if (!s) return MG_OK;
    if (!(s->p >= 0.0 && s->p <= 1.0)) return mg_fail(ctx, MG_ERR_ARG, "the share to drop must be in [0, 1]");
    if (s->site > 0xFFFFu) return mg_fail(ctx, MG_ERR_ARG, "a dropout's site must be below 65536");
    if (reinterpret_cast<uintptr_t>(s->row_keys) % 8) return mg_fail(ctx, MG_ERR_ARG, "row keys must be 8-byte aligned");
    d->limit = (uint32_t)nearbyint(s->p * 65536.0);
    d->on = d->limit > 0;
    d->factor = d->limit < 65536u ? 65536.f / (float)(65536u - d->limit) : 0.f;
    d->k0 = (uint32_t)s->seed; d->k1 = (uint32_t)(s->seed >> 32);
    d->tag = kDropTag + s->site;
    d->first_row = s->first_row; d->keys = s->row_keys;
    return MG_OK;
}

// a matrix of the caller's: rows `stride` elements apart (what is only read may be one row over and over)
int check_matrix(mg_ctx* ctx, const char* what, const void* p, int64_t stride, int dtype, int64_t rows, int32_t channels, bool written) {
    if (rows > 0 && !p) return mg_fail(ctx, MG_ERR_ARG, "null %s", what);
    if (reinterpret_cast<uintptr_t>(p) % elem_size(dtype)) return mg_fail(ctx, MG_ERR_ARG, "%s is not aligned to its elements", what);
    if (rows > 1 && (stride < 0 || stride > 1ll << 28)) return mg_fail(ctx, MG_ERR_ARG, "the rows of %s must be 0 to 2^28 elements apart", what);
    if (rows > 1 && written && stride < channels) return mg_fail(ctx, MG_ERR_ARG, "the rows of %s overlap", what);
    return MG_OK;
}

// What is written may be one of the inputs, element for element, or lie apart from it (between its rows, say); nothing in between.
int check_apart(mg_ctx* ctx, const char* what, const void* in, int64_t in_stride, const void* out, int64_t out_stride, int dtype, int64_t rows, int32_t channels) {
    const int64_t e = elem_size(dtype);
    const uintptr_t i0 = reinterpret_cast<uintptr_t>(in), o0 = reinterpret_cast<uintptr_t>(out);
    const uintptr_t i1 = i0 + (uintptr_t)(((rows - 1) * in_stride + channels) * e), o1 = o0 + (uintptr_t)(((rows - 1) * out_stride + channels) * e);
    if (rows <= 0 || i1 <= o0 || o1 <= i0 || (i0 == o0 && (in_stride == out_stride || rows == 1))) return MG_OK;
    if (in_stride == out_stride && rows > 1) {
        const int64_t step = in_stride * e, between = ((int64_t)(o0 - i0) % step + step) % step;
        if (between >= channels * e && between <= step - channels * e) return MG_OK;
    }
    return mg_fail(ctx, MG_ERR_ARG, "the output overlaps %s without being the same matrix", what);
}

int check_rows(mg_ctx* ctx, int dtype, int64_t rows, int32_t channels) {
    if (dtype != MG_DTYPE_F32 && dtype != MG_DTYPE_F16 && dtype != MG_DTYPE_BF16) return mg_fail(ctx, MG_ERR_ARG, "unknown dtype");
    if (rows < 0 || rows >= 1ll << 31) return mg_fail(ctx, MG_ERR_ARG, "the number of rows must be in [0, 2^31)");
    if (channels < 1 || channels > 1 << 24) return mg_fail(ctx, MG_ERR_ARG, "the number of channels must be in [1, 2^24]");
    return MG_OK;
}

int check_norm(mg_ctx* ctx, const mg_norm_spec* s) {
    if (!s) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    if (int rc = check_rows(ctx, s->dtype, s->rows, s->channels)) return rc;
    if (s->groups < 1 || s->channels % s->groups) return mg_fail(ctx, MG_ERR_ARG, "the groups must divide the channels");
    if (s->activation < MG_ACT_NONE || s->activation > MG_ACT_GELU) return mg_fail(ctx, MG_ERR_ARG, "unknown activation");
    if (!(s->eps > 0.f) || isinf(s->eps)) return mg_fail(ctx, MG_ERR_ARG, "eps must be positive and finite");
    if (s->sample_offsets) {
        if (s->n_samples < 1 || s->n_samples > MG_MAX_BATCHES) return mg_fail(ctx, MG_ERR_ARG, "the number of samples must be in [1, %d]", MG_MAX_BATCHES);
        if (s->sample_offsets[0] != 0) return mg_fail(ctx, MG_ERR_ARG, "the first sample starts at row 0");
        for (int32_t i = 0; i < s->n_samples; ++i)
            if (s->sample_offsets[i + 1] < s->sample_offsets[i]) return mg_fail(ctx, MG_ERR_ARG, "the samples' offsets must not decrease");
        if (s->sample_offsets[s->n_samples] > s->rows) return mg_fail(ctx, MG_ERR_ARG, "the samples end behind the last row");
    } else if (s->rows_per_sample < 1 || s->rows % s->rows_per_sample) {
        return mg_fail(ctx, MG_ERR_ARG, "the rows must be a multiple of rows_per_sample, which must be positive");
    }
    return MG_OK;
}

int64_t sample_count(const mg_norm_spec* s) { return s->sample_offsets ? s->n_samples : s->rows / s->rows_per_sample; }

size_t norm_workspace(const mg_norm_spec* s) { return s->sample_offsets ? sizeof(int64_t) * (size_t)(s->n_samples + 1) : 0; }


struct Matrix { const char* what; const void* p; int64_t stride; bool written; };

// the output (the last of the matrices) may be one of the inputs
int check_matrices(mg_ctx* ctx, const Matrix* m, int n, int dtype, int64_t rows, int32_t channels) {
    for (int i = 0; i < n; ++i)
        if (int rc = check_matrix(ctx, m[i].what, m[i].p, m[i].stride, dtype, rows, channels, m[i].written)) return rc;
    for (int i = 0; i + 1 < n; ++i)
        if (int rc = check_apart(ctx, m[i].what, m[i].p, m[i].stride, m[n - 1].p, m[n - 1].stride, dtype, rows, channels)) return rc;
    return MG_OK;
}

// every check of an entry point's arguments but the workspace's; `d`: the dropout as the kernels take it
int check_dropout_call(mg_ctx* ctx, const void* x, int64_t x_stride, const void* y, int64_t y_stride, int dtype, int64_t rows, int32_t channels,
                       const mg_dropout_spec* spec, DropArgs* d) {
    if (!spec) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    if (int rc = check_rows(ctx, dtype, rows, channels)) return rc;
    if (int rc = check_dropout(ctx, spec, d)) return rc;
    const Matrix m[2] = {{"x", x, x_stride, false}, {"y", y, y_stride, true}};
    return check_matrices(ctx, m, 2, dtype, rows, channels);
}

int check_norm_call(mg_ctx* ctx, const mg_norm_spec* s, const void* x, int64_t x_stride, const void* d_y, int64_t d_y_stride, bool backward,
                    const void* out, int64_t out_stride, const float* mean, const float* rstd, const void* workspace, DropArgs* d) {
    if (int rc = check_norm(ctx, s)) return rc;
    if (int rc = check_dropout(ctx, s->dropout, d)) return rc;
    const Matrix fwd[2] = {{"x", x, x_stride, false}, {"y", out, out_stride, true}};
    const Matrix bwd[3] = {{"x", x, x_stride, false}, {"d_y", d_y, d_y_stride, false}, {"d_x", out, out_stride, true}};
    if (int rc = check_matrices(ctx, backward ? bwd : fwd, backward ? 3 : 2, s->dtype, s->rows, s->channels)) return rc;
    if (sample_count(s) > 0 && (!mean || !rstd)) return mg_fail(ctx, MG_ERR_ARG, "null statistics");
    for (const void* p : {(const void*)mean, (const void*)rstd, (const void*)s->weight, (const void*)s->bias})
        if (reinterpret_cast<uintptr_t>(p) % 4) return mg_fail(ctx, MG_ERR_ARG, "statistics, weight and bias must be 4-byte aligned");
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return mg_fail(ctx, MG_ERR_ARG, "the workspace must be 16-byte aligned");
    return MG_OK;
}

}  // namespace
