// Host side of the calls that work on the caller's matrices: checks of arguments, and the device they go to.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "mg_internal.cuh"

namespace {

inline int elem_size(int dtype) { return dtype == MG_DTYPE_F32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == MG_DTYPE_F32 || dtype == MG_DTYPE_F16 || dtype == MG_DTYPE_BF16; }

// a matrix of the caller's: rows `stride` elements apart (what is only read may be one row over and over)
inline int check_matrix(mg_ctx* ctx, const char* what, const void* p, int64_t stride, int dtype, int64_t rows, int32_t channels, bool written) {
    if (rows > 0 && !p) return mg_fail(ctx, MG_ERR_ARG, "null %s", what);
    if (reinterpret_cast<uintptr_t>(p) % elem_size(dtype)) return mg_fail(ctx, MG_ERR_ARG, "%s is not aligned to its elements", what);
    if (rows > 1 && (stride < 0 || stride > 1ll << 28)) return mg_fail(ctx, MG_ERR_ARG, "the rows of %s must be 0 to 2^28 elements apart", what);
    if (rows > 1 && written && stride < channels) return mg_fail(ctx, MG_ERR_ARG, "the rows of %s overlap", what);
    return MG_OK;
}

// What is written may be one of the inputs, element for element, or lie apart from it (between its rows, say); nothing in between.
inline int check_apart(mg_ctx* ctx, const char* what, const void* in, int64_t in_stride, const void* out, int64_t out_stride, int dtype, int64_t rows, int32_t channels) {
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

struct DeviceScope {   // work goes to the context's device; the caller's current one stays
    int before = -1;
    cudaError_t err;
    explicit DeviceScope(int device) {
        err = cudaGetDevice(&before);
        if (err == cudaSuccess && before != device) err = cudaSetDevice(device);
        else if (err == cudaSuccess) before = -1;
    }
    ~DeviceScope() { if (before >= 0) cudaSetDevice(before); }
};

// `by_type<T>(...)` for the rows' type
#define MG_BY_TYPE(dtype, call)                              \
    do {                                                     \
        if ((dtype) == MG_DTYPE_F32) { using T = float; call; }          \
        else if ((dtype) == MG_DTYPE_F16) { using T = __half; call; }    \
        else { using T = __nv_bfloat16; call; }              \
    } while (0)

}  // namespace
