// What a translation unit of its own launches: forward passes by operator, gradients.
#pragma once

#include "mg_loss.cuh"

namespace mgloss {

// (elements of 16-byte vectors: 4 of fp32, 8 of two bytes)
struct ForwardLaunch {
    int dtype;
    bool whole;            // rows begin and end with a vector
    int nv, lanes;         // narrow rows: vectors to a lane, lanes to a row (1: a thread each); wide ones: 0
    int parts_log2, threads;   // wide rows: blocks to a row, threads to a block
    int64_t blocks;
};
void launch_scores(const ForwardLaunch& l, const ScoreArgs& a, cudaStream_t st);
void launch_distill(const ForwardLaunch& l, const ScoreArgs& a, const TeacherArgs& t, float* loss, cudaStream_t st);

struct GradLaunch {
    int dtype;
    bool same, whole;      // logits' and gradient's vectors begin alike; rows begin and end with one
    int lanes, chunks;     // threads to a row (256: a block), pieces of it ...
    int32_t piece;         // ... of so many vectors
    int64_t blocks;
    int flat_rows;         // rows to a block that takes them as one run, 0: not so
};
void launch_scores_grad(const GradLaunch& l, const GradArgs& a, cudaStream_t st);
void launch_distill_grad(const GradLaunch& l, const GradArgs& a, cudaStream_t st);

template <typename K, typename... A>
void launch_cluster(K kernel, int ring_bytes, const ForwardLaunch& l, cudaStream_t st, const A&... args) {
    const int parts = 1 << l.parts_log2;
    if (parts > 8) cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (ring_bytes > 32 << 10) cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes);   // (beside the static, beyond 48 KB)
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)parts; attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t how = {};
    how.gridDim = dim3((unsigned)l.blocks); how.blockDim = dim3((unsigned)l.threads); how.stream = st;
    how.dynamicSmemBytes = (size_t)ring_bytes;
    how.attrs = &attr; how.numAttrs = parts > 1 ? 1 : 0;
    cudaLaunchKernelEx(&how, kernel, args...);   // (an error is found by cudaGetLastError)
}

// `call` with T, the rows' type
#define MG_LOSS_BY_TYPE(dtype, call)                                       \
    do {                                                                   \
        if ((dtype) == MG_DTYPE_F32) { using T = float; call; }            \
        else if ((dtype) == MG_DTYPE_F16) { using T = __half; call; }      \
        else { using T = __nv_bfloat16; call; }                            \
    } while (0)
// ... and with NV, the vectors to a lane that there are kernels for: 1, 2, 4, 6 or 8 of fp32, 1 to 4 of two-byte types
#define MG_LOSS_BY_VECTORS(n, call)                                                              \
    do {                                                                                         \
        constexpr bool wide = sizeof(T) == 4;                                                    \
        if ((n) <= 1) { constexpr int NV = 1; call; }                                            \
        else if ((n) <= 2) { constexpr int NV = 2; call; }                                       \
        else if (!wide && (n) <= 3) { constexpr int NV = wide ? 4 : 3; call; }                   \
        else if ((n) <= 4) { constexpr int NV = 4; call; }                                       \
        else if ((n) <= 6) { constexpr int NV = wide ? 6 : 4; call; }                            \
        else { constexpr int NV = wide ? 8 : 4; call; }                                          \
    } while (0)

}  // namespace mgloss
