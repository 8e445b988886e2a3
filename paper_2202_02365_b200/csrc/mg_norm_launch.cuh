// Launches of dropout's and group norm's kernels, by vector width.
#pragma once

#include "mg_norm_tiles.cuh"

namespace mgnorm {

template <typename T>
void launch_dropout(int vec, const void* x, int64_t x_stride, void* y, int64_t y_stride, int64_t rows, int32_t channels, const DropArgs& d, int grid, cudaStream_t st) {
    const T* from = static_cast<const T*>(x);
    T* to = static_cast<T*>(y);
    constexpr int kTwo = sizeof(T) == 2 ? 2 : 1;
    if (vec == 8) k_dropout<T, 8><<<grid, kNormThreads, 0, st>>>(from, x_stride, to, y_stride, (int32_t)rows, channels, d);
    else if (vec == 4) k_dropout_pieces<T, 4><<<grid, kNormThreads, 0, st>>>(from, x_stride, to, y_stride, (int32_t)rows, channels, d);
    else if (vec == kTwo && kTwo == 2) k_dropout_pieces<T, kTwo><<<grid, kNormThreads, 0, st>>>(from, x_stride, to, y_stride, (int32_t)rows, channels, d);
    else k_dropout_pieces<T, 1><<<grid, kNormThreads, 0, st>>>(from, x_stride, to, y_stride, (int32_t)rows, channels, d);
}

template <typename T, int VEC, int NV>
void launch_rows_of(const RowLaunch& l, const NormArgs& a, cudaStream_t st) {
    const size_t sums = 2 * sizeof(float) * (size_t)a.channels;
    const size_t params = (l.backward ? Params<VEC, NV, true>::kHeld : Params<VEC, NV, false>::kHeld) ? 0 : sums;
    if (l.backward) {
        const auto kernel = l.cut == ROW_EVEN ? k_norm_rows_backward<T, VEC, NV, ROW_EVEN> : l.cut == ROW_NARROW ? k_norm_rows_backward<T, VEC, NV, ROW_NARROW> : k_norm_rows_backward<T, VEC, NV, ROW_MASKS>;
        kernel<<<l.grid, kNormThreads, params + sums, st>>>(a, l.shape);
    } else {
        const auto kernel = l.cut == ROW_EVEN ? k_norm_rows<T, VEC, NV, ROW_EVEN> : l.cut == ROW_NARROW ? k_norm_rows<T, VEC, NV, ROW_NARROW> : k_norm_rows<T, VEC, NV, ROW_MASKS>;
        kernel<<<l.grid, kNormThreads, params, st>>>(a, l.shape);
    }
}

// (vectors per lane: the next number that there is a kernel for; lanes beyond the row's vectors do nothing)
template <typename T>
void launch_rows(const RowLaunch& l, const NormArgs& a, cudaStream_t st) {
    constexpr int kTwo = sizeof(T) == 2 ? 2 : 1;
    if (l.vec == 8) {
        if (l.nv == 1) launch_rows_of<T, 8, 1>(l, a, st);
        else if (l.nv == 2) launch_rows_of<T, 8, 2>(l, a, st);
        else launch_rows_of<T, 8, 4>(l, a, st);
    } else if (l.vec == 4) {
        if (l.nv <= 2) launch_rows_of<T, 4, 2>(l, a, st);
        else launch_rows_of<T, 4, 8>(l, a, st);
    } else if (l.vec == kTwo && kTwo == 2) {
        if (l.nv <= 4) launch_rows_of<T, kTwo, 4>(l, a, st);
        else launch_rows_of<T, kTwo, 16>(l, a, st);
    } else {
        if (l.nv <= 4) launch_rows_of<T, 1, 4>(l, a, st);
        else launch_rows_of<T, 1, 32>(l, a, st);
    }
}

// K rows in flight per thread, MINB blocks to an SM
template <typename T, int VEC>
void launch_sums(const TileLaunch& l, const TileArgs& a, cudaStream_t st) {
    const unsigned grid = (unsigned)((int64_t)a.tiles * a.sums.chunks);
    constexpr bool wide = sizeof(T) * VEC == 32;
    if (l.backward) k_norm_sums<T, VEC, true, wide ? 1 : VEC == 8 ? 2 : VEC == 1 ? 8 : 4, 3><<<grid, kNormThreads, 0, st>>>(a);
    else if constexpr (!wide) k_norm_sums<T, VEC, false, VEC == 1 ? 16 : VEC == 2 ? 8 : 4, 4><<<grid, kNormThreads, 0, st>>>(a);   // (nothing is gained by more than 16 bytes here)
}
template <typename T, int VEC>
void launch_results(const TileLaunch& l, const TileArgs& a, cudaStream_t st) {
    const unsigned grid = (unsigned)((int64_t)a.tiles * a.parts_of_tile * a.results.chunks);
    constexpr bool wide = sizeof(T) * VEC == 32;
    if (l.backward) launch_chained(dim3(grid), kNormThreads, st, k_norm_results<T, VEC, true, wide ? 1 : VEC == 1 ? 8 : VEC == 2 ? 4 : 2, 3>, a);
    else launch_chained(dim3(grid), kNormThreads, st, k_norm_results<T, VEC, false, wide ? 2 : VEC == 1 ? 16 : VEC == 2 ? 8 : 4, 4>, a);
}

template <typename T, int VEC>
void launch_block(const TileLaunch& l, const TileArgs& a, cudaStream_t st) {
    constexpr int K = sizeof(T) * VEC == 32 ? 2 : 4;
    if (l.cluster == 1) {
        if (l.backward) k_norm_block<T, VEC, true, false, K><<<l.block_grid, kNormThreads, 0, st>>>(a);
        else k_norm_block<T, VEC, false, false, K><<<l.block_grid, kNormThreads, 0, st>>>(a);
        return;
    }
    const auto kernel = l.backward ? k_norm_block<T, VEC, true, true, VEC == 8 ? 2 : 4> : k_norm_block<T, VEC, false, true, 4>;
    if (l.cluster > 8) cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)l.cluster; attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t how = {};
    how.gridDim = dim3((unsigned)l.block_grid); how.blockDim = dim3(kNormThreads); how.stream = st;
    how.attrs = &attr; how.numAttrs = 1;
    cudaLaunchKernelEx(&how, kernel, a);   // (an error is found by cudaGetLastError)
}

template <typename T, int VEC>
void launch_wide(const TileLaunch& l, const TileArgs& a, cudaStream_t st) {
    if (l.backward) k_norm_wide<T, VEC, true, VEC == 8 ? 1 : 2, kWideBlocks<VEC>><<<l.block_grid, kNormThreads, 0, st>>>(a);
    else k_norm_wide<T, VEC, false, VEC == 8 ? 2 : 4, 4><<<l.block_grid, kNormThreads, 0, st>>>(a);
}

template <typename T>
void launch_tiles(const TileLaunch& l, const TileArgs& a, cudaStream_t st) {
    constexpr int kTwo = sizeof(T) == 2 ? 2 : 1;
    if (l.block_grid && !l.cluster) {
        if (l.vec == 8) launch_wide<T, 8>(l, a, st);
        else if (l.vec == 4) launch_wide<T, 4>(l, a, st);
        else if (l.vec == kTwo && kTwo == 2) launch_wide<T, kTwo>(l, a, st);
        else launch_wide<T, 1>(l, a, st);
        return;
    }
    if (l.block_grid) {
        if (l.vec == 8) launch_block<T, 8>(l, a, st);
        else if (l.vec == 4) launch_block<T, 4>(l, a, st);
        else if (l.vec == kTwo && kTwo == 2) launch_block<T, kTwo>(l, a, st);
        else launch_block<T, 1>(l, a, st);
        return;
    }
    if (l.sums_vec == 8) launch_sums<T, 8>(l, a, st);
    else if (l.sums_vec == 4) launch_sums<T, 4>(l, a, st);
    else if (l.sums_vec == kTwo && kTwo == 2) launch_sums<T, kTwo>(l, a, st);
    else launch_sums<T, 1>(l, a, st);
    if (l.vec == 8) launch_results<T, 8>(l, a, st);
    else if (l.vec == 4) launch_results<T, 4>(l, a, st);
    else if (l.vec == kTwo && kTwo == 2) launch_results<T, kTwo>(l, a, st);
    else launch_results<T, 1>(l, a, st);
}

}  // namespace mgnorm
