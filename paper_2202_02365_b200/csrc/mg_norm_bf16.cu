// Dropout and group norm of bf16 rows.
#include "mg_norm_launch.cuh"

namespace mgnorm {
template void launch_dropout<__nv_bfloat16>(int, const void*, int64_t, void*, int64_t, int64_t, int32_t, const DropArgs&, int, cudaStream_t);
template void launch_rows<__nv_bfloat16>(const RowLaunch&, const NormArgs&, cudaStream_t);
template void launch_tiles<__nv_bfloat16>(const TileLaunch&, const TileArgs&, cudaStream_t);
}
