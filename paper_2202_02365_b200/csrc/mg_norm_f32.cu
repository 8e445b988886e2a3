// Dropout and group norm of fp32 rows.
#include "mg_norm_launch.cuh"

namespace mgnorm {
template void launch_dropout<float>(int, const void*, int64_t, void*, int64_t, int64_t, int32_t, const DropArgs&, int, cudaStream_t);
template void launch_rows<float>(const RowLaunch&, const NormArgs&, cudaStream_t);
template void launch_tiles<float>(const TileLaunch&, const TileArgs&, cudaStream_t);
}
