// Launches of the distillation's kernels.
#include "mg_loss_launch.cuh"
#include "mg_loss_rows.cuh"
#include "mg_loss_wide.cuh"

namespace mgloss {

template <typename T, int NV, int LANES>
static void launch_rows(const ForwardLaunch& l, const ScoreArgs& a, const TeacherArgs& t, float* loss, cudaStream_t st) {
    const auto go = [&](auto kernel) { kernel<<<(unsigned)l.blocks, kRowThreads, 0, st>>>(a, t, loss); };
    a.row_sums ? go(k_distill_rows<T, NV, LANES, false, true>) : l.whole ? go(k_distill_rows<T, NV, LANES, true, false>) : go(k_distill_rows<T, NV, LANES, false, false>);
}

template <typename T, int THREADS>
static void launch_wide(const ForwardLaunch& l, const ScoreArgs& a, const TeacherArgs& t, float* loss, cudaStream_t st) {
    if (l.whole) launch_cluster(k_distill_wide<T, THREADS, false>, kWideAhead * THREADS * 16, l, st, a, t, loss, l.parts_log2);
    else launch_cluster(k_distill_wide<T, THREADS, true>, kWideAhead * THREADS * 16, l, st, a, t, loss, l.parts_log2);
}

void launch_distill(const ForwardLaunch& l, const ScoreArgs& a, const TeacherArgs& t, float* loss, cudaStream_t st) {
    if (!l.lanes) MG_LOSS_BY_TYPE(l.dtype, (l.threads == kWideThreads ? launch_wide<T, kWideThreads>(l, a, t, loss, st) : l.threads == kWideLeastThreads ? launch_wide<T, kWideLeastThreads>(l, a, t, loss, st) : launch_wide<T, kWideMostThreads>(l, a, t, loss, st)));
    else if (l.lanes == 16) MG_LOSS_BY_TYPE(l.dtype, MG_LOSS_BY_VECTORS(l.nv, (launch_rows<T, NV, 16>(l, a, t, loss, st))));
    else if (l.lanes == 8) MG_LOSS_BY_TYPE(l.dtype, MG_LOSS_BY_VECTORS(l.nv, (launch_rows<T, NV, 8>(l, a, t, loss, st))));
    else MG_LOSS_BY_TYPE(l.dtype, MG_LOSS_BY_VECTORS(l.nv, (launch_rows<T, NV, 32>(l, a, t, loss, st))));
}

}  // namespace mgloss
