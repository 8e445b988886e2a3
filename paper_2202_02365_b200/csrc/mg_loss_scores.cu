// Launches of the log probabilities' kernels.
#include "mg_loss_launch.cuh"
#include "mg_loss_rows.cuh"
#include "mg_loss_wide.cuh"

namespace mgloss {

template <typename T, int NV, int LANES>
static void launch_rows(const ForwardLaunch& l, const ScoreArgs& a, cudaStream_t st) {
    const auto go = [&](auto kernel) { kernel<<<(unsigned)l.blocks, kRowThreads, 0, st>>>(a); };
    a.row_sums ? go(k_scores_rows<T, NV, LANES, false, true>) : l.whole ? go(k_scores_rows<T, NV, LANES, true, false>) : go(k_scores_rows<T, NV, LANES, false, false>);
}

template <typename T, int THREADS>
static void launch_wide(const ForwardLaunch& l, const ScoreArgs& a, cudaStream_t st) {
    if (l.whole) launch_cluster(k_scores_wide<T, THREADS, false>, kWideAhead * THREADS * 16, l, st, a, l.parts_log2);
    else launch_cluster(k_scores_wide<T, THREADS, true>, kWideAhead * THREADS * 16, l, st, a, l.parts_log2);
}

template <typename T, int MOST>
static void launch_tiny(const ForwardLaunch& l, const ScoreArgs& a, cudaStream_t st) {
    const auto go = [&](auto kernel) { kernel<<<(unsigned)l.blocks, kRowThreads, 0, st>>>(a); };
    a.row_sums ? go(k_scores_tiny<T, MOST, false, true>) : l.whole ? go(k_scores_tiny<T, MOST, true, false>) : go(k_scores_tiny<T, MOST, false, false>);
}

void launch_scores(const ForwardLaunch& l, const ScoreArgs& a, cudaStream_t st) {
    if (l.lanes == 1) MG_LOSS_BY_TYPE(l.dtype, (a.classes <= 8 ? launch_tiny<T, 8>(l, a, st) : a.classes <= 16 ? launch_tiny<T, 16>(l, a, st) : launch_tiny<T, 32>(l, a, st)));
    else if (!l.lanes) MG_LOSS_BY_TYPE(l.dtype, (l.threads == kWideThreads ? launch_wide<T, kWideThreads>(l, a, st) : l.threads == kWideLeastThreads ? launch_wide<T, kWideLeastThreads>(l, a, st) : launch_wide<T, kWideMostThreads>(l, a, st)));
    else if (l.lanes == 16) MG_LOSS_BY_TYPE(l.dtype, MG_LOSS_BY_VECTORS(l.nv, (launch_rows<T, NV, 16>(l, a, st))));
    else if (l.lanes == 8) MG_LOSS_BY_TYPE(l.dtype, MG_LOSS_BY_VECTORS(l.nv, (launch_rows<T, NV, 8>(l, a, st))));
    else MG_LOSS_BY_TYPE(l.dtype, MG_LOSS_BY_VECTORS(l.nv, (launch_rows<T, NV, 32>(l, a, st))));
}

}  // namespace mgloss
