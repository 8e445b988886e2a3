// Launches of the losses' gradients.
#include "mg_loss_grad.cuh"
#include "mg_loss_launch.cuh"

namespace mgloss {

template <bool ABOUT>
static void scores_grad(const GradLaunch& l, const GradArgs& a, cudaStream_t st) {
    if (l.flat_rows) {
        const uint32_t reciprocal = (uint32_t)((1ull << 32) / (uint64_t)a.classes + 1);   // (values to a block times classes are below 2^32)
        const auto flat = [&](auto kernel) { kernel<<<(unsigned)l.blocks, kGradThreads, 0, st>>>(a, l.flat_rows, reciprocal); };
        MG_LOSS_BY_TYPE(l.dtype, (l.whole ? flat(k_scores_grad_flat<T, false, ABOUT>) : flat(k_scores_grad_flat<T, true, ABOUT>)));
        return;
    }
    int lanes_log2 = 0;
    while (1 << lanes_log2 < l.lanes) ++lanes_log2;
    const auto go = [&](auto kernel) { kernel<<<(unsigned)l.blocks, kGradThreads, 0, st>>>(a, lanes_log2, l.chunks, l.piece); };
    MG_LOSS_BY_TYPE(l.dtype, (l.whole ? go(k_scores_grad<T, ABOUT, true, true>) : l.same ? go(k_scores_grad<T, ABOUT, true, false>) : go(k_scores_grad<T, ABOUT, false, false>)));
}

template <typename T, int LANES, bool ABOUT>
static void distill_grad_rows(const GradLaunch& l, const GradArgs& a, cudaStream_t st) {
    const auto go = [&](auto kernel) { kernel<<<(unsigned)l.blocks, kGradThreads, 0, st>>>(a); };
    l.whole ? go(k_distill_grad_rows<T, LANES, ABOUT, true, true>) : l.same ? go(k_distill_grad_rows<T, LANES, ABOUT, true, false>) : go(k_distill_grad_rows<T, LANES, ABOUT, false, false>);
}

template <bool ABOUT>
static void distill_grad(const GradLaunch& l, const GradArgs& a, cudaStream_t st) {
    const auto block = [&](auto kernel) { kernel<<<(unsigned)l.blocks, kGradThreads, 0, st>>>(a, l.chunks, l.piece); };
    if (l.lanes == 8) MG_LOSS_BY_TYPE(l.dtype, (distill_grad_rows<T, 8, ABOUT>(l, a, st)));
    else if (l.lanes == 32) MG_LOSS_BY_TYPE(l.dtype, (distill_grad_rows<T, 32, ABOUT>(l, a, st)));
    else MG_LOSS_BY_TYPE(l.dtype, (l.whole ? block(k_distill_grad<T, ABOUT, true, true>) : l.same ? block(k_distill_grad<T, ABOUT, true, false>) : block(k_distill_grad<T, ABOUT, false, false>)));
}

void launch_scores_grad(const GradLaunch& l, const GradArgs& a, cudaStream_t st) { a.row_sums ? scores_grad<true>(l, a, st) : scores_grad<false>(l, a, st); }
void launch_distill_grad(const GradLaunch& l, const GradArgs& a, cudaStream_t st) { a.row_sums ? distill_grad<true>(l, a, st) : distill_grad<false>(l, a, st); }

}  // namespace mgloss
