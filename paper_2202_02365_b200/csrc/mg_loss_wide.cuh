// Wide rows of logits, forward: blocks that go along a row in segments of registers, one or a cluster of them to a row.
#pragma once

#include <cooperative_groups.h>

#include "mg_loss.cuh"

namespace mgloss {

constexpr int kWideThreads = 256, kWideWarps = kWideThreads / 32, kWideVecs = 8;
constexpr int kWideRoom = 1024, kWideTrim = 256;   // candidates for the best classes: room, and how many of them are cut down to the best again

// packed values of one type: two halves to a word, or a float
template <typename T> struct Word {
    static constexpr int N = sizeof(T) == 4 ? 1 : 2;
    static __device__ __forceinline__ uint32_t least() { return sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00FC00u : 0xFF80FF80u; }   // -infinity
    static __device__ __forceinline__ uint32_t max(uint32_t a, uint32_t b) {   // (not a NaN where there is a number)
        if constexpr (sizeof(T) == 4) return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
        else {
            uint32_t r;
            if constexpr (std::is_same<T, __half>::value) asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
            else asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
            return r;
        }
    }
    static __device__ __forceinline__ void floats(uint32_t w, float* lo, float* hi) {
        if constexpr (std::is_same<T, __half>::value) {
            const float2 f = __half22float2(reinterpret_cast<const __half2&>(w));
            *lo = f.x; *hi = f.y;
        } else {
            *lo = __uint_as_float(w << 16); *hi = __uint_as_float(w & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ float largest(uint32_t w) {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w);
        else {
            float lo, hi;
            floats(w, &lo, &hi);
            return fmaxf(lo, hi);
        }
    }
};

// One thread's part of a row's sums, as it goes along: whenever its largest value grows, what it has is scaled down.
template <bool WEIGHTED> struct Running {
    float max = kNegInf;
    Pair sum = {0}, weighted = {0};
    __device__ __forceinline__ void raise(float m, float scale2) {
        if (!(m > max)) return;
        if (max != kNegInf) {
            const float by = (max - m) * scale2, f = fast_exp2(by);
            const Pair ff = pair(f, f);
            // sum 2^(y + by) (y + by)
            if (WEIGHTED) weighted = f == 0.f ? Pair{0} : mul2(ff, fma2(sum, pair(by, by), weighted));   // (0 times infinity, where `by` is that large)
            sum = mul2(ff, sum);
        }
        max = m;
    }
    __device__ __forceinline__ void add(float a, float b, float scale2) {
        const float m = -centre(max);
        const Pair y = mul2(add2(pair(a, b), pair(m, m)), pair(scale2, scale2));
        float y0, y1;
        split(y, &y0, &y1);
        const Pair e = pair(fast_exp2(y0), fast_exp2(y1));
        sum = add2(sum, e);
        if (WEIGHTED) weighted = fma2(e, pair(fmaxf(y0, kLeast), fmaxf(y1, kLeast)), weighted);
    }
    __device__ __forceinline__ RowSums both() const {
        float a, b, c, d;
        split(sum, &a, &b);
        split(weighted, &c, &d);
        return {max, a + b, c + d};
    }
};

// sums about different largest values brought together about the larger
template <bool WEIGHTED>
__device__ __forceinline__ RowSums joined(RowSums a, RowSums b, float scale2) {
    const float m = fmaxf(a.max, b.max), by_a = (a.max - m) * scale2, by_b = (b.max - m) * scale2;
    // (a part without a class has no sum; one with a NaN alone keeps it)
    const float fa = a.max == kNegInf ? 1.f : fast_exp2(by_a), fb = b.max == kNegInf ? 1.f : fast_exp2(by_b);
    RowSums r{m, fmaf(a.sum, fa, b.sum * fb), 0.f};
    if (WEIGHTED) {
        const float wa = fa == 0.f || a.max == kNegInf ? 0.f : fa * fmaf(a.sum, by_a, a.weighted), wb = fb == 0.f || b.max == kNegInf ? 0.f : fb * fmaf(b.sum, by_b, b.weighted);
        r.weighted = wa + wb;
    }
    return r;
}

struct WideShared {
    float max[kWideWarps], sum[kWideWarps], weighted[kWideWarps], least[kWideWarps];
    float part[3];                 // of a block: what others of its cluster read
    int n;                         // candidates so far; more than there is room for: the best are found one by one
    uint64_t room[kWideRoom];
    uint64_t best[MG_MAX_TOP];
    uint64_t warp_best[kWideWarps];
};

// the `top` best of the block's candidates to sh->best, the best first (every thread; behind a barrier, and before one)
__device__ __forceinline__ void rank_candidates(WideShared* sh, int n, int32_t top) {
    for (int i = threadIdx.x; i < n; i += kWideThreads) {
        const uint64_t key = sh->room[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += sh->room[j] > key;
        if (rank < top) sh->best[rank] = key;
    }
}

// A row's part `part` of `parts`: its classes are vectors [lo, hi) of the cut, the first part's the edges too.
template <typename T, bool WEIGHTED, bool EDGES>
__device__ RowSums go_along(const T* x, int32_t classes, float scale2, int part, int parts, int32_t top, WideShared* sh) {
    constexpr int VEC = 16 / sizeof(T), WORDS = 4;
    const Cut<VEC> cut(x, sizeof(T), classes);
    const int32_t lo = (int32_t)((int64_t)cut.vecs * part / parts), hi = (int32_t)((int64_t)cut.vecs * (part + 1) / parts);
    // segments of about equal length, eight vectors to a thread at most
    const int32_t segments = max(1, (hi - lo + kWideThreads * kWideVecs - 1) / (kWideThreads * kWideVecs)), each = max(1, (hi - lo + segments - 1) / segments);
    Running<WEIGHTED> run;
    float least = kNegInf;      // what lies below is not among the best
    bool known = false;
    for (int32_t s = 0; s < segments; ++s) {
        const int32_t from = lo + s * each, to = min(from + each, hi);
        Raw<T, VEC> raw[kWideVecs];
#pragma unroll
        for (int j = 0; j < kWideVecs; ++j) {
            const int32_t v = from + j * kWideThreads + (int32_t)threadIdx.x;
            if (v < to) raw[j].load(x + cut.head + v * VEC);
            else
#pragma unroll
                for (int w = 0; w < WORDS; ++w) raw[j].w[w] = Word<T>::least();
        }
        float edge = kNegInf;
        const bool has_edge = EDGES && s == 0 && part == 0 && (int)threadIdx.x < cut.edges;
        if (has_edge) edge = to_float(x[cut.edge(threadIdx.x)]);
        uint32_t most = Word<T>::least();
#pragma unroll
        for (int j = 0; j < kWideVecs; ++j)
#pragma unroll
            for (int w = 0; w < WORDS; ++w) most = Word<T>::max(most, raw[j].w[w]);
        const float own = fmaxf(Word<T>::largest(most), edge);
        run.raise(own, scale2);
#pragma unroll
        for (int j = 0; j < kWideVecs; ++j)
#pragma unroll
            for (int w = 0; w < WORDS; w += 3 - Word<T>::N) {
                float a, b;
                if constexpr (sizeof(T) == 4) { a = __uint_as_float(raw[j].w[w]); b = __uint_as_float(raw[j].w[w + 1]); }
                else Word<T>::floats(raw[j].w[w], &a, &b);
                run.add(a, b, scale2);
            }
        if (EDGES) run.add(edge, kNegInf, scale2);
        if (top) {
            if (!known) {
                // The warps' ceil(top / warps)-th largest of their threads' largest: the least of these is no larger than the row's top-th largest value.
                // (Warps all of whose threads have a vector; none, and all values are candidates.)
                const int full = min((to - from) / 32, kWideWarps), each_warp = (top + full - 1) / max(full, 1);
                float left = own, of_warp = kNegInf;
                for (int k = 0; k < each_warp; ++k) {
                    of_warp = value_of(__reduce_max_sync(0xFFFFFFFFu, order_of(left)));
                    const uint32_t holders = __ballot_sync(0xFFFFFFFFu, left == of_warp);
                    if ((int)(threadIdx.x & 31) == __ffs(holders) - 1) left = kNegInf;
                }
                if ((threadIdx.x & 31) == 0) sh->least[threadIdx.x / 32] = of_warp;
                if (threadIdx.x == 0) sh->n = 0;
                __syncthreads();
                least = full ? sh->least[0] : kNegInf;
#pragma unroll
                for (int w = 1; w < kWideWarps; ++w)
                    if (w < full) least = fminf(least, sh->least[w]);
                known = true;
            }
            if (own >= least) {
#pragma unroll
                for (int j = 0; j < kWideVecs; ++j)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float v = raw[j].get(e);
                        const int32_t at = from + j * kWideThreads + (int32_t)threadIdx.x;
                        if (v >= least && at < to) {
                            const int i = atomicAdd(&sh->n, 1);
                            if (i < kWideRoom) sh->room[i] = key_of(v, cut.head + at * VEC + e);
                        }
                    }
                if (has_edge && edge >= least) {
                    const int i = atomicAdd(&sh->n, 1);
                    if (i < kWideRoom) sh->room[i] = key_of(edge, cut.edge(threadIdx.x));
                }
            }
            if (s + 1 < segments) {
                __syncthreads();
                const int n = sh->n;
                if (n > kWideTrim && n <= kWideRoom) {
                    rank_candidates(sh, n, top);
                    __syncthreads();
                    if ((int)threadIdx.x < top) sh->room[threadIdx.x] = sh->best[threadIdx.x];
                    if (threadIdx.x == 0) sh->n = top;
                    least = value_of((uint32_t)(sh->best[top - 1] >> 32));
                }
                __syncthreads();
            }
        }
    }
    // over the block, in an order that does not change
    RowSums r = run.both();
    for (int o = 16; o; o >>= 1) {
        const RowSums other{__shfl_xor_sync(0xFFFFFFFFu, r.max, o), __shfl_xor_sync(0xFFFFFFFFu, r.sum, o), WEIGHTED ? __shfl_xor_sync(0xFFFFFFFFu, r.weighted, o) : 0.f};
        r = joined<WEIGHTED>(r, other, scale2);
    }
    if ((threadIdx.x & 31) == 0) { sh->max[threadIdx.x / 32] = r.max; sh->sum[threadIdx.x / 32] = r.sum; sh->weighted[threadIdx.x / 32] = r.weighted; }
    __syncthreads();
    r = {sh->max[0], sh->sum[0], sh->weighted[0]};
#pragma unroll
    for (int w = 1; w < kWideWarps; ++w) r = joined<WEIGHTED>(r, {sh->max[w], sh->sum[w], sh->weighted[w]}, scale2);
    return r;
}

// The best of the part one by one, each a pass over it: where candidates overflow (more equal values than there is room for, values that rise along the row, NaN).
template <typename T>
__device__ __noinline__ void best_one_by_one(const T* x, int32_t classes, int part, int parts, int32_t top, WideShared* sh) {
    constexpr int VEC = 16 / sizeof(T);
    const Cut<VEC> cut(x, sizeof(T), classes);
    const int32_t lo = (int32_t)((int64_t)cut.vecs * part / parts), hi = (int32_t)((int64_t)cut.vecs * (part + 1) / parts);
    uint64_t last = ~0ull;
    for (int k = 0; k < top; ++k) {
        uint64_t best = 0;
        for (int32_t c = cut.head + lo * VEC + (int32_t)threadIdx.x; c < cut.head + hi * VEC; c += kWideThreads) {
            const uint64_t key = key_of(to_float(x[c]), c);
            if (key < last && key > best) best = key;
        }
        if (part == 0 && (int)threadIdx.x < cut.edges) {
            const int32_t c = cut.edge(threadIdx.x);
            const uint64_t key = key_of(to_float(x[c]), c);
            if (key < last && key > best) best = key;
        }
        best = lanes_max(best, 32);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh->warp_best[threadIdx.x / 32] = best;
        __syncthreads();
        last = sh->warp_best[0];
        for (int w = 1; w < kWideWarps; ++w) last = max(last, sh->warp_best[w]);
        if (threadIdx.x == 0) sh->best[k] = last;   // (zero where the part has fewer classes)
        if (last == 0) last = 1;
    }
    __syncthreads();
}

// the parts' sums, in rank 0's hands
template <bool WEIGHTED>
__device__ __forceinline__ RowSums over_cluster(RowSums r, int parts, float scale2, WideShared* sh) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    if (threadIdx.x == 0) { sh->part[0] = r.max; sh->part[1] = r.sum; sh->part[2] = r.weighted; }
    cluster.sync();
    if (cluster.block_rank() == 0)
        for (int p = 1; p < parts; ++p) {
            const float* from = cluster.map_shared_rank(sh->part, p);
            r = joined<WEIGHTED>(r, {from[0], from[1], from[2]}, scale2);
        }
    return r;
}

template <typename T, bool EDGES>
__global__ void __launch_bounds__(kWideThreads, 4) k_scores_wide(const __grid_constant__ ScoreArgs a, int parts) {
    namespace cg = cooperative_groups;
    __shared__ WideShared sh;
    const int64_t r = blockIdx.x / parts;
    const int part = (int)(blockIdx.x - (unsigned)(r * parts));
    const T* x = static_cast<const T*>(a.x) + r * a.stride;
    const int32_t label = threadIdx.x == 0 && part == 0 && a.log_prob ? class_at(a.labels, a.labels_are_i64, r, a.classes) : -1;
    const float at_label = label >= 0 ? to_float(x[label]) : 0.f;
    RowSums s = go_along<T, true, EDGES>(x, a.classes, a.scale2, part, parts, a.top, &sh);
    if (a.top) {
        // (behind go_along's last barrier)
        const int n = sh.n;
        if (n > kWideRoom || n < a.top || !(s.sum < __builtin_huge_valf()) || !(s.max > kNegInf)) best_one_by_one(x, a.classes, part, parts, a.top, &sh);
        else rank_candidates(&sh, n, a.top);
        __syncthreads();
    }
    if (parts > 1) s = over_cluster<true>(s, parts, a.scale2, &sh);
    if (part == 0) {
        const RowResult res(s, a.scale);
        if (threadIdx.x == 0) {
            if (a.lse) a.lse[r] = res.lse;
            if (a.entropy) a.entropy[r] = res.entropy;
            if (a.log_prob) a.log_prob[r] = label >= 0 ? res.log_p(at_label) : 0.f;
        }
        if (a.top && parts > 1) {
            cg::cluster_group cluster = cg::this_cluster();
            const int n = parts * a.top;      // (MG_MAX_TOP from each of 16 blocks: there is room)
            for (int i = threadIdx.x; i < n; i += kWideThreads) sh.room[i] = cluster.map_shared_rank(sh.best, i / a.top)[i % a.top];
            __syncthreads();
            rank_candidates(&sh, n, a.top);
            __syncthreads();
        }
        if ((int)threadIdx.x < a.top) {
            const uint64_t key = sh.best[threadIdx.x];
            if (a.top_ids) a.top_ids[r * a.top + threadIdx.x] = class_of(key);
            if (a.top_log_probs) a.top_log_probs[r * a.top + threadIdx.x] = res.log_p(value_of((uint32_t)(key >> 32)));
        }
    }
    if (parts > 1) cg::this_cluster().sync();   // (nobody leaves while its memory is read)
}

__device__ __forceinline__ float block_sum(float v, float* warps) {
    v = lanes_sum(v, 32);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x / 32] = v;
    __syncthreads();
    v = warps[0];
    for (int w = 1; w < kWideWarps; ++w) v += warps[w];
    return v;
}
__device__ __forceinline__ float block_max(float v, float* warps) {
    v = lanes_max(v, 32);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x / 32] = v;
    __syncthreads();
    v = warps[0];
    for (int w = 1; w < kWideWarps; ++w) v = fmaxf(v, warps[w]);
    return v;
}

// A block's view of a teacher's row: four entries to a thread at most (class -1: none).
constexpr int kTeacherEach = MG_MAX_TEACHER / kWideThreads;
struct TeacherRow {
    int32_t c[kTeacherEach];
    float q[kTeacherEach], log_q[kTeacherEach];
    __device__ __forceinline__ void load(const TeacherArgs& t, int64_t r, int32_t classes, float scale, float* warps) {
        float m = kNegInf;
#pragma unroll
        for (int i = 0; i < kTeacherEach; ++i) {
            const int k = threadIdx.x + i * kWideThreads;
            c[i] = k < t.entries ? class_at(t.ids, t.ids_are_i64, r * t.ids_stride + k, classes) : -1;
            log_q[i] = c[i] >= 0 ? scale * float_at(t.values, t.dtype, r * t.values_stride + k) : kNegInf;
            m = fmaxf(m, log_q[i]);
        }
        float sum = 1.f, shift;
        if (t.lse) shift = t.lse[r];
        else {
            m = block_max(m, warps);
            shift = m == kNegInf ? 0.f : m;
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < kTeacherEach; ++i)
                if (c[i] >= 0) sum += fast_exp2((log_q[i] - shift) * kLog2e);
            sum = block_sum(sum, warps);
        }
        const float log_sum = logf(sum), part = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int i = 0; i < kTeacherEach; ++i) {
            const float d = log_q[i] - shift;
            q[i] = c[i] >= 0 ? fast_exp2(d * kLog2e) * part : 0.f;
            log_q[i] = d - log_sum;
        }
    }
};

template <typename T, bool EDGES>
__global__ void __launch_bounds__(kWideThreads, 4) k_distill_wide(const __grid_constant__ ScoreArgs a, const __grid_constant__ TeacherArgs t, float* loss, int parts) {
    __shared__ WideShared sh;
    namespace cg = cooperative_groups;
    const int64_t r = blockIdx.x / parts;
    const int part = (int)(blockIdx.x - (unsigned)(r * parts));
    const T* x = static_cast<const T*>(a.x) + r * a.stride;
    RowSums s = go_along<T, false, EDGES>(x, a.classes, a.scale2, part, parts, 0, &sh);
    if (parts > 1) s = over_cluster<false>(s, parts, a.scale2, &sh);
    if (part == 0) {
        const RowResult res(s, a.scale);
        TeacherRow row;
        __syncthreads();
        row.load(t, r, a.classes, a.scale, sh.max);
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < kTeacherEach; ++i)
            if (row.q[i] != 0.f) v = fmaf(row.q[i], row.log_q[i] - res.log_p(to_float(x[row.c[i]])), v);
        v = block_sum(v, sh.max);
        if (threadIdx.x == 0) {
            loss[r] = v;
            if (a.lse) a.lse[r] = res.lse;
        }
    }
    if (parts > 1) cg::this_cluster().sync();
}

}  // namespace mgloss
