// Narrow rows of logits, forward: a warp or a part of one to a row, which it holds in registers.
#pragma once

#include "mg_loss.cuh"

namespace mgloss {

constexpr int kRowThreads = 256, kRowWarps = kRowThreads / 32;
constexpr int kRowRoom = 8;        // candidates for the best classes that shared memory has room for, for each lane of a row

// A row's values in the registers of its lanes: NV vectors and, where rows do not start and end with a vector, one element of the edges; -infinity where the row has
// no more.  (There are no more edges than lanes: 6 in fp32 and eight lanes, 14 in 16 bits and sixteen.)
template <typename T, int NV, bool EDGES> struct HeldRow {
    static constexpr int VEC = 16 / sizeof(T), N = NV * VEC + (EDGES ? 1 : 0);
    float f[N];
    int32_t first, step, edge;   // classes: of the lane's first vector, from one of its vectors to the next, of its edge
    int mine;                    // vectors of the lane
    bool has_edge;
    __device__ __forceinline__ void load(const T* x, int32_t classes, int sub, int lanes, bool on) {
        const Cut<VEC> cut(x, sizeof(T), classes);
        first = cut.head + sub * VEC; step = lanes * VEC;
        mine = on && sub < cut.vecs ? (cut.vecs - sub + lanes - 1) / lanes : 0;
        Raw<T, VEC> raw[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (j < mine) raw[j].load(x + first + j * step);
        float last = kNegInf;
        edge = 0;
        has_edge = EDGES && on && sub < cut.edges;
        if (has_edge) {
            edge = cut.edge(sub);
            last = to_float(x[edge]);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[j * VEC + e] = j < mine ? raw[j].get(e) : kNegInf;
        if (EDGES) f[N - 1] = last;
    }
    __device__ __forceinline__ bool held(int i) const { return EDGES && i == N - 1 ? has_edge : i / VEC < mine; }
    __device__ __forceinline__ int32_t class_of_value(int i) const { return EDGES && i == N - 1 ? edge : first + i / VEC * step + i % VEC; }
    __device__ __forceinline__ float own_max() const {
        float m = f[0];
#pragma unroll
        for (int i = 1; i < N; ++i) m = fmaxf(m, f[i]);
        return m;
    }
    // (max: over the row)
    template <bool WEIGHTED>
    __device__ __forceinline__ RowSums sums(float max, float scale2, int lanes) const {
        RowSums s{max, 0.f, 0.f};
        const float m = centre(max);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = (f[i] - m) * scale2, e = fast_exp2(y);
            s.sum += e;
            if (WEIGHTED) s.weighted = fmaf(e, fmaxf(y, kLeast), s.weighted);
        }
        s.sum = lanes_sum(s.sum, lanes);
        if (WEIGHTED) s.weighted = lanes_sum(s.weighted, lanes);
        return s;
    }
    // the row's best below `last`
    __device__ __forceinline__ uint64_t best_below(uint64_t last, int lanes) const {
        uint64_t best = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t key = key_of(f[i], class_of_value(i));
            if (held(i) && key < last && key > best) best = key;
        }
        return lanes_max(best, lanes);
    }
};

// The best of a row: the top-th largest of the lanes' own largest values is no larger than the top-th largest of all, so what lies below it is out; the others, as many and some
// more, are put into shared memory and ranked against each other.  Where that does not work out (fewer lanes than `top`, too many equal values, rows that
// allow fewer classes or hold a NaN) the best are found one by one.
template <typename T, int NV, bool EDGES>
__device__ __forceinline__ void best_of(const HeldRow<T, NV, EDGES>& row, float own, int sub, int lanes, bool on, const RowResult& r, int32_t top, int32_t* ids, float* log_probs,
                                        uint64_t* room, int* count) {
    const int lane = threadIdx.x & 31;
    const uint32_t peers = (lanes == 32 ? 0xFFFFFFFFu : (1u << lanes) - 1u) << (lane & ~(lanes - 1));
    bool slow = top > lanes;
    float left = own, least = kNegInf;
    if (!__all_sync(0xFFFFFFFFu, slow)) {
        for (int k = 0; k < top; ++k) {
            least = lanes_max(left, lanes);
            const uint32_t holders = __ballot_sync(0xFFFFFFFFu, left == least) & peers;
            if (lane == __ffs(holders) - 1) left = kNegInf;
        }
        slow = !(least > kNegInf) || !(r.log_sum < __builtin_huge_valf());
        if (sub == 0) *count = 0;
        __syncwarp();
        if (!slow && own >= least) {
#pragma unroll
            for (int i = 0; i < HeldRow<T, NV, EDGES>::N; ++i)
                if (row.f[i] >= least) {
                    const int at = atomicAdd(count, 1);
                    if (at < kRowRoom * lanes) room[at] = key_of(row.f[i], row.class_of_value(i));
                }
        }
        __syncwarp();
        const int n = *count;
        slow = slow || n > kRowRoom * lanes;
        if (!slow && on)
            for (int i = sub; i < n; i += lanes) {
                const uint64_t key = room[i];
                int rank = 0;
                for (int j = 0; j < n; ++j) rank += room[j] > key;
                if (rank < top) {
                    if (ids) ids[rank] = class_of(key);
                    if (log_probs) log_probs[rank] = r.log_p(value_of((uint32_t)(key >> 32)));
                }
            }
        __syncwarp();
    }
    if (!__any_sync(0xFFFFFFFFu, slow && on)) return;
    uint64_t last = ~0ull;
    for (int k = 0; k < top; ++k) {
        last = row.best_below(last, lanes);
        if (slow && on && sub == 0) {
            if (ids) ids[k] = class_of(last);
            if (log_probs) log_probs[k] = r.log_p(value_of((uint32_t)(last >> 32)));
        }
    }
}

template <typename T, int NV, bool EDGES>
__global__ void __launch_bounds__(kRowThreads) k_scores_rows(const __grid_constant__ ScoreArgs a, int lanes) {
    __shared__ uint64_t room[kRowThreads * kRowRoom];
    __shared__ int count[kRowThreads / 8];
    const int group = (int)threadIdx.x / lanes, sub = (int)threadIdx.x & (lanes - 1), groups = kRowThreads / lanes;
    for (int64_t r0 = (int64_t)blockIdx.x * groups; r0 < a.rows; r0 += (int64_t)gridDim.x * groups) {
        const int64_t r = r0 + group;
        const bool on = r < a.rows;
        const T* x = static_cast<const T*>(a.x) + (on ? r : 0) * a.stride;
        HeldRow<T, NV, EDGES> row;
        row.load(x, a.classes, sub, lanes, on);
        const int32_t label = on && a.log_prob ? class_at(a.labels, a.labels_are_i64, r, a.classes) : -1;
        const float at_label = label >= 0 ? to_float(x[label]) : 0.f;
        const float own = row.own_max(), m = lanes_max(own, lanes);
        const RowResult res(row.template sums<true>(m, a.scale2, lanes), a.scale);
        if (on && sub == 0) {
            if (a.lse) a.lse[r] = res.lse;
            if (a.entropy) a.entropy[r] = res.entropy;
            if (a.log_prob) a.log_prob[r] = label >= 0 ? res.log_p(at_label) : 0.f;
        }
        if (a.top)
            best_of(row, own, sub, lanes, on, res, a.top, a.top_ids ? a.top_ids + r * a.top : nullptr, a.top_log_probs ? a.top_log_probs + r * a.top : nullptr,
                    room + group * lanes * kRowRoom, count + group);
    }
}

// The teacher's largest value of a row and the sum of exponentials about it, times the scale; with its own lse, that and 1.
__device__ __forceinline__ void teacher_sums(const TeacherArgs& t, int64_t r, bool on, int32_t classes, float scale, int sub, int lanes, float* shift, float* sum) {
    if (t.lse) { *shift = on ? t.lse[r] : 0.f; *sum = 1.f; return; }
    float m = kNegInf, s = 0.f;
    for (int k = sub; on && k < t.entries; k += lanes)
        if (class_at(t.ids, t.ids_are_i64, r * t.ids_stride + k, classes) >= 0) m = fmaxf(m, scale * float_at(t.values, t.dtype, r * t.values_stride + k));
    m = lanes_max(m, lanes);
    if (m == kNegInf) m = 0.f;
    for (int k = sub; on && k < t.entries; k += lanes)
        if (class_at(t.ids, t.ids_are_i64, r * t.ids_stride + k, classes) >= 0) s += fast_exp2((scale * float_at(t.values, t.dtype, r * t.values_stride + k) - m) * kLog2e);
    *shift = m; *sum = lanes_sum(s, lanes);
}

template <typename T, int NV, bool EDGES>
__global__ void __launch_bounds__(kRowThreads) k_distill_rows(const __grid_constant__ ScoreArgs a, const __grid_constant__ TeacherArgs t, float* loss, int lanes) {
    const int group = (int)threadIdx.x / lanes, sub = (int)threadIdx.x & (lanes - 1), groups = kRowThreads / lanes;
    for (int64_t r0 = (int64_t)blockIdx.x * groups; r0 < a.rows; r0 += (int64_t)gridDim.x * groups) {
        const int64_t r = r0 + group;
        const bool on = r < a.rows;
        const T* x = static_cast<const T*>(a.x) + (on ? r : 0) * a.stride;
        HeldRow<T, NV, EDGES> row;
        row.load(x, a.classes, sub, lanes, on);
        float shift, sum;
        teacher_sums(t, r, on, a.classes, a.scale, sub, lanes, &shift, &sum);
        const float m = lanes_max(row.own_max(), lanes);
        const RowResult res(row.template sums<false>(m, a.scale2, lanes), a.scale);
        const float log_sum = logf(sum), part = sum == 0.f ? 0.f : 1.f / sum;
        float v = 0.f;
        for (int k = sub; on && k < t.entries; k += lanes) {
            const int32_t c = class_at(t.ids, t.ids_are_i64, r * t.ids_stride + k, a.classes);
            if (c < 0) continue;
            const float d = a.scale * float_at(t.values, t.dtype, r * t.values_stride + k) - shift, q = fast_exp2(d * kLog2e) * part;
            if (q != 0.f) v = fmaf(q, (d - log_sum) - res.log_p(to_float(x[c])), v);
        }
        v = lanes_sum(v, lanes);
        if (on && sub == 0) {
            loss[r] = v;
            if (a.lse) a.lse[r] = res.lse;
        }
    }
}

}  // namespace mgloss
