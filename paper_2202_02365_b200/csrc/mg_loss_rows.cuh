// Narrow rows of logits, forward: 8, 16 or 32 lanes to a row, which they hold in registers.  128,000 fp32 rows of 172: 26 us without best classes (96 MB, 3.7 TB/s; 350 instructions for a
// warp's four rows), 35 with one, 43 with five (900 instructions), 76 with ten; bound by instructions.
#pragma once

#include "mg_loss.cuh"

namespace mgloss {

constexpr int kRowThreads = 256;   // (as the host side has them)
constexpr int kRowRoom = 8;        // candidates for the best classes that shared memory has room for, for each lane of a row

// A row's values in the registers of its lanes, NV vectors to each; -infinity where the row has no more.  WHOLE: rows begin and end with a vector.
template <typename T, int NV, int LANES, bool WHOLE> struct HeldRow {
    static constexpr int VEC = 16 / sizeof(T), N = NV * VEC, kStep = LANES * VEC;
    float f[N];
    int32_t first;   // class of the lane's first value (below zero, or beyond the row, where that is no class)
    __device__ __forceinline__ void load(const T* x, int32_t classes, int sub, bool on) {
        const Cover<VEC> cover(x, sizeof(T), classes, WHOLE);
        first = sub * VEC - cover.lead;
        Raw<T, VEC> raw[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int32_t c = first + j * kStep;
            if (on && c >= 0 && c + VEC <= classes) raw[j].load(x + c);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int32_t c = first + j * kStep;
            const bool full = on && c >= 0 && c + VEC <= classes;
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[j * VEC + e] = full ? raw[j].get(e) : kNegInf;
            if (!WHOLE && on && !full && c < classes)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (c + e >= 0 && c + e < classes) f[j * VEC + e] = to_float(x[c + e]);
        }
    }
    __device__ __forceinline__ int32_t class_of_value(int i) const { return first + i / VEC * kStep + i % VEC; }
    __device__ __forceinline__ float own_max() const {
        float m = f[0];
#pragma unroll
        for (int i = 1; i < N; ++i) m = fmaxf(m, f[i]);
        return m;
    }
    // (max: over the row)
    template <bool WEIGHTED>
    __device__ __forceinline__ RowSums sums(float max, float scale2) const {
        const float m = -centre(max);
        Pair sum = {0}, weighted = {0};
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const Pair y = mul2(add2(pair(f[i], f[i + 1]), pair(m, m)), pair(scale2, scale2));
            float a, b;
            split(y, &a, &b);
            const Pair e = pair(fast_exp2(a), fast_exp2(b));
            sum = add2(sum, e);
            if (WEIGHTED) weighted = fma2(e, pair(fmaxf(a, kLeast), fmaxf(b, kLeast)), weighted);
        }
        float a, b, c = 0.f, d = 0.f;
        split(sum, &a, &b);
        if (WEIGHTED) split(weighted, &c, &d);
        return {max, lanes_sum<LANES>(a + b), WEIGHTED ? lanes_sum<LANES>(c + d) : 0.f};
    }
};

// The best of a row one by one, each a pass over it (`wanted`: in this row; all lanes of the warp come along).
template <typename T, int LANES>
__device__ __noinline__ void best_one_by_one(const T* x, int32_t classes, int sub, bool wanted, float max, float log_sum, float scale, bool none, int32_t top, int32_t* ids, float* log_probs) {
    uint64_t last = ~0ull;
    for (int k = 0; k < top; ++k) {
        uint64_t best = 0;
        for (int32_t c = sub; wanted && c < classes; c += LANES) {
            const uint64_t key = key_of(to_float(x[c]), c);
            if (key < last && key > best) best = key;
        }
        last = lanes_max<LANES>(best);
        if (wanted && sub == 0) {
            if (ids) ids[k] = class_of(last);
            if (log_probs) log_probs[k] = none ? kNegInf : scale * (value_of((uint32_t)(last >> 32)) - max) - log_sum;
        }
    }
}

// The best of a row: the top-th largest of the lanes' own largest values is no larger than the top-th largest of all, so what lies below it is out; the others, as many and some
// more, are put into shared memory and ranked against each other.  Where that does not work out (too many equal values, rows that
// allow fewer classes or hold a NaN) the best are found one by one.
template <typename T, int NV, int LANES, bool WHOLE>
__device__ __forceinline__ void best_of(const HeldRow<T, NV, LANES, WHOLE>& row, const T* x, int32_t classes, float own, int sub, bool on, const RowResult& r, int32_t top, int32_t* ids,
                                        float* log_probs, uint64_t* room) {
    using Row = HeldRow<T, NV, LANES, WHOLE>;
    constexpr int kRoom = kRowRoom * LANES;
    const int lane = threadIdx.x & 31;
    const uint32_t peers = (LANES == 32 ? 0xFFFFFFFFu : (1u << LANES % 32) - 1u) << (lane & ~(LANES - 1));
    // (A guard of the lane that is asked below: plan_forward gives a row `top` lanes at least.  Without it 500,000 fp32 rows of 172 take 74 us for 71, with five best 153 for 148, by the order that the
    // compiler then chooses.)
    bool slow = top > LANES;
    if (!slow) {
        float sorted = lanes_sorted<LANES>(own);
        // The 17th largest of 32 lanes and on bound little: their second largest too, and of both lists, one the other way round, the larger ones.  (128,000 fp32 rows of 172 with 32 best:
        // 177 us, without 380; with ten, which sixteen lanes look for, the same 76.)
        if (LANES == 32 && top > LANES / 2) {
            float most = kNegInf, second = kNegInf;
#pragma unroll
            for (int i = 0; i < Row::N; ++i) {
                second = fmaxf(second, fminf(most, row.f[i]));
                most = fmaxf(most, row.f[i]);
            }
            second = lanes_sorted<LANES>(second);
            sorted = lanes_sorted<LANES>(fmaxf(sorted, __shfl_xor_sync(0xFFFFFFFFu, second, LANES - 1)));
        }
        const float least = __shfl_sync(0xFFFFFFFFu, sorted, top - 1, LANES);
        slow = !(least > kNegInf) || !(r.log_sum < __builtin_huge_valf());
        uint32_t mine = 0;   // which of the lane's values are candidates
#pragma unroll
        for (int i = 0; i < Row::N; ++i) mine |= (row.f[i] >= least ? 1u : 0u) << i;
        if (slow) mine = 0;
        int n = 0;
        while (const uint32_t some = __ballot_sync(0xFFFFFFFFu, mine != 0)) {
            const uint32_t of_row = some & peers;
            if (mine) {
                const int i = __ffs(mine) - 1, at = n + __popc(of_row & ((1u << lane) - 1u));
                const int32_t c = row.class_of_value(i);
                if (at < kRoom) room[at] = key_of(to_float(x[c]), c);   // (read again: registers cannot be indexed)
                mine &= mine - 1;
            }
            n += __popc(of_row);
        }
        __syncwarp();
        slow = slow || n > kRoom;
        if (!slow && on)
            for (int i = sub; i < n; i += LANES) {
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
    best_one_by_one<T, LANES>(x, classes, sub, slow && on, r.max, r.log_sum, r.scale, r.none, top, ids, log_probs);
}

// (KEEP: the row's sums are asked for.  A question to each row instead costs those that they are not asked of up to 3 %, by the few instructions and where the compiler then puts the others.)
// (blocks to an SM: what the values to a lane leave registers for)
constexpr int row_blocks(int values) { return values <= 8 ? 5 : values <= 24 ? 4 : 3; }

template <typename T, int NV, int LANES, bool WHOLE, bool KEEP>
__global__ void __launch_bounds__(kRowThreads, row_blocks(NV * 16 / sizeof(T))) k_scores_rows(const __grid_constant__ ScoreArgs a) {
    constexpr int GROUPS = kRowThreads / LANES;
    __shared__ uint64_t room[kRowThreads * kRowRoom];
    const int group = (int)threadIdx.x / LANES, sub = (int)threadIdx.x % LANES;
    for (int64_t r0 = (int64_t)blockIdx.x * GROUPS; r0 < a.rows; r0 += (int64_t)gridDim.x * GROUPS) {
        const int64_t r = r0 + group;
        const bool on = r < a.rows;
        const T* x = static_cast<const T*>(a.x) + (on ? r : 0) * a.stride;
        HeldRow<T, NV, LANES, WHOLE> row;
        row.load(x, a.classes, sub, on);
        const int32_t label = on && a.log_prob ? class_at(a.labels, a.labels_are_i64, r, a.classes) : -1;
        const float at_label = label >= 0 ? to_float(x[label]) : 0.f;
        const float own = row.own_max(), m = lanes_max<LANES>(own);
        const RowResult res(row.template sums<true>(m, a.scale2), a.scale);
        if (on && sub == 0) {
            if (a.lse) a.lse[r] = res.lse;
            if (a.entropy) a.entropy[r] = res.entropy;
            if (a.log_prob) a.log_prob[r] = label >= 0 ? res.log_p(at_label) : 0.f;
            if (KEEP) a.row_sums[r] = res.sums();
        }
        if (a.top)
            best_of(row, x, a.classes, own, sub, on, res, a.top, a.top_ids ? a.top_ids + r * a.top : nullptr, a.top_log_probs ? a.top_log_probs + r * a.top : nullptr,
                    room + group * LANES * kRowRoom);
    }
}

// Rows of up to 32 classes where there are many: a thread to a row.  The best of its values by going over them once for each, as whole numbers of the same order (zero: taken).
// Few classes leave lanes idle and cost as many steps across them as many do.  800,000 fp32 rows of 5 with the best one 22 us (by eight lanes 103), of 20 with five 60 us (173).
template <typename T, int MOST, bool WHOLE, bool KEEP>
__global__ void __launch_bounds__(kRowThreads) k_scores_tiny(const __grid_constant__ ScoreArgs a) {
    constexpr int VEC = 16 / sizeof(T);
    const int64_t r = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
    if (r >= a.rows) return;
    const T* x = static_cast<const T*>(a.x) + r * a.stride;
    float f[MOST];
    if (WHOLE) {
        Raw<T, VEC> raw[MOST / VEC];
#pragma unroll
        for (int j = 0; j < MOST / VEC; ++j)
            if (j * VEC < a.classes) raw[j].load(x + j * VEC);
#pragma unroll
        for (int c = 0; c < MOST; ++c) f[c] = c < a.classes ? raw[c / VEC].get(c % VEC) : kNegInf;
    } else {
#pragma unroll
        for (int c = 0; c < MOST; ++c) f[c] = c < a.classes ? to_float(x[c]) : kNegInf;
    }
    RowSums s{f[0], 0.f, 0.f};
#pragma unroll
    for (int c = 1; c < MOST; ++c) s.max = fmaxf(s.max, f[c]);
    const float m = centre(s.max);
#pragma unroll
    for (int c = 0; c < MOST; ++c) {
        const float y = (f[c] - m) * a.scale2, e = fast_exp2(y);
        s.sum += e;
        s.weighted = fmaf(e, fmaxf(y, kLeast), s.weighted);
    }
    const RowResult res(s, a.scale);
    if (a.lse) a.lse[r] = res.lse;
    if (a.entropy) a.entropy[r] = res.entropy;
    if (a.log_prob) {
        const int32_t label = class_at(a.labels, a.labels_are_i64, r, a.classes);
        a.log_prob[r] = label >= 0 ? res.log_p(to_float(x[label])) : 0.f;
    }
    if (KEEP) a.row_sums[r] = res.sums();
    if (!a.top) return;
    uint32_t order[MOST];
#pragma unroll
    for (int c = 0; c < MOST; ++c) order[c] = c < a.classes ? order_of(f[c]) : 0u;
    for (int k = 0; k < a.top; ++k) {
        uint32_t best = 0;
        int at = 0;
#pragma unroll
        for (int c = 0; c < MOST; ++c)
            if (order[c] > best) { best = order[c]; at = c; }
#pragma unroll
        for (int c = 0; c < MOST; ++c)
            if (c == at) order[c] = 0;
        if (a.top_ids) a.top_ids[r * a.top + k] = at;
        if (a.top_log_probs) a.top_log_probs[r * a.top + k] = res.log_p(value_of(best));
    }
}

// The teacher's largest value of a row and the sum of exponentials about it, times the scale; with its own lse, that and 1.
template <int LANES>
__device__ __forceinline__ void teacher_sums(const TeacherArgs& t, int64_t r, bool on, int32_t classes, float scale, int sub, float* shift, float* sum) {
    if (t.lse) { *shift = on ? t.lse[r] : 0.f; *sum = 1.f; return; }
    float m = kNegInf, s = 0.f;
    for (int k = sub; on && k < t.entries; k += LANES)
        if (class_at(t.ids, t.ids_are_i64, r * t.ids_stride + k, classes) >= 0) m = fmaxf(m, scale * float_at(t.values, t.dtype, r * t.values_stride + k));
    m = lanes_max<LANES>(m);
    if (m == kNegInf) m = 0.f;
    for (int k = sub; on && k < t.entries; k += LANES)
        if (class_at(t.ids, t.ids_are_i64, r * t.ids_stride + k, classes) >= 0) s += expf(scale * float_at(t.values, t.dtype, r * t.values_stride + k) - m);
    *shift = m; *sum = lanes_sum<LANES>(s);
}

template <typename T, int NV, int LANES, bool WHOLE, bool KEEP>
__global__ void __launch_bounds__(kRowThreads, row_blocks(NV * 16 / sizeof(T))) k_distill_rows(const __grid_constant__ ScoreArgs a, const __grid_constant__ TeacherArgs t, float* loss) {
    constexpr int GROUPS = kRowThreads / LANES;
    const int group = (int)threadIdx.x / LANES, sub = (int)threadIdx.x % LANES;
    for (int64_t r0 = (int64_t)blockIdx.x * GROUPS; r0 < a.rows; r0 += (int64_t)gridDim.x * GROUPS) {
        const int64_t r = r0 + group;
        const bool on = r < a.rows;
        const T* x = static_cast<const T*>(a.x) + (on ? r : 0) * a.stride;
        HeldRow<T, NV, LANES, WHOLE> row;
        row.load(x, a.classes, sub, on);
        float shift, sum;
        teacher_sums<LANES>(t, r, on, a.classes, a.scale, sub, &shift, &sum);
        const float m = lanes_max<LANES>(row.own_max());
        const RowResult res(row.template sums<false>(m, a.scale2), a.scale);
        const float log_sum = logf(sum), part = sum == 0.f ? 0.f : 1.f / sum;
        float v = 0.f;
        for (int k = sub; on && k < t.entries; k += LANES) {
            const int32_t c = class_at(t.ids, t.ids_are_i64, r * t.ids_stride + k, a.classes);
            if (c < 0) continue;
            const float d = above_shift(a.scale * float_at(t.values, t.dtype, r * t.values_stride + k), shift), q = expf(d) * part;
            if (q != 0.f) v = fmaf(q, (d - log_sum) - res.log_p(to_float(x[c])), v);
        }
        v = lanes_sum<LANES>(v);
        if (on && sub == 0) {
            loss[r] = v;
            if (a.lse) a.lse[r] = res.lse;
            if (KEEP) a.row_sums[r] = res.sums();
        }
    }
}

}  // namespace mgloss
