// Gradients with respect to logits: rows, or pieces of rows, from the logits and a few values by row; each value is read and written once.
#pragma once

#include "mg_loss_rows.cuh"
#include "mg_loss_wide.cuh"

namespace mgloss {

constexpr int kGradThreads = 256, kGradBatch = 4;   // vectors of a thread that are on their way at once

// what a row's gradient is made of: p (base + slope log p), and `more` at the label
struct RowGrad { float scale, minus_lse, base, slope, more; int32_t label; };

// the gradients of the classes c .. c + N - 1, in place of their logits
template <bool LABELS, int N>
__device__ __forceinline__ void grads(const RowGrad& g, float (&v)[N], int32_t c) {
    if constexpr (N == 1) {
        const float log_p = fmaf(v[0], g.scale, g.minus_lse);
        v[0] = fast_exp2(log_p * kLog2e) * (LABELS ? fmaf(fmaxf(log_p, kLeast), g.slope, g.base) : g.base);
    } else {
        const Pair scale = pair(g.scale, g.scale), lse = pair(g.minus_lse, g.minus_lse), base = pair(g.base, g.base), slope = pair(g.slope, g.slope), log2e = pair(kLog2e, kLog2e);
        const bool sloped = LABELS && g.slope != 0.f;
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const Pair log_p = fma2(pair(v[i], v[i + 1]), scale, lse), y = mul2(log_p, log2e);
            float a, b;
            split(y, &a, &b);
            const Pair p = pair(fast_exp2(a), fast_exp2(b));
            Pair d;
            if (sloped) {
                split(log_p, &a, &b);
                d = mul2(p, fma2(pair(fmaxf(a, kLeast), fmaxf(b, kLeast)), slope, base));
            } else d = mul2(p, base);
            split(d, &v[i], &v[i + 1]);
        }
    }
    if (LABELS && (uint32_t)(g.label - c) < (uint32_t)N) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (c + i == g.label) v[i] += g.more;
    }
}

// Vectors [lo, hi) of a row cut where the gradient's vectors begin, and with `edges` the elements before and behind all vectors; by `lanes` threads.  SAME: the logits' vectors
// begin there too; else they are read element by element.
template <bool LABELS, bool SAME, typename T>
__device__ __forceinline__ void stream_row(const RowGrad& g, bool zero, const T* x, T* d, const Cut<16 / sizeof(T)>& cut, int32_t lo, int32_t hi, bool edges, int sub, int lanes) {
    constexpr int VEC = 16 / sizeof(T);
    for (int32_t v0 = lo + sub; v0 < hi; v0 += kGradBatch * lanes) {
        Raw<T, VEC> raw[kGradBatch];
        T one[SAME ? 1 : kGradBatch * VEC];
        if (!zero) {
#pragma unroll
            for (int j = 0; j < kGradBatch; ++j)
                if (v0 + j * lanes < hi) {
                    const T* at = x + cut.head + (v0 + j * lanes) * VEC;
                    if constexpr (SAME) raw[j].load(at);
                    else
#pragma unroll
                        for (int e = 0; e < VEC; ++e) one[j * VEC + e] = at[e];
                }
        }
#pragma unroll
        for (int j = 0; j < kGradBatch; ++j)
            if (v0 + j * lanes < hi) {
                const int32_t c = cut.head + (v0 + j * lanes) * VEC;
                float f[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    if constexpr (SAME) f[e] = raw[j].get(e);
                    else f[e] = to_float(one[j * VEC + e]);
                }
                if (zero) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) f[e] = 0.f;
                } else grads<LABELS>(g, f, c);
                raw[j].put(f);
                raw[j].store(d + c);
            }
    }
    if (edges)
        for (int e = sub; e < cut.edges; e += lanes) {
            const int32_t c = cut.edge(e);
            float f[1] = {0.f};
            if (!zero) {
                f[0] = to_float(x[c]);
                grads<LABELS>(g, f, c);
            }
            Raw<T, 1> one;
            one.put(f);
            one.store(d + c);
        }
}

// `lanes` threads to a row, or to one of its `chunks` pieces
template <typename T, bool SAME>
__global__ void __launch_bounds__(kGradThreads) k_scores_grad(const __grid_constant__ GradArgs a, int lanes, int chunks) {
    const int group = (int)threadIdx.x / lanes, sub = (int)threadIdx.x & (lanes - 1), groups = kGradThreads / lanes;
    const int64_t items = a.rows * chunks;
    for (int64_t i = (int64_t)blockIdx.x * groups + group; i < items; i += (int64_t)gridDim.x * groups) {
        const int64_t r = chunks == 1 ? i : i / chunks;
        const int32_t chunk = (int32_t)(i - r * chunks);
        const T* x = static_cast<const T*>(a.x) + r * a.stride;
        T* d = static_cast<T*>(a.d) + r * a.d_stride;
        const Cut<16 / sizeof(T)> cut(d, sizeof(T), a.classes);
        const float lse = a.lse[r];
        RowGrad g;
        g.label = a.d_log_prob ? class_at(a.labels, a.labels_are_i64, r, a.classes) : -1;
        const float of_label = g.label >= 0 ? a.d_log_prob[r] : 0.f, h = a.d_entropy ? a.d_entropy[r] : 0.f, l = a.d_lse ? a.d_lse[r] : 0.f;
        const float entropy = h != 0.f ? a.entropy[r] : 0.f;
        const bool zero = (of_label == 0.f && h == 0.f && l == 0.f) || lse == kNegInf;
        g.scale = a.scale; g.minus_lse = -lse; g.base = a.scale * (l - of_label - h * entropy); g.slope = -a.scale * h; g.more = a.scale * of_label;
        stream_row<true, SAME>(g, zero, x, d, cut, (int32_t)((int64_t)cut.vecs * chunk / chunks), (int32_t)((int64_t)cut.vecs * (chunk + 1) / chunks), chunk == 0, sub, lanes);
    }
}

// Where a teacher's pairs name a class, its gradient is made apart: from the logit, which is read before anything is written (the gradient may take the logits' place),
// and written over the one that all classes get.  The first pair that names a class has the others' probabilities, in their order.
__device__ __forceinline__ bool first_of_class(const int32_t* c, const float* q, int k, int entries, float* sum) {
    const int32_t own = c[k];
    float s = 0.f;
    bool first = own >= 0;
    for (int j = 0; j < entries; ++j)
        if (c[j] == own) {
            s += q[j];
            first = first && j >= k;
        }
    *sum = s;
    return first;
}

constexpr int kTeacherRoom = 8;   // pairs that a row of the narrow kernel may have, for each of its lanes

template <typename T, bool SAME>
__global__ void __launch_bounds__(kGradThreads) k_distill_grad_rows(const __grid_constant__ GradArgs a, int lanes) {
    __shared__ int32_t all_c[kGradThreads * kTeacherRoom];
    __shared__ float all_q[kGradThreads * kTeacherRoom], all_d[kGradThreads * kTeacherRoom];
    const TeacherArgs& t = a.teacher;
    const int group = (int)threadIdx.x / lanes, sub = (int)threadIdx.x & (lanes - 1), groups = kGradThreads / lanes;
    int32_t* c = all_c + group * lanes * kTeacherRoom;
    float *q = all_q + group * lanes * kTeacherRoom, *own = all_d + group * lanes * kTeacherRoom;
    for (int64_t r0 = (int64_t)blockIdx.x * groups; r0 < a.rows; r0 += (int64_t)gridDim.x * groups) {
        const int64_t r = r0 + group;
        const bool on = r < a.rows;
        const T* x = static_cast<const T*>(a.x) + (on ? r : 0) * a.stride;
        T* d = static_cast<T*>(a.d) + (on ? r : 0) * a.d_stride;
        const float lse = on ? a.lse[r] : 0.f, d_loss = on ? a.d_loss[r] : 0.f;
        float shift, sum, mass = 0.f;
        teacher_sums(t, r, on, a.classes, a.scale, sub, lanes, &shift, &sum);
        const float part = sum == 0.f ? 0.f : 1.f / sum;
        for (int k = sub; on && k < t.entries; k += lanes) {
            c[k] = class_at(t.ids, t.ids_are_i64, r * t.ids_stride + k, a.classes);
            q[k] = c[k] >= 0 ? fast_exp2((a.scale * float_at(t.values, t.dtype, r * t.values_stride + k) - shift) * kLog2e) * part : 0.f;
            mass += q[k];
        }
        mass = lanes_sum(mass, lanes);
        const bool zero = d_loss == 0.f || mass == 0.f || lse == kNegInf;
        RowGrad g;
        g.scale = a.scale; g.minus_lse = -lse; g.base = a.scale * d_loss * mass; g.slope = g.more = 0.f; g.label = -1;
        __syncwarp();
        uint32_t first = 0;   // which of the lane's pairs are the first of their class
        for (int k = sub, i = 0; on && !zero && k < t.entries; k += lanes, ++i) {
            float of_class;
            if (first_of_class(c, q, k, t.entries, &of_class)) {
                float f[1] = {to_float(x[c[k]])};
                grads<false>(g, f, 0);
                own[k] = f[0] - a.scale * d_loss * of_class;
                first |= 1u << i;
            }
        }
        __syncwarp();
        const Cut<16 / sizeof(T)> cut(d, sizeof(T), a.classes);
        if (on) stream_row<false, SAME>(g, zero, x, d, cut, 0, cut.vecs, true, sub, lanes);
        __syncwarp();
        for (int k = sub; first; k += lanes, first >>= 1)
            if (first & 1) {
                Raw<T, 1> one;
                const float f[1] = {own[k]};
                one.put(f);
                one.store(d + c[k]);
            }
        __syncwarp();
    }
}

// a block to a row, or to one of its `chunks` pieces
template <typename T, bool SAME>
__global__ void __launch_bounds__(kGradThreads) k_distill_grad(const __grid_constant__ GradArgs a, int chunks) {
    __shared__ int32_t c[MG_MAX_TEACHER];
    __shared__ float q[MG_MAX_TEACHER], warps[kWideWarps];
    constexpr int VEC = 16 / sizeof(T);
    const TeacherArgs& t = a.teacher;
    const int64_t r = blockIdx.x / (unsigned)chunks;
    const int32_t chunk = (int32_t)(blockIdx.x - (unsigned)r * (unsigned)chunks);
    const T* x = static_cast<const T*>(a.x) + r * a.stride;
    T* d = static_cast<T*>(a.d) + r * a.d_stride;
    const float lse = a.lse[r], d_loss = a.d_loss[r];
    TeacherRow row;
    row.load(t, r, a.classes, a.scale, warps);
    float mass = 0.f;
#pragma unroll
    for (int i = 0; i < kTeacherEach; ++i) {
        const int k = threadIdx.x + i * kWideThreads;
        if (k < t.entries) { c[k] = row.c[i]; q[k] = row.q[i]; }
        mass += row.q[i];
    }
    mass = block_sum(mass, warps);   // (and c and q are there for all)
    const bool zero = d_loss == 0.f || mass == 0.f || lse == kNegInf;
    RowGrad g;
    g.scale = a.scale; g.minus_lse = -lse; g.base = a.scale * d_loss * mass; g.slope = g.more = 0.f; g.label = -1;
    const Cut<VEC> cut(d, sizeof(T), a.classes);
    const int32_t lo = (int32_t)((int64_t)cut.vecs * chunk / chunks), hi = (int32_t)((int64_t)cut.vecs * (chunk + 1) / chunks);
    float own[kTeacherEach];
#pragma unroll
    for (int i = 0; i < kTeacherEach; ++i) {
        const int k = threadIdx.x + i * kWideThreads;
        const int32_t at = row.c[i] - cut.head;
        const bool here = row.c[i] >= 0 && !zero && (at >= 0 && at < cut.vecs * VEC ? at >= lo * VEC && at < hi * VEC : chunk == 0);
        float of_class;
        if (here && first_of_class(c, q, k, t.entries, &of_class)) {
            float f[1] = {to_float(x[row.c[i]])};
            grads<false>(g, f, 0);
            own[i] = f[0] - a.scale * d_loss * of_class;
        } else row.c[i] = -1;
    }
    __syncthreads();
    stream_row<false, SAME>(g, zero, x, d, cut, lo, hi, chunk == 0, (int)threadIdx.x, kGradThreads);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTeacherEach; ++i)
        if (row.c[i] >= 0) {
            Raw<T, 1> one;
            const float f[1] = {own[i]};
            one.put(f);
            one.store(d + row.c[i]);
        }
}

}  // namespace mgloss
