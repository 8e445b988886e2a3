// Gradients with respect to logits: rows, or pieces of rows, from the logits and a few values by row; each value is read and written once.
#pragma once

#include "mg_loss_rows.cuh"
#include "mg_loss_wide.cuh"

namespace mgloss {

constexpr int kGradThreads = 256, kGradBatch = 4;   // vectors of a thread that are on their way at once

// In the place of smaller logarithms, whose probabilities are zero in fp32 (e^-104): times any gradient of the entropy, up to 1e36, it stays a number.
constexpr float kLeastLog = -200.f;

// What a row's gradient is made of: p (base + slope log p), log p = scale (x - about) + minus_lse (ABOUT), or without `about`: kernels of their own, since the difference and its register cost those
// that do without up to 7 %.
struct RowGrad { float scale, about, minus_lse, base, slope; };

// What the forward call has left of a row: what its sum of exponentials was taken about and the sum's logarithm, or one number for both, of which a large one has lost the second.
// (As they are loaded: an operation on them here holds the loads behind them up; 777,777 fp16 rows of 153 107 us, 111.)
struct RowLog {
    float about, lse;
    __device__ __forceinline__ bool none() const { return lse == kNegInf; }   // no class is allowed
};
template <bool ABOUT>
__device__ __forceinline__ RowLog row_log(const GradArgs& a, int64_t r) {
    if (ABOUT) {
        const float2 s = a.row_sums[r];
        return {s.x, s.y};
    }
    return {0.f, a.lse[r]};
}

// The exponentials of two logarithms of probabilities.  Of fp32 rows by expf: the special function unit's power of two is as many units of 2^-24 off as the logarithm has (three times
// the plain form's error over a gradient), which the rounding to two bytes covers.  2,048 rows of 50,257 take as long.
template <bool EXACT>
__device__ __forceinline__ Pair exp_of(Pair log_p) {
    float a, b;
    if (EXACT) {
        split(log_p, &a, &b);
        return pair(expf(a), expf(b));
    }
    split(mul2(log_p, pair(kLog2e, kLog2e)), &a, &b);
    return pair(fast_exp2(a), fast_exp2(b));
}

// the gradients of neighbouring classes, in place of their logits
template <bool EXACT, bool ABOUT, int N>
__device__ __forceinline__ void grads(const RowGrad& g, float (&v)[N]) {
    if constexpr (N == 1) {
        const float log_p = fmaf(ABOUT ? v[0] - g.about : v[0], g.scale, g.minus_lse);
        v[0] = expf(log_p) * fmaf(fmaxf(log_p, kLeastLog), g.slope, g.base);
    } else {
        const Pair scale = pair(g.scale, g.scale), about = pair(-g.about, -g.about), lse = pair(g.minus_lse, g.minus_lse), base = pair(g.base, g.base), slope = pair(g.slope, g.slope);
        const bool sloped = g.slope != 0.f;
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            Pair x = pair(v[i], v[i + 1]);
            if (ABOUT) x = add2(x, about);
            const Pair log_p = fma2(x, scale, lse), p = exp_of<EXACT>(log_p);
            Pair d;
            if (sloped) {
                float a, b;
                split(log_p, &a, &b);
                d = mul2(p, fma2(pair(fmaxf(a, kLeastLog), fmaxf(b, kLeastLog)), slope, base));
            } else d = mul2(p, base);
            split(d, &v[i], &v[i + 1]);
        }
    }
}

// one class's gradient, and `more`
template <bool ABOUT, typename T>
__device__ __forceinline__ void write_one(const RowGrad& g, float x, float more, T* to) {
    float f[1] = {x};
    grads<true, ABOUT>(g, f);
    f[0] += more;
    Raw<T, 1> one;
    one.put(f);
    one.store(to);
}

// Vectors [lo, hi) of what covers the gradient's row, by `lanes` threads.  WHOLE: rows of both begin and end with a vector; SAME: the logits' vectors begin where the
// gradient's do, else they are read element by element (2,048 fp32 rows of 50,257: 135 us, with logits that begin elsewhere 140; 4,096 bf16 ones 154 and 195).
// Bound by the bytes: 824 MB in 139 us, 92 % of the copy's rate, with a teacher's pairs.
template <bool ABOUT, bool SAME, bool WHOLE, typename T>
__device__ __forceinline__ void stream_row(const RowGrad& g, bool zero, const T* x, T* d, int32_t classes, int32_t lead, int32_t lo, int32_t hi, int sub, int lanes) {
    constexpr int VEC = 16 / sizeof(T);
    for (int32_t v0 = lo + sub; v0 < hi; v0 += kGradBatch * lanes) {
        Raw<T, VEC> raw[kGradBatch];
        T one[SAME ? 1 : kGradBatch * VEC];
        if (!zero) {
#pragma unroll
            for (int j = 0; j < kGradBatch; ++j) {
                const int32_t c = (v0 + j * lanes) * VEC - lead;
                if (v0 + j * lanes < hi && (WHOLE || (c >= 0 && c + VEC <= classes))) {
                    if constexpr (SAME) raw[j].load(x + c);
                    else
#pragma unroll
                        for (int e = 0; e < VEC; ++e) one[j * VEC + e] = x[c + e];
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kGradBatch; ++j) {
            if (v0 + j * lanes >= hi) continue;
            const int32_t c = (v0 + j * lanes) * VEC - lead;
            const bool full = WHOLE || (c >= 0 && c + VEC <= classes);
            float f[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if constexpr (SAME) f[e] = raw[j].get(e);
                else f[e] = to_float(one[j * VEC + e]);
            }
            if (!full && !zero)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (c + e >= 0 && c + e < classes) f[e] = to_float(x[c + e]);
            if (zero) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = 0.f;
            } else grads<sizeof(T) == 4, ABOUT>(g, f);
            raw[j].put(f);
            if (full) raw[j].store(d + c);
            else
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (c + e >= 0 && c + e < classes) {
                        Raw<T, 1> one_out;
                        const float v[1] = {f[e]};
                        one_out.put(v);
                        one_out.store(d + c + e);
                    }
        }
    }
}

// `lanes` threads to a row, or to one of its `chunks` pieces.  The label's gradient is written over what its vector got, by the thread that had the vector.
template <typename T, bool ABOUT, bool SAME, bool WHOLE>
__global__ void __launch_bounds__(kGradThreads) k_scores_grad(const __grid_constant__ GradArgs a, int lanes_log2, int chunks, int32_t piece) {
    constexpr int VEC = 16 / sizeof(T);
    const int lanes = 1 << lanes_log2, group = (int)threadIdx.x >> lanes_log2, sub = (int)threadIdx.x & (lanes - 1), groups = kGradThreads >> lanes_log2;
    const int64_t r = chunks == 1 ? (int64_t)blockIdx.x * groups + group : blockIdx.x / (unsigned)chunks;
    if (r < a.rows) {
        const int32_t chunk = chunks == 1 ? 0 : (int32_t)(blockIdx.x - (unsigned)r * (unsigned)chunks);
        const T* x = static_cast<const T*>(a.x) + r * a.stride;
        T* d = static_cast<T*>(a.d) + r * a.d_stride;
        const Cover<VEC> cover(d, sizeof(T), a.classes, WHOLE);
        int32_t lo = 0, hi = cover.vecs;
        if (chunks > 1) { lo = min(chunk * piece, cover.vecs); hi = min(lo + piece, cover.vecs); }
        const RowLog of = row_log<ABOUT>(a, r);
        const int32_t label = a.d_log_prob ? class_at(a.labels, a.labels_are_i64, r, a.classes) : -1;
        const float of_label = label >= 0 ? a.d_log_prob[r] : 0.f, h = a.d_entropy ? a.d_entropy[r] : 0.f, l = a.d_lse ? a.d_lse[r] : 0.f;
        const float entropy = h != 0.f ? a.entropy[r] : 0.f;
        const bool zero = (of_label == 0.f && h == 0.f && l == 0.f) || of.none();
        const RowGrad g{a.scale, of.about, -of.lse, a.scale * (l - of_label - h * entropy), -a.scale * h};
        const int32_t at = (label + cover.lead) / VEC;
        const bool mine = label >= 0 && !zero && at >= lo && at < hi && ((at - lo) & (lanes - 1)) == sub;
        const float x_label = mine ? to_float(x[label]) : 0.f;
        stream_row<ABOUT, SAME, WHOLE>(g, zero, x, d, a.classes, cover.lead, lo, hi, sub, lanes);
        if (mine) write_one<ABOUT>(g, x_label, a.scale * of_label, d + label);
    }
}

// Rows of up to some thousand classes that lie one behind the other, in both matrices: blocks of rows as one run of vectors, whatever rows these cross.  What a row's gradient
// goes by is worked out once, by one thread, into shared memory; a vector's two rows are told apart value by value (CROSS; else no vector crosses).  Rows taken one
// by one, 777,777 fp16 ones of 153 took 150 us, 30 instructions a value, most of them for vectors that begin or end within a row; so 113 for 498 MB (4.4 TB/s), 16 instructions a value.  What
// bounds it are the latencies at a block's beginning and end; vectors are asked for before the rows' values.
struct FlatRow { float minus_lse, base, slope; int32_t zero; };
constexpr int kFlatRows = 256;   // a block's, at most
template <typename T, bool CROSS, bool ABOUT>
__global__ void __launch_bounds__(kGradThreads, 4) k_scores_grad_flat(const __grid_constant__ GradArgs a, int rows_each, uint32_t reciprocal) {
    constexpr int VEC = 16 / sizeof(T);
    __shared__ FlatRow params[kFlatRows + 1];
    __shared__ float minus_about[ABOUT ? kFlatRows + 1 : 1];
    const int64_t r0 = (int64_t)blockIdx.x * rows_each;
    const int rows = (int)min((int64_t)rows_each, a.rows - r0);
    const T* x = static_cast<const T*>(a.x) + r0 * a.classes;
    T* d = static_cast<T*>(a.d) + r0 * a.classes;
    const int32_t values = rows * a.classes, vecs = values / VEC;
    uint4 raw[kGradBatch];   // on their way while the rows' values are worked out
#pragma unroll
    for (int j = 0; j < kGradBatch; ++j)
        if ((int)threadIdx.x + j * kGradThreads < vecs) raw[j] = reinterpret_cast<const uint4*>(x)[threadIdx.x + j * kGradThreads];
    int32_t label = -1;
    float x_label = 0.f, more = 0.f;
    RowGrad own{a.scale, 0.f, 0.f, 0.f, 0.f};
    if ((int)threadIdx.x < rows) {
        const int64_t r = r0 + threadIdx.x;
        const RowLog of = row_log<ABOUT>(a, r);
        const float of_label = a.d_log_prob ? a.d_log_prob[r] : 0.f, h = a.d_entropy ? a.d_entropy[r] : 0.f, l = a.d_lse ? a.d_lse[r] : 0.f;
        const float entropy = a.d_entropy ? a.entropy[r] : 0.f;
        if (a.d_log_prob) label = class_at(a.labels, a.labels_are_i64, r, a.classes);
        if (label >= 0) x_label = to_float(x[(int64_t)threadIdx.x * a.classes + label]);
        const float g = label >= 0 ? of_label : 0.f;
        const bool zero = (g == 0.f && h == 0.f && l == 0.f) || of.none();
        own.about = of.about; own.minus_lse = -of.lse; own.base = a.scale * (l - g - (h != 0.f ? h * entropy : 0.f)); own.slope = -a.scale * h;
        more = a.scale * g;
        if (zero) label = -1;
        params[threadIdx.x] = {own.minus_lse, own.base, own.slope, zero};
        if (ABOUT) minus_about[threadIdx.x] = -own.about;
    }
    __syncthreads();
    const bool sloped = a.d_entropy != nullptr;
    const Pair scale = pair(a.scale, a.scale);
    for (int32_t v0 = threadIdx.x; v0 < vecs; v0 += kGradBatch * kGradThreads) {
#pragma unroll
        for (int j = 0; j < kGradBatch; ++j) {
            const int32_t v = v0 + j * kGradThreads;
            if (v >= vecs) break;
            const int32_t row = (int32_t)__umulhi((uint32_t)(v * VEC), reciprocal), left = (row + 1) * a.classes - v * VEC;   // values of the first row
            const FlatRow p = params[row];
            FlatRow q = p;
            if (CROSS && left < VEC) q = params[row + 1];   // (there is one: the block's values end behind the vector)
            float p_about = 0.f, q_about = 0.f;
            if (ABOUT) {
                p_about = q_about = minus_about[row];
                if (CROSS && left < VEC) q_about = minus_about[row + 1];
            }
            Raw<T, VEC> one;
            one.w[0] = raw[j].x; one.w[1] = raw[j].y; one.w[2] = raw[j].z; one.w[3] = raw[j].w;
            if (v + kGradBatch * kGradThreads < vecs) raw[j] = reinterpret_cast<const uint4*>(x)[v + kGradBatch * kGradThreads];
            float f[VEC];
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
                const bool first = !CROSS || e < left, second = !CROSS || e + 1 < left;
                const Pair lse = CROSS ? pair(first ? p.minus_lse : q.minus_lse, second ? p.minus_lse : q.minus_lse) : pair(p.minus_lse, p.minus_lse);
                Pair factor = CROSS ? pair(first ? p.base : q.base, second ? p.base : q.base) : pair(p.base, p.base);
                Pair x_both = pair(one.get(e), one.get(e + 1));
                if (ABOUT) x_both = add2(x_both, CROSS ? pair(first ? p_about : q_about, second ? p_about : q_about) : pair(p_about, p_about));
                const Pair log_p = fma2(x_both, scale, lse), p_both = exp_of<sizeof(T) == 4>(log_p);
                float s, t;
                if (sloped) {
                    split(log_p, &s, &t);
                    const Pair slope = CROSS ? pair(first ? p.slope : q.slope, second ? p.slope : q.slope) : pair(p.slope, p.slope);
                    factor = fma2(pair(fmaxf(s, kLeastLog), fmaxf(t, kLeastLog)), slope, factor);
                }
                split(mul2(p_both, factor), &f[e], &f[e + 1]);
            }
            if (p.zero | q.zero) {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (!CROSS || e < left ? p.zero : q.zero) f[e] = 0.f;
            }
            one.put(f);
            one.store(d + v * VEC);
        }
    }
    // what is left behind the last vector of the last block's rows
    if ((int)threadIdx.x < values - vecs * VEC) {
        const int32_t at = vecs * VEC + (int32_t)threadIdx.x;
        const FlatRow p = params[rows - 1];   // (less than a vector, and a row has one at least)
        if (p.zero) { Raw<T, 1> none; none.zero(); none.store(d + at); }
        else write_one<ABOUT>({a.scale, ABOUT ? -minus_about[rows - 1] : 0.f, p.minus_lse, p.base, p.slope}, to_float(x[at]), 0.f, d + at);
    }
    __syncthreads();
    if (label >= 0) write_one<ABOUT>(own, x_label, more, d + (int64_t)threadIdx.x * a.classes + label);
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

template <typename T, int LANES, bool ABOUT, bool SAME, bool WHOLE>
__global__ void __launch_bounds__(kGradThreads) k_distill_grad_rows(const __grid_constant__ GradArgs a) {
    constexpr int GROUPS = kGradThreads / LANES;
    __shared__ int32_t all_c[kGradThreads * kTeacherRoom];
    __shared__ float all_q[kGradThreads * kTeacherRoom], all_x[kGradThreads * kTeacherRoom];
    const TeacherArgs& t = a.teacher;
    const int group = (int)threadIdx.x / LANES, sub = (int)threadIdx.x % LANES;
    int32_t* c = all_c + group * LANES * kTeacherRoom;
    float *q = all_q + group * LANES * kTeacherRoom, *at_class = all_x + group * LANES * kTeacherRoom;
    for (int64_t r0 = (int64_t)blockIdx.x * GROUPS; r0 < a.rows; r0 += (int64_t)gridDim.x * GROUPS) {
        const int64_t r = r0 + group;
        const bool on = r < a.rows;
        const T* x = static_cast<const T*>(a.x) + (on ? r : 0) * a.stride;
        T* d = static_cast<T*>(a.d) + (on ? r : 0) * a.d_stride;
        const RowLog of = row_log<ABOUT>(a, on ? r : 0);
        const float d_loss = on ? a.d_loss[r] : 0.f;
        // the pairs' classes, values (times the scale) and logits
        float m = kNegInf, shift, sum = 1.f, mass = 0.f;
        for (int k = sub; on && k < t.entries; k += LANES) {
            c[k] = class_at(t.ids, t.ids_are_i64, r * t.ids_stride + k, a.classes);
            if (c[k] < 0) continue;
            q[k] = a.scale * float_at(t.values, t.dtype, r * t.values_stride + k);
            at_class[k] = to_float(x[c[k]]);
            m = fmaxf(m, q[k]);
        }
        if (t.lse) shift = on ? t.lse[r] : 0.f;
        else {
            shift = centre(lanes_max<LANES>(m));
            sum = 0.f;
            for (int k = sub; on && k < t.entries; k += LANES)
                if (c[k] >= 0) sum += expf(q[k] - shift);
            sum = lanes_sum<LANES>(sum);
        }
        const float part = sum == 0.f ? 0.f : 1.f / sum;
        for (int k = sub; on && k < t.entries; k += LANES) {
            q[k] = c[k] >= 0 ? expf(above_shift(q[k], shift)) * part : 0.f;
            mass += q[k];
        }
        mass = lanes_sum<LANES>(mass);
        const bool zero = d_loss == 0.f || mass == 0.f || of.none();
        const RowGrad g{a.scale, of.about, -of.lse, a.scale * d_loss * mass, 0.f};
        __syncwarp();
        const Cover<16 / sizeof(T)> cover(d, sizeof(T), a.classes, WHOLE);
        if (on) stream_row<ABOUT, SAME, WHOLE>(g, zero, x, d, a.classes, cover.lead, 0, cover.vecs, sub, LANES);
        __syncwarp();
        for (int k = sub; on && !zero && k < t.entries; k += LANES) {
            float of_class;
            if (first_of_class(c, q, k, t.entries, &of_class)) write_one<ABOUT>(g, at_class[k], -a.scale * d_loss * of_class, d + c[k]);
        }
        __syncwarp();
    }
}

// a block to a row, or to one of its `chunks` pieces
template <typename T, bool ABOUT, bool SAME, bool WHOLE>
__global__ void __launch_bounds__(kGradThreads) k_distill_grad(const __grid_constant__ GradArgs a, int chunks, int32_t piece) {
    constexpr int VEC = 16 / sizeof(T);
    __shared__ int32_t c[MG_MAX_TEACHER];
    __shared__ float q[MG_MAX_TEACHER], at_class[MG_MAX_TEACHER], scratch[kTeacherThreads / 32], sh_mass;
    const TeacherArgs& t = a.teacher;
    const int64_t r = blockIdx.x / (unsigned)chunks;
    const int32_t chunk = (int32_t)(blockIdx.x - (unsigned)r * (unsigned)chunks);
    const T* x = static_cast<const T*>(a.x) + r * a.stride;
    T* d = static_cast<T*>(a.d) + r * a.d_stride;
    const RowLog of = row_log<ABOUT>(a, r);
    const float d_loss = a.d_loss[r];
    const Cover<VEC> cover(d, sizeof(T), a.classes, WHOLE);
    const int32_t lo = min(chunk * piece, cover.vecs), hi = min(lo + piece, cover.vecs);
    const int warps = teacher_warps<kTeacherThreads>(t);
    const auto here = [&](int32_t of) { return of >= 0 && (of + cover.lead) / VEC >= lo && (of + cover.lead) / VEC < hi; };
    if ((int)threadIdx.x < warps * 32) {
        const TeacherRow teacher = teacher_row<kTeacherThreads>(t, r, x, a.classes, a.scale, warps, scratch, q, at_class, c, here);
        for (int k = threadIdx.x; k < t.entries; k += kTeacherThreads) q[k] = expf(q[k]) * teacher.part;
        if (threadIdx.x == 0) sh_mass = teacher.mass;
    }
    __syncthreads();
    const float mass = sh_mass;
    const bool zero = d_loss == 0.f || mass == 0.f || of.none();
    const RowGrad g{a.scale, of.about, -of.lse, a.scale * d_loss * mass, 0.f};
    stream_row<ABOUT, SAME, WHOLE>(g, zero, x, d, a.classes, cover.lead, lo, hi, (int)threadIdx.x, kGradThreads);
    __syncthreads();
    if (zero || (int)threadIdx.x >= warps * 32) return;
    for (int k = threadIdx.x; k < t.entries; k += kTeacherThreads) {
        float of_class;
        if (here(c[k]) && first_of_class(c, q, k, t.entries, &of_class)) write_one<ABOUT>(g, at_class[k], -a.scale * d_loss * of_class, d + c[k]);
    }
}

}  // namespace mgloss
