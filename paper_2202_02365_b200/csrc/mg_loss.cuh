// Device-side pieces of the losses: rows of logits cut into aligned vectors, pairs of floats, sums over parts of a warp.
#pragma once

#include "mg_norm.cuh"
#include "mgdense.h"

namespace mgloss {

constexpr float kNegInf = -__builtin_huge_valf(), kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
constexpr float kLeast = -1e30f;   // in the place of -infinity where it is a factor beside a zero

// Floats as whole numbers of the same order, between 0 and 2^32 - 1: equal values (both zeros among them) are equal, NaN is above all.
constexpr uint32_t kNanOrder = 0xFFFFFFFEu;
__device__ __forceinline__ uint32_t order_of(float v) {
    if (v != v) return kNanOrder;
    const uint32_t b = __float_as_uint(v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
    return o == kNanOrder ? __uint_as_float(0x7FFFFFFFu) : __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}
// a class and its value: the larger the better, equal values by ascending class
__device__ __forceinline__ uint64_t key_of(float v, int32_t c) { return (uint64_t)order_of(v) << 32 | (uint32_t)~c; }
__device__ __forceinline__ int32_t class_of(uint64_t key) { return (int32_t) ~(uint32_t)key; }

__device__ __forceinline__ int64_t id_at(const void* ids, int is_i64, int64_t i) {
    return is_i64 ? static_cast<const int64_t*>(ids)[i] : (int64_t)static_cast<const int32_t*>(ids)[i];
}
// a whole number of the caller's as a class, -1 where it is none
__device__ __forceinline__ int32_t class_at(const void* ids, int is_i64, int64_t i, int32_t classes) {
    const int64_t c = id_at(ids, is_i64, i);
    return c >= 0 && c < classes ? (int32_t)c : -1;
}
__device__ __forceinline__ float float_at(const void* p, int dtype, int64_t i) {
    if (dtype == 0) return static_cast<const float*>(p)[i];
    if (dtype == 1) return __half2float(static_cast<const __half*>(p)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
template <typename T> __device__ __forceinline__ float to_float(T v) { return (float)v; }

// Two floats in one register pair: sm_100's instructions on both at once.
struct Pair { uint64_t v; };
__device__ __forceinline__ Pair pair(float a, float b) { Pair r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void split(Pair p, float* a, float* b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(p.v)); }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { Pair r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }
__device__ __forceinline__ Pair add2(Pair a, Pair b) { Pair r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ Pair mul2(Pair a, Pair b) { Pair r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }

// A row cut where 16-byte vectors begin: `head` elements, `vecs` vectors, the rest.  The elements before and behind the vectors, the edges, are
// numbered through; they are fewer than 2 VEC - 1.
template <int VEC> struct Cut {
    int32_t head, vecs, edges;
    __device__ __forceinline__ Cut(const void* row, int elem, int32_t classes) {
        head = min(classes, (int32_t)((16u - (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) / elem);
        vecs = (classes - head) / VEC;
        edges = classes - vecs * VEC;
    }
    __device__ __forceinline__ int32_t edge(int32_t e) const { return e < head ? e : e + vecs * VEC; }
};

// A row covered by 16-byte vectors of memory: the first and the last may reach beyond it.  Vector v has the classes from v VEC - lead on.
template <int VEC> struct Cover {
    int32_t lead, vecs;
    __device__ __forceinline__ Cover(const void* row, int elem, int32_t classes, bool whole) {
        lead = whole ? 0 : (int32_t)((uint32_t)(reinterpret_cast<uintptr_t>(row) & 15u) / (uint32_t)elem);
        vecs = (lead + classes + VEC - 1) / VEC;
    }
};

// the largest of a warp's values (not a NaN where there is a number), in one instruction of sm_100a
__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// over the LANES lanes of one row, side by side
template <int LANES, typename F>
__device__ __forceinline__ float over_lanes(float v, F f) {
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) v = f(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}
template <int LANES> __device__ __forceinline__ float lanes_sum(float v) { return over_lanes<LANES>(v, [](float a, float b) { return a + b; }); }
template <int LANES>
__device__ __forceinline__ float lanes_max(float v) {
    if constexpr (LANES == 32) return warp_max(v);
    else return over_lanes<LANES>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int LANES>
__device__ __forceinline__ uint64_t lanes_max(uint64_t v) {
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) v = max(v, (uint64_t)__shfl_xor_sync(0xFFFFFFFFu, (unsigned long long)v, o));
    return v;
}

// sorted over the LANES lanes of one row, the largest first (a bitonic network)
template <int LANES>
__device__ __forceinline__ float lanes_sorted(float v) {
    const int lane = threadIdx.x & (LANES - 1);
#pragma unroll
    for (int size = 2; size <= LANES; size *= 2)
#pragma unroll
        for (int o = size / 2; o; o >>= 1) {
            const float other = __shfl_xor_sync(0xFFFFFFFFu, v, o);
            v = ((lane & o) == 0) == ((lane & size) == 0) ? fmaxf(v, other) : fminf(v, other);
        }
    return v;
}

// Sums over a row, of powers of two: y = (x - max) scale log2(e), sum = sum 2^y, weighted = sum 2^y y; max: the largest x, in the place of which 0 is taken where no
// class is allowed.  (The difference first: x scale - max scale in one instruction goes beyond fp32 where a mask writes the type's lowest value over a row.)
struct RowSums { float max, sum, weighted; };
__device__ __forceinline__ float centre(float max) { return max == kNegInf ? 0.f : max; }

// what a row's sums say: log sum exp(scale (x - max)), and the rest by it
struct RowResult {
    float max, log_sum, entropy, lse, scale;
    bool none;   // no class is allowed
    __device__ __forceinline__ RowResult(const RowSums& s, float scale) : scale(scale) {
        none = s.max == kNegInf && s.sum == 0.f;
        max = centre(s.max);
        log_sum = logf(s.sum);
        entropy = none ? 0.f : log_sum - kLn2 * (s.weighted / s.sum);
        lse = fmaf(scale, max, log_sum);
    }
    __device__ __forceinline__ float log_p(float x) const { return none ? kNegInf : scale * (x - max) - log_sum; }
    __device__ __forceinline__ float2 sums() const { return make_float2(max, log_sum); }   // (no class is allowed: log_sum is -infinity)
};

struct ScoreArgs {
    const void* x; int64_t stride, rows; int32_t classes; float scale, scale2;   // scale2: scale log2(e)
    const void* labels; int labels_are_i64;
    int32_t top;
    float *log_prob, *entropy, *lse; int32_t* top_ids; float* top_log_probs;
    float2* row_sums;
};

struct TeacherArgs {
    const void *ids, *values; const float* lse;
    int64_t ids_stride, values_stride;
    int ids_are_i64, dtype;
    int32_t entries;
};

// A teacher's value less what its probabilities are taken about.  -infinity is a probability of zero whatever that is: the lse of a row that allows the teacher no class is -infinity, that
// of a row that is padding may be anything.
__device__ __forceinline__ float above_shift(float v, float shift) { return v > kNegInf ? v - shift : v; }

struct GradArgs {
    const void* x; int64_t stride, rows; int32_t classes; float scale;
    void* d; int64_t d_stride;
    const float* lse;
    const void* labels; int labels_are_i64;   // log probabilities
    const float *d_log_prob, *entropy, *d_entropy, *d_lse;
    TeacherArgs teacher;                      // distillation
    const float* d_loss;
    const float2* row_sums;                   // in the place of lse, where there are
};

}  // namespace mgloss
