// Device-side pieces of dropout and of group norm: elements of the three row types, the dropout's mask, activations.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "mg_device.cuh"

constexpr uint32_t kDropTag = 0x64720000u;   // counter word 3 of a dropout's draws; the sampler's and the negatives' are far below or all ones

struct DropArgs {
    int on = 0;
    uint32_t below = 0;      // kept: a 16-bit half at or above the limit, that is, as the upper half of a word above limit * 65536 - 1
    float factor = 1.f;      // 65536 / (65536 - limit); 0 where all are dropped
    uint32_t k0[10] = {0}, k1[10] = {0};   // the rounds' keys: those of the seed, and 0x9E3779B9, 0xBB67AE85 more with every round
    uint32_t tag = 0;
    int64_t first_row = 0;
    const int64_t* keys = nullptr;
};

// VEC neighbouring elements of a row as they lie in memory: 2, 4, 8, 16 or 32 bytes in one access
template <typename T, int VEC> struct Raw {
    static constexpr int kBytes = (int)sizeof(T) * VEC, kWords = (kBytes + 3) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    // (volatile, and after what comes before: a row may be read again behind a wait, or be the output too)
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (kBytes == 32)
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
        else if constexpr (kBytes == 16) asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p) : "memory");
        else if constexpr (kBytes == 8) asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p) : "memory");
        else if constexpr (kBytes == 4) asm volatile("ld.global.b32 %0, [%1];" : "=r"(w[0]) : "l"(p) : "memory");
        else {
            uint16_t h;
            asm volatile("ld.global.b16 %0, [%1];" : "=h"(h) : "l"(p) : "memory");
            w[0] = h;
        }
    }
    __device__ __forceinline__ void store(T* p) const {
        if constexpr (kBytes == 32)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
        else if constexpr (kBytes == 16) asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
        else if constexpr (kBytes == 8) asm volatile("st.global.v2.b32 [%0], {%1, %2};" ::"l"(p), "r"(w[0]), "r"(w[1]) : "memory");
        else if constexpr (kBytes == 4) asm volatile("st.global.b32 [%0], %1;" ::"l"(p), "r"(w[0]) : "memory");
        else asm volatile("st.global.b16 [%0], %1;" ::"l"(p), "h"((uint16_t)w[0]) : "memory");
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        else return __half2float(__ushort_as_half((unsigned short)(w[i / 2] >> (i & 1) * 16)));
    }
    // (rounded once, to nearest: off by half a step of the type at most)
    __device__ __forceinline__ void put(const float (&f)[VEC]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) w[i] = __float_as_uint(f[i]);
        } else if constexpr (VEC == 1) {
            if constexpr (std::is_same<T, __half>::value) w[0] = __half_as_ushort(__float2half_rn(f[0]));
            else w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
        } else {
#pragma unroll
            for (int i = 0; i < VEC; i += 2) {
                if constexpr (std::is_same<T, __half>::value) {
                    const __half2 h = __floats2half2_rn(f[i], f[i + 1]);
                    w[i / 2] = reinterpret_cast<const uint32_t&>(h);
                } else {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(f[i], f[i + 1]);
                    w[i / 2] = reinterpret_cast<const uint32_t&>(h);
                }
            }
        }
    }
};

__device__ __forceinline__ uint64_t drop_key(const DropArgs& d, int64_t row) { return (uint64_t)(d.keys ? d.keys[row] : d.first_row + row); }

// philox4x32_10 with the rounds' keys from the kernel's parameters
__device__ __forceinline__ void drop_block(const DropArgs& d, uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t out[4]) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ d.k0[r]; c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ d.k1[r]; c3 = (uint32_t)p0;
    }
    out[0] = c0; out[1] = c1; out[2] = c2; out[3] = c3;
}

// Which of elements c .. c + VEC - 1 of the row with this key are kept (c a multiple of VEC; VEC of 1, 2, 4 or 8): the halves of one Philox
// block per eight elements.  16 bits an element, so that a block serves 16 or 32 bytes of a row: p is met to 2^-17, and the factor goes by
// the p that is met.
template <int VEC> struct Keep {
    uint32_t w[(VEC + 1) / 2];
    __device__ __forceinline__ void draw(const DropArgs& d, uint64_t key, uint32_t c) {
        uint32_t all[4];
        drop_block(d, (uint32_t)key, (uint32_t)(key >> 32), c >> 3, d.tag, all);
        if constexpr (VEC == 8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = all[i];
        } else if constexpr (VEC == 4) {
            w[0] = c & 4 ? all[2] : all[0];
            w[1] = c & 4 ? all[3] : all[1];
        } else {
            const uint32_t lo = c & 2 ? all[1] : all[0], hi = c & 2 ? all[3] : all[2];
            w[0] = c & 4 ? hi : lo;
            if (VEC == 1 && (c & 1)) w[0] >>= 16;
        }
    }
    __device__ __forceinline__ bool operator()(const DropArgs& d, int i) const { return (i & 1 ? w[i / 2] : w[i / 2] << 16) > d.below; }
};

enum { ACT_NONE = 0, ACT_RELU = 1, ACT_SILU = 2, ACT_GELU = 3 };   // MG_ACT_*

// The special function unit's power of two and reciprocal, each off by 2^-22 of itself (results below 2^-126 are zero).  Activations alone use them; sums and
// statistics do without.  Against 64 bits a SiLU of n is off by 3 * 2^-24 |n| at most, a GELU by 6 (below -4, where its value is a small difference, by more of itself:
// half of what 1 + erff costs there); their slopes by 17 and 6 units of 2^-24.  (expf and a division take four times the instructions.)
__device__ __forceinline__ float fast_exp2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float fast_rcp(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float sigmoid(float n) { return fast_rcp(1.f + fast_exp2(-1.4426950408889634f * n)); }

// (1 + erf(n / sqrt 2)) / 2 to 4 * 2^-24, by Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26 (1.5e-7 off in erf, its
// polynomial's coefficients halved here); `bell` = e^(-n^2 / 2), which the slope wants too.  A third of erff's instructions.
__device__ __forceinline__ float normal_cdf(float n, float* bell) {
    const float t = fast_rcp(fmaf(0.3275911f * 0.70710678118654752f, fabsf(n), 1.f));
    *bell = fast_exp2(n * n * -0.72134752044448170f);
    const float tail = *bell * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5307027145f, -0.7265760135f), 0.7107068705f), -0.142248368f), 0.127414796f);
    return n < 0.f ? tail : 1.f - tail;
}

__device__ __forceinline__ float max_nan(float a, float b) {   // (NaN stays)
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

template <int N>
__device__ __forceinline__ void act_values(int act, float (&n)[N]) {
    if (act == ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) n[e] = max_nan(n[e], 0.f);
    } else if (act == ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; ++e) n[e] *= sigmoid(n[e]);
    } else if (act == ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) { float bell; n[e] *= normal_cdf(n[e], &bell); }
    }
}

// d times the slope of the activation at n, which is fmaf(hat-like factor, weight-like factor, b): exact(e) has element e's in 64 bits.  A ReLU's slope
// jumps at zero: which side n lies on is decided in 64 bits where 32 leave it open, so that the gradient does not go by how a sum was rounded.
template <int N, typename Exact>
__device__ __forceinline__ void act_slopes(int act, float (&d)[N], const float (&n)[N], const float (&b)[N], Exact exact) {
    if (act == ACT_RELU) {
        float side[N];
        bool near = false;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            // |rounding of n| < 4 * 2^-24 * (|n - b| + |b|): three roundings of the product (it enters the sum unrounded), one of the sum
            side[e] = n[e];
            near = near || fabsf(n[e]) <= 3e-7f * fmaf(2.f, fabsf(b[e]), fabsf(n[e]));
        }
        if (near) {   // (hardly ever)
#pragma unroll
            for (int e = 0; e < N; ++e) side[e] = exact(e) <= 0.0 ? -1.f : 1.f;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) d[e] = side[e] <= 0.f ? 0.f : d[e];
    } else if (act == ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float s = sigmoid(n[e]);
            d[e] *= s * fmaf(n[e], 1.f - s, 1.f);
        }
    } else if (act == ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float bell;
            const float cdf = normal_cdf(n[e], &bell);
            d[e] *= fmaf(n[e] * 0.39894228040143268f, bell, cdf);
        }
    }
}

// dropout of a vector's values
template <int VEC>
__device__ __forceinline__ void drop_vector(const DropArgs& d, uint64_t key, int32_t c, float (&f)[VEC]) {
    if (!d.on) return;
    Keep<VEC> keep;
    keep.draw(d, key, (uint32_t)c);
#pragma unroll
    for (int e = 0; e < VEC; ++e) f[e] = keep(d, e) ? f[e] * d.factor : 0.f;
}
