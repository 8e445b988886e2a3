// Device-side pieces of dropout and of group norm: elements of the three row types, the dropout's mask, activations.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "mg_device.cuh"

constexpr uint32_t kDropTag = 0x64720000u;   // counter word 3 of a dropout's draws; the sampler's and the negatives' are far below or all ones

struct DropArgs {
    int on = 0;
    uint32_t limit = 0;      // kept: a 16-bit half at or above it
    float factor = 1.f;      // 65536 / (65536 - limit); 0 where all are dropped
    uint32_t k0 = 0, k1 = 0, tag = 0;
    int64_t first_row = 0;
    const int64_t* keys = nullptr;
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
// (rounded once, to nearest: off by half a step of the type at most)
__device__ __forceinline__ void from_float(float v, float* out) { *out = v; }
__device__ __forceinline__ void from_float(float v, __half* out) { *out = __float2half_rn(v); }
__device__ __forceinline__ void from_float(float v, __nv_bfloat16* out) { *out = __float2bfloat16_rn(v); }

template <typename T, int VEC> struct alignas(sizeof(T) * VEC) Pack { T v[VEC]; };

__device__ __forceinline__ uint64_t drop_key(const DropArgs& d, int64_t row) { return (uint64_t)(d.keys ? d.keys[row] : d.first_row + row); }

// bit i: element c + i of the row with this key is kept (c a multiple of VEC, VEC of 1, 2, 4 or 8): the halves of one Philox block per eight
// elements.  16 bits an element, so that a block serves 16 or 32 bytes of a row: p is met to 2^-17, and the factor goes by the p that is met.
template <int VEC>
__device__ __forceinline__ uint32_t drop_bits(const DropArgs& d, uint64_t key, uint32_t c) {
    uint32_t w[4];
    philox4x32_10((uint32_t)key, (uint32_t)(key >> 32), c >> 3, d.tag, d.k0, d.k1, w);
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bits |= (uint32_t)((w[i] & 0xFFFFu) >= d.limit) << (2 * i);
        bits |= (uint32_t)((w[i] >> 16) >= d.limit) << (2 * i + 1);
    }
    return VEC == 8 ? bits : bits >> (c & 7u);
}

enum { ACT_NONE = 0, ACT_RELU = 1, ACT_SILU = 2, ACT_GELU = 3 };   // MG_ACT_*

__device__ __forceinline__ float act_value(int act, float n) {
    if (act == ACT_RELU) return n < 0.f ? 0.f : n;   // (NaN stays)
    if (act == ACT_SILU) return n / (1.f + expf(-n));
    if (act == ACT_GELU) return 0.5f * n * (1.f + erff(n * 0.70710678118654752f));
    return n;
}

// slope of the activation at n = hat * w + b.  A ReLU's slope jumps at zero: which side n lies on is decided in 64 bits where 32 leave it open,
// so that the gradient does not go by how a sum was rounded.
__device__ __forceinline__ float act_slope(int act, float n, float x, float mean, float rstd, float w, float b) {
    if (act == ACT_RELU) {
        // |rounding of n| < 4 * 2^-24 * (|n - b| + |b|): three roundings of hat * w, one of the sum
        const float reach = 3e-7f * (fabsf(n - b) + fabsf(b));
        if (fabsf(n) > reach) return n > 0.f ? 1.f : 0.f;
        const double at = ((double)x - (double)mean) * (double)rstd * (double)w + (double)b;
        return at <= 0.0 ? 0.f : 1.f;
    }
    if (act == ACT_SILU) {
        const float s = 1.f / (1.f + expf(-n));
        return s * (1.f + n * (1.f - s));
    }
    if (act == ACT_GELU) return 0.5f * (1.f + erff(n * 0.70710678118654752f)) + n * expf(-0.5f * n * n) * 0.39894228040143268f;
    return 1.f;
}
