// What lies between two layers: dropout whose mask comes from a counter-based generator and is never stored, and group norm over rows
// with their channels last, an activation and a dropout behind it.  Both directions; rows of fp32, fp16 or bf16, everything in between
// in fp32.
#include "mg_norm_plan.cuh"

namespace {

constexpr int kThreads = 256;

// ---- dropout ----------------------------------------------------------------------------

template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) k_dropout(const T* x, int64_t x_stride, T* y, int64_t y_stride, int64_t rows, int32_t channels, DropArgs d) {
    const int64_t vecs = (channels + VEC - 1) / VEC, n = rows * vecs;
    for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / vecs;
        const int32_t c = (int32_t)(i - row * vecs) * VEC;
        Pack<T, VEC> p = *reinterpret_cast<const Pack<T, VEC>*>(x + row * x_stride + c);
        const uint32_t bits = d.on ? drop_bits<VEC>(d, drop_key(d, row), (uint32_t)c) : 0xFFu;
#pragma unroll
        for (int e = 0; e < VEC; ++e) from_float(bits >> e & 1u ? to_float(p.v[e]) * d.factor : 0.f, &p.v[e]);
        *reinterpret_cast<Pack<T, VEC>*>(y + row * y_stride + c) = p;
    }
}

// ---- group norm --------------------------------------------------------------------------

struct NormArgs {
    const void* x = nullptr; const void* d_y = nullptr; void* out = nullptr;
    int64_t x_stride = 0, d_y_stride = 0, out_stride = 0;
    const float* weight = nullptr; const float* bias = nullptr;
    float* mean = nullptr; float* rstd = nullptr;         // [samples, groups]
    float* d_weight = nullptr; float* d_bias = nullptr;
    const int64_t* offsets = nullptr;           // device [samples + 1], or null: equal samples
    int64_t rows_per_sample = 0, samples = 0, rows = 0;   // rows: of the samples
    int32_t channels = 0, groups = 0, act = 0;
    float eps = 0.f;
    DropArgs drop;
};

__device__ __forceinline__ float block_sum(float v) {
    __shared__ float part[kThreads / 32];
    __shared__ float all;
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
        float s = 0.f;
        for (int i = 0; i < kThreads / 32; ++i) s += part[i];
        all = s;
    }
    __syncthreads();
    return all;
}

// A block per (sample, group): its values are read for the mean, for the deviation from it and for the result.
template <typename T>
__global__ void __launch_bounds__(kThreads) k_norm(NormArgs a) {
    const int32_t each = a.channels / a.groups;
    const T* x = static_cast<const T*>(a.x);
    T* y = static_cast<T*>(a.out);
    for (int64_t p = blockIdx.x; p < a.samples * a.groups; p += gridDim.x) {
        const int64_t s = p / a.groups;
        const int32_t c0 = (int32_t)(p - s * a.groups) * each;
        const int64_t r0 = a.offsets ? a.offsets[s] : s * a.rows_per_sample, r1 = a.offsets ? a.offsets[s + 1] : r0 + a.rows_per_sample;
        const int64_t n = (r1 - r0) * each;
        float sum = 0.f, sq = 0.f;
        for (int64_t i = threadIdx.x; i < n; i += kThreads) sum += to_float(x[(r0 + i / each) * a.x_stride + c0 + i % each]);
        const float mean = n ? block_sum(sum) / (float)n : 0.f;
        for (int64_t i = threadIdx.x; i < n; i += kThreads) {
            const float d = to_float(x[(r0 + i / each) * a.x_stride + c0 + i % each]) - mean;
            sq += d * d;
        }
        const float rstd = n ? rsqrtf(block_sum(sq) / (float)n + a.eps) : 0.f;
        if (threadIdx.x == 0) { a.mean[p] = mean; a.rstd[p] = rstd; }
        for (int64_t i = threadIdx.x; i < n; i += kThreads) {
            const int64_t row = r0 + i / each;
            const int32_t c = c0 + (int32_t)(i % each);
            float v = (to_float(x[row * a.x_stride + c]) - mean) * rstd;
            v = act_value(a.act, v * (a.weight ? a.weight[c] : 1.f) + (a.bias ? a.bias[c] : 0.f));
            if (a.drop.on) v = drop_bits<1>(a.drop, drop_key(a.drop, row), (uint32_t)c) & 1u ? v * a.drop.factor : 0.f;
            from_float(v, y + row * a.out_stride + c);
        }
    }
}

// gradient in front of the normalisation's weight and bias, and the normalised value
template <typename T>
__device__ __forceinline__ float grad_of(const NormArgs& a, int64_t row, int32_t c, float mean, float rstd, float* hat) {
    const float x = to_float(static_cast<const T*>(a.x)[row * a.x_stride + c]);
    const float w = a.weight ? a.weight[c] : 1.f, b = a.bias ? a.bias[c] : 0.f;
    float g = to_float(static_cast<const T*>(a.d_y)[row * a.d_y_stride + c]);
    if (a.drop.on) g = drop_bits<1>(a.drop, drop_key(a.drop, row), (uint32_t)c) & 1u ? g * a.drop.factor : 0.f;
    *hat = (x - mean) * rstd;
    return g == 0.f ? 0.f : g * act_slope(a.act, *hat * w + b, x, mean, rstd, w, b);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_norm_params(NormArgs a) {   // a block per channel
    const int32_t each = a.channels / a.groups;
    for (int32_t c = blockIdx.x; c < a.channels; c += gridDim.x) {
        float dw = 0.f, db = 0.f;
        for (int64_t s = 0; s < a.samples; ++s) {
            const int64_t r0 = a.offsets ? a.offsets[s] : s * a.rows_per_sample, r1 = a.offsets ? a.offsets[s + 1] : r0 + a.rows_per_sample;
            const float mean = a.mean[s * a.groups + c / each], rstd = a.rstd[s * a.groups + c / each];
            for (int64_t r = r0 + threadIdx.x; r < r1; r += kThreads) {
                float hat;
                const float g = grad_of<T>(a, r, c, mean, rstd, &hat);
                dw += g * hat; db += g;
            }
        }
        dw = block_sum(dw); db = block_sum(db);
        if (threadIdx.x == 0) { if (a.d_weight) a.d_weight[c] = dw; if (a.d_bias) a.d_bias[c] = db; }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_norm_backward(NormArgs a) {
    const int32_t each = a.channels / a.groups;
    T* dx = static_cast<T*>(a.out);
    for (int64_t p = blockIdx.x; p < a.samples * a.groups; p += gridDim.x) {
        const int64_t s = p / a.groups;
        const int32_t c0 = (int32_t)(p - s * a.groups) * each;
        const int64_t r0 = a.offsets ? a.offsets[s] : s * a.rows_per_sample, r1 = a.offsets ? a.offsets[s + 1] : r0 + a.rows_per_sample;
        const int64_t n = (r1 - r0) * each;
        if (n == 0) continue;
        const float mean = a.mean[p], rstd = a.rstd[p];
        float s1 = 0.f, s2 = 0.f, hat;
        for (int64_t i = threadIdx.x; i < n; i += kThreads) {
            const int32_t c = c0 + (int32_t)(i % each);
            const float g = grad_of<T>(a, r0 + i / each, c, mean, rstd, &hat) * (a.weight ? a.weight[c] : 1.f);
            s1 += g; s2 += g * hat;
        }
        s1 = block_sum(s1) / (float)n; s2 = block_sum(s2) / (float)n;
        for (int64_t i = threadIdx.x; i < n; i += kThreads) {
            const int64_t row = r0 + i / each;
            const int32_t c = c0 + (int32_t)(i % each);
            const float g = grad_of<T>(a, row, c, mean, rstd, &hat) * (a.weight ? a.weight[c] : 1.f);
            from_float(rstd * (g - s1 - hat * s2), dx + row * a.out_stride + c);
        }
    }
}

constexpr int kOffsetsPerLaunch = 480;   // (in the kernel's parameters: a host array need not outlive the call, nor a captured graph)
struct OffsetArgs { int64_t at[kOffsetsPerLaunch]; int32_t n; };
__global__ void k_norm_offsets(OffsetArgs a, int64_t* out) {
    for (int i = threadIdx.x; i < a.n; i += blockDim.x) out[i] = a.at[i];
}

struct DeviceScope {   // work goes to the context's device; the caller's current one stays
    int before = -1;
    cudaError_t err;
    explicit DeviceScope(int device) {
        err = cudaGetDevice(&before);
        if (err == cudaSuccess && before != device) err = cudaSetDevice(device);
        else if (err == cudaSuccess) before = -1;
    }
    ~DeviceScope() { if (before >= 0) cudaSetDevice(before); }
};

int norm_args(mg_ctx* ctx, const mg_norm_spec* s, NormArgs* a, void* workspace, size_t workspace_bytes, cudaStream_t st) {
    if (workspace_bytes < norm_workspace(s) || (norm_workspace(s) && !workspace)) return mg_fail(ctx, MG_ERR_CAPACITY, "the workspace is smaller than mg_group_norm_workspace says");
    a->weight = s->weight; a->bias = s->bias;
    a->rows_per_sample = s->rows_per_sample; a->samples = sample_count(s);
    a->rows = s->sample_offsets ? s->sample_offsets[s->n_samples] : s->rows;
    a->channels = s->channels; a->groups = s->groups; a->act = s->activation; a->eps = s->eps;
    if (s->sample_offsets) {
        a->offsets = static_cast<const int64_t*>(workspace);
        for (int32_t lo = 0; lo <= s->n_samples; lo += kOffsetsPerLaunch) {
            OffsetArgs o;
            o.n = std::min(kOffsetsPerLaunch, s->n_samples + 1 - lo);
            memcpy(o.at, s->sample_offsets + lo, sizeof(int64_t) * (size_t)o.n);
            k_norm_offsets<<<1, 256, 0, st>>>(o, static_cast<int64_t*>(workspace) + lo);
            ctx->launches++;
        }
    }
    return MG_OK;
}

template <typename T, int VEC>
void launch_dropout(const void* x, int64_t xs, void* y, int64_t ys, int64_t rows, int32_t channels, const DropArgs& d, int grid, cudaStream_t st) {
    k_dropout<T, VEC><<<grid, kThreads, 0, st>>>(static_cast<const T*>(x), xs, static_cast<T*>(y), ys, rows, channels, d);
}

}  // namespace

extern "C" int mg_dropout(mg_ctx* ctx, const void* x, int64_t x_stride, void* y, int64_t y_stride, int dtype, int64_t rows, int32_t channels,
                          const mg_dropout_spec* spec, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    DropArgs d;
    if (int rc = check_dropout_call(ctx, x, x_stride, y, y_stride, dtype, rows, channels, spec, &d)) return rc;
    if (rows == 0) return MG_OK;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    cudaStream_t st = (cudaStream_t)stream;
    const int grid = mg_grid(ctx, 8);
    const int64_t e = elem_size(dtype);
    const bool wide = channels * e % 16 == 0 && x_stride * e % 16 == 0 && y_stride * e % 16 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0 && reinterpret_cast<uintptr_t>(y) % 16 == 0;
    if (dtype == MG_DTYPE_F32) (wide ? launch_dropout<float, 4> : launch_dropout<float, 1>)(x, x_stride, y, y_stride, rows, channels, d, grid, st);
    else if (dtype == MG_DTYPE_F16) (wide ? launch_dropout<__half, 8> : launch_dropout<__half, 1>)(x, x_stride, y, y_stride, rows, channels, d, grid, st);
    else (wide ? launch_dropout<__nv_bfloat16, 8> : launch_dropout<__nv_bfloat16, 1>)(x, x_stride, y, y_stride, rows, channels, d, grid, st);
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

extern "C" int mg_group_norm_workspace(mg_ctx* ctx, const mg_norm_spec* spec, int backward, size_t* bytes) {
    if (!ctx) return MG_ERR_ARG;
    if (!bytes) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    if (int rc = check_norm(ctx, spec)) return rc;
    (void)backward;
    *bytes = norm_workspace(spec);
    return MG_OK;
}

extern "C" int mg_group_norm(mg_ctx* ctx, const mg_norm_spec* spec, const void* x, int64_t x_stride, void* y, int64_t y_stride, float* mean, float* rstd,
                             void* workspace, size_t workspace_bytes, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    NormArgs a;
    int rc = check_norm_call(ctx, spec, x, x_stride, nullptr, 0, false, y, y_stride, mean, rstd, workspace, &a.drop);
    if (rc || sample_count(spec) == 0) return rc;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    cudaStream_t st = (cudaStream_t)stream;
    if ((rc = norm_args(ctx, spec, &a, workspace, workspace_bytes, st))) return rc;
    a.x = x; a.x_stride = x_stride; a.out = y; a.out_stride = y_stride; a.mean = mean; a.rstd = rstd;
    const int grid = (int)std::min<int64_t>(a.samples * a.groups, mg_grid(ctx, 64));
    if (spec->dtype == MG_DTYPE_F32) k_norm<float><<<grid, kThreads, 0, st>>>(a);
    else if (spec->dtype == MG_DTYPE_F16) k_norm<__half><<<grid, kThreads, 0, st>>>(a);
    else k_norm<__nv_bfloat16><<<grid, kThreads, 0, st>>>(a);
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

extern "C" int mg_group_norm_backward(mg_ctx* ctx, const mg_norm_spec* spec, const void* x, int64_t x_stride, const void* d_y, int64_t d_y_stride,
                                      const float* mean, const float* rstd, void* d_x, int64_t d_x_stride, float* d_weight, float* d_bias,
                                      void* workspace, size_t workspace_bytes, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    NormArgs a;
    int rc = check_norm_call(ctx, spec, x, x_stride, d_y, d_y_stride, true, d_x, d_x_stride, mean, rstd, workspace, &a.drop);
    if (rc) return rc;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    cudaStream_t st = (cudaStream_t)stream;
    if ((rc = norm_args(ctx, spec, &a, workspace, workspace_bytes, st))) return rc;
    a.x = x; a.x_stride = x_stride; a.d_y = d_y; a.d_y_stride = d_y_stride; a.out = d_x; a.out_stride = d_x_stride;
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd); a.d_weight = d_weight; a.d_bias = d_bias;
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(a.samples * a.groups, mg_grid(ctx, 64)));
    const auto go = [&](auto params, auto rows_kernel) {
        if (d_weight || d_bias) { params<<<std::min(spec->channels, mg_grid(ctx, 8)), kThreads, 0, st>>>(a); ctx->launches++; }   // (first: d_x may be d_y or x)
        rows_kernel<<<grid, kThreads, 0, st>>>(a);
        ctx->launches++;
    };
    if (spec->dtype == MG_DTYPE_F32) go(k_norm_params<float>, k_norm_backward<float>);
    else if (spec->dtype == MG_DTYPE_F16) go(k_norm_params<__half>, k_norm_backward<__half>);
    else go(k_norm_params<__nv_bfloat16>, k_norm_backward<__nv_bfloat16>);
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}
