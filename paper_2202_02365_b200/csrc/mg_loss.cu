// Losses of a layer's output: log probabilities with entropy and top alternatives, distillation from a teacher's top logits, and their gradients.
#include "mg_loss_plan.cuh"
#include "mg_norm.cuh"

namespace {

constexpr int kLossThreads = 256;
constexpr float kNegInf = -__builtin_huge_valf();

template <typename T> __device__ __forceinline__ float to_float(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ int64_t id_at(const void* ids, int is_i64, int64_t i) {
    return is_i64 ? static_cast<const int64_t*>(ids)[i] : (int64_t)static_cast<const int32_t*>(ids)[i];
}

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

template <typename F>
__device__ float block_reduce(float v, F f) {
    __shared__ float part[kLossThreads / 32];
    for (int o = 16; o; o >>= 1) v = f(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < kLossThreads / 32; ++w) v = f(v, part[w]);
    return v;
}
__device__ __forceinline__ float block_sum(float v) { return block_reduce(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float block_max(float v) { return block_reduce(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ uint64_t block_max_key(uint64_t v) {
    __shared__ uint64_t part[kLossThreads / 32];
    for (int o = 16; o; o >>= 1) v = max(v, (uint64_t)__shfl_xor_sync(0xFFFFFFFFu, (unsigned long long)v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < kLossThreads / 32; ++w) v = max(v, part[w]);
    return v;
}

// m = the largest logit (0 where none is allowed), sum of exp(scale (x - m)), and of it times scale (x - m)
struct RowStats { float m, sum, weighted; bool none; };

template <typename T>
__device__ RowStats row_stats(const T* x, int32_t classes, float scale) {
    float m = kNegInf;
    for (int32_t c = threadIdx.x; c < classes; c += kLossThreads) m = fmaxf(m, to_float(x[c]));
    m = block_max(m);
    float bad = 0.f;
    RowStats s{m, 0.f, 0.f, false};
    if (m == kNegInf) s.m = 0.f;
    for (int32_t c = threadIdx.x; c < classes; c += kLossThreads) {
        const float d = scale * (to_float(x[c]) - s.m), e = expf(d);
        s.sum += e;
        if (e > 0.f) s.weighted += e * d;
        if (d != d) bad = 1.f;
    }
    s.sum = block_sum(s.sum);
    s.weighted = block_sum(s.weighted);
    s.none = m == kNegInf && block_sum(bad) == 0.f;
    return s;
}

struct ScoreArgs {
    const void* labels; int labels_are_i64;
    int32_t top;
    float *log_prob, *entropy, *lse; int32_t* top_ids; float* top_log_probs;
};

template <typename T>
__global__ void __launch_bounds__(kLossThreads) k_log_probs(const T* all, int64_t stride, int64_t rows, int32_t classes, float scale, ScoreArgs a) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* x = all + r * stride;
        const RowStats s = row_stats(x, classes, scale);
        const float log_sum = logf(s.sum);   // (-infinity where no class is allowed)
        const auto log_p = [&](float v) { return s.none ? kNegInf : scale * (v - s.m) - log_sum; };
        if (threadIdx.x == 0) {
            if (a.lse) a.lse[r] = fmaf(scale, s.m, log_sum);
            if (a.entropy) a.entropy[r] = s.none ? 0.f : log_sum - s.weighted / s.sum;
            if (a.log_prob) {
                const int64_t label = id_at(a.labels, a.labels_are_i64, r);
                a.log_prob[r] = label >= 0 && label < classes ? log_p(to_float(x[label])) : 0.f;
            }
        }
        uint64_t last = ~0ull;
        for (int k = 0; k < a.top; ++k) {
            uint64_t best = 0;
            for (int32_t c = threadIdx.x; c < classes; c += kLossThreads) {
                const uint64_t key = (uint64_t)order_of(to_float(x[c])) << 32 | (uint32_t)~c;
                if (key < last && key > best) best = key;
            }
            last = block_max_key(best);
            if (threadIdx.x == 0) {
                if (a.top_ids) a.top_ids[r * a.top + k] = (int32_t) ~(uint32_t)last;
                if (a.top_log_probs) a.top_log_probs[r * a.top + k] = log_p(value_of((uint32_t)(last >> 32)));
            }
        }
        __syncthreads();
    }
}

struct ScoreGradArgs {
    const float* lse;
    const void* labels; int labels_are_i64;
    const float *d_log_prob, *entropy, *d_entropy, *d_lse;
};

template <typename T>
__global__ void __launch_bounds__(kLossThreads) k_log_probs_backward(const T* all, int64_t stride, int64_t rows, int32_t classes, float scale, ScoreGradArgs a, T* d_all, int64_t d_stride) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* x = all + r * stride;
        T* d = d_all + r * d_stride;
        const float lse = a.lse[r];
        int64_t label = a.d_log_prob ? id_at(a.labels, a.labels_are_i64, r) : -1;
        if (label >= classes) label = -1;
        const float g = label >= 0 ? a.d_log_prob[r] : 0.f, h = a.d_entropy ? a.d_entropy[r] : 0.f, l = a.d_lse ? a.d_lse[r] : 0.f;
        const float entropy = h != 0.f ? a.entropy[r] : 0.f;
        const bool zero = (g == 0.f && h == 0.f && l == 0.f) || lse == kNegInf;
        for (int32_t c = threadIdx.x; c < classes; c += kLossThreads) {
            float v = 0.f;
            if (!zero) {
                const float log_p = fmaf(scale, to_float(x[c]), -lse), p = expf(log_p);
                v = p == 0.f ? 0.f : p * (l - g - (h != 0.f ? h * (log_p + entropy) : 0.f));
                if (c == label) v += g;
            }
            d[c] = from_float<T>(scale * v);
        }
    }
}

struct TeacherArgs {
    const void *ids, *values; const float* lse;
    int64_t ids_stride, values_stride;
    int ids_are_i64, dtype;
    int32_t entries;
};

// the teacher's classes of a row (-1: no pair) and their probabilities, and the sum of these
__device__ float teacher_row(const TeacherArgs& t, int64_t r, int32_t classes, float scale, int32_t* ids, float* q, float* log_q) {
    float m = kNegInf;
    for (int k = threadIdx.x; k < t.entries; k += kLossThreads) {
        const int64_t id = id_at(t.ids, t.ids_are_i64, r * t.ids_stride + k);
        ids[k] = id >= 0 && id < classes ? (int32_t)id : -1;
        const int64_t at = r * t.values_stride + k;
        float v = kNegInf;
        if (ids[k] >= 0) v = scale * (t.dtype == MG_DTYPE_F32 ? static_cast<const float*>(t.values)[at] : t.dtype == MG_DTYPE_F16 ? to_float(static_cast<const __half*>(t.values)[at]) : to_float(static_cast<const __nv_bfloat16*>(t.values)[at]));
        log_q[k] = v;
        m = fmaxf(m, v);
        if (v != v) m = v;
    }
    float sum = 0.f, shift;
    if (t.lse) shift = t.lse[r];
    else {
        m = block_max(m);
        if (m == kNegInf) m = 0.f;
        for (int k = threadIdx.x; k < t.entries; k += kLossThreads) sum += expf(log_q[k] - m);
        sum = block_sum(sum);
        shift = sum == 0.f ? 0.f : m + logf(sum);
    }
    sum = 0.f;
    for (int k = threadIdx.x; k < t.entries; k += kLossThreads) {
        if (ids[k] >= 0) log_q[k] -= shift;
        q[k] = ids[k] >= 0 ? expf(log_q[k]) : 0.f;
        sum += q[k];
    }
    return block_sum(sum);
}

template <typename T>
__global__ void __launch_bounds__(kLossThreads) k_distill(const T* all, int64_t stride, int64_t rows, int32_t classes, float scale, TeacherArgs t, float* loss, float* lse) {
    __shared__ int32_t ids[MG_MAX_TEACHER];
    __shared__ float q[MG_MAX_TEACHER], log_q[MG_MAX_TEACHER];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* x = all + r * stride;
        const RowStats s = row_stats(x, classes, scale);
        const float log_sum = logf(s.sum);
        teacher_row(t, r, classes, scale, ids, q, log_q);
        float v = 0.f;
        for (int k = threadIdx.x; k < t.entries; k += kLossThreads)
            if (ids[k] >= 0 && q[k] != 0.f) v += q[k] * (log_q[k] - (s.none ? kNegInf : scale * (to_float(x[ids[k]]) - s.m) - log_sum));
        v = block_sum(v);
        if (threadIdx.x == 0) {
            loss[r] = v;
            if (lse) lse[r] = fmaf(scale, s.m, log_sum);
        }
        __syncthreads();
    }
}

template <typename T>
__global__ void __launch_bounds__(kLossThreads) k_distill_backward(const T* all, int64_t stride, int64_t rows, int32_t classes, float scale, const float* all_lse, TeacherArgs t, const float* d_loss, T* d_all, int64_t d_stride) {
    __shared__ int32_t ids[MG_MAX_TEACHER];
    __shared__ float q[MG_MAX_TEACHER], log_q[MG_MAX_TEACHER];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* x = all + r * stride;
        T* d = d_all + r * d_stride;
        const float lse = all_lse[r], g = d_loss[r], mass = teacher_row(t, r, classes, scale, ids, q, log_q);
        const bool zero = g == 0.f || mass == 0.f || lse == kNegInf;
        __syncthreads();
        for (int32_t c = threadIdx.x; c < classes; c += kLossThreads) {
            float v = 0.f;
            if (!zero) {
                v = mass * expf(fmaf(scale, to_float(x[c]), -lse));
                for (int k = 0; k < t.entries; ++k)
                    if (ids[k] == c) v -= q[k];
            }
            d[c] = from_float<T>(scale * g * v);
        }
        __syncthreads();
    }
}

TeacherArgs teacher_args(const mg_teacher* t) { return {t->ids, t->values, t->lse, t->ids_stride, t->values_stride, t->ids_are_i64, t->dtype, t->entries}; }

}  // namespace

extern "C" int mg_log_probs(mg_ctx* ctx, const mg_logits* z, const void* labels, int labels_are_i64, int32_t top, float* log_prob, float* entropy, float* lse,
                            int32_t* top_ids, float* top_log_probs, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_log_probs(ctx, z, labels, labels_are_i64, top, log_prob, entropy, lse, top_ids, top_log_probs)) return rc;
    if (z->rows == 0) return MG_OK;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const ScoreArgs a{labels, labels_are_i64, top, log_prob, entropy, lse, top_ids, top_log_probs};
    const int grid = (int)std::min<int64_t>(z->rows, mg_grid(ctx, 8));
    MG_BY_TYPE(z->dtype, (k_log_probs<T><<<grid, kLossThreads, 0, (cudaStream_t)stream>>>(static_cast<const T*>(z->x), z->stride, z->rows, z->classes, z->scale, a)));
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

extern "C" int mg_log_probs_backward(mg_ctx* ctx, const mg_logits* z, const float* lse, const void* labels, int labels_are_i64, const float* d_log_prob,
                                     const float* entropy, const float* d_entropy, const float* d_lse, void* d_x, int64_t d_x_stride, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_log_probs_backward(ctx, z, lse, labels, labels_are_i64, d_log_prob, entropy, d_entropy, d_lse, d_x, d_x_stride)) return rc;
    if (z->rows == 0) return MG_OK;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const ScoreGradArgs a{lse, labels, labels_are_i64, d_log_prob, entropy, d_entropy, d_lse};
    const int grid = (int)std::min<int64_t>(z->rows, mg_grid(ctx, 8));
    MG_BY_TYPE(z->dtype, (k_log_probs_backward<T><<<grid, kLossThreads, 0, (cudaStream_t)stream>>>(static_cast<const T*>(z->x), z->stride, z->rows, z->classes, z->scale, a, static_cast<T*>(d_x), d_x_stride)));
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

extern "C" int mg_distill(mg_ctx* ctx, const mg_logits* z, const mg_teacher* teacher, float* loss, float* lse, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_distill(ctx, z, teacher, loss, lse)) return rc;
    if (z->rows == 0) return MG_OK;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const int grid = (int)std::min<int64_t>(z->rows, mg_grid(ctx, 8));
    MG_BY_TYPE(z->dtype, (k_distill<T><<<grid, kLossThreads, 0, (cudaStream_t)stream>>>(static_cast<const T*>(z->x), z->stride, z->rows, z->classes, z->scale, teacher_args(teacher), loss, lse)));
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

extern "C" int mg_distill_backward(mg_ctx* ctx, const mg_logits* z, const float* lse, const mg_teacher* teacher, const float* d_loss, void* d_x,
                                   int64_t d_x_stride, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_distill_backward(ctx, z, lse, teacher, d_loss, d_x, d_x_stride)) return rc;
    if (z->rows == 0) return MG_OK;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const int grid = (int)std::min<int64_t>(z->rows, mg_grid(ctx, 8));
    MG_BY_TYPE(z->dtype, (k_distill_backward<T><<<grid, kLossThreads, 0, (cudaStream_t)stream>>>(static_cast<const T*>(z->x), z->stride, z->rows, z->classes, z->scale, lse, teacher_args(teacher), d_loss, static_cast<T*>(d_x), d_x_stride)));
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}
