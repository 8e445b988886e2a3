// What lies between two layers: dropout whose mask comes from a counter-based generator and is never stored, and group norm over rows
// with their channels last, an activation and a dropout behind it.  Both directions; rows of fp32, fp16 or bf16, everything in between
// in fp32.
#include "mg_norm_plan.cuh"

namespace {

// Sums of `n` parts ([n][columns]) by column: 32 columns a block, 32 threads to a column; blockIdx.y: a slice of the parts.  In the last step the
// columns are the weight's gradients, then the bias's.
constexpr int kParamThreads = 1024, kParamParts = 1024;   // (more parts are added up in two steps)
__global__ void __launch_bounds__(kParamThreads) k_norm_params(const float* parts, int64_t n, int64_t columns, float* out, float* d_weight, float* d_bias) {
    constexpr int W = kParamThreads / 32, U = 8;
    __shared__ float part[W][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    chain_wait();
    const int64_t c0 = (int64_t)blockIdx.x * 32, c = c0 + lane, lo = n * blockIdx.y / gridDim.y, hi = n * (blockIdx.y + 1) / gridDim.y;
    float s = 0.f;
    if (c < columns)
        for (int64_t i = lo + warp; i < hi; i += U * W) {
            float v[U];
#pragma unroll
            for (int k = 0; k < U; ++k) v[k] = i + k * W < hi ? __ldcg(parts + (i + k * W) * columns + c) : 0.f;
#pragma unroll
            for (int k = 0; k < U; ++k) s += v[k];
        }
    part[warp][lane] = s;
    __syncthreads();
    // warp w: column c0 + w
    s = part[lane][warp];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    const int64_t to = c0 + warp;
    if (lane || to >= columns) return;
    if (out) { out[blockIdx.y * columns + to] = s; return; }
    float* grad = to < columns / 2 ? d_weight : d_bias;
    if (grad) grad[to < columns / 2 ? to : to - columns / 2] = s;
}

constexpr int kSamplesPerLaunch = 480;   // (in the kernel's parameters: a host array need not outlive the call, nor a captured graph)
struct TableArgs { int2 at[kSamplesPerLaunch]; int32_t n; };
__global__ void k_norm_table(const __grid_constant__ TableArgs a, int2* out) {
    for (int i = threadIdx.x; i < a.n; i += blockDim.x) out[i] = a.at[i];
}

// both directions, arguments checked; `m`: the matrices, the output last
int run_norm(mg_ctx* ctx, const mg_norm_spec* s, const Matrix* m, int n_matrices, bool backward, float* mean, float* rstd, float* d_weight, float* d_bias,
             const DropArgs& drop, void* workspace, size_t workspace_bytes, cudaStream_t st) {
    const int mode = norm_mode(s);
    char* ws = static_cast<char*>(workspace);
    TileArgs a;
    NormPlan p;
    a.x = m[0].p; a.x_stride = m[0].stride;
    if (backward) { a.d_y = m[1].p; a.d_y_stride = m[1].stride; }
    a.out = const_cast<void*>(m[n_matrices - 1].p); a.out_stride = m[n_matrices - 1].stride;
    a.weight = s->weight; a.bias = s->bias; a.mean = mean; a.rstd = rstd;
    a.rows = s->rows; a.channels = s->channels; a.groups = s->groups; a.act = s->activation; a.eps = s->eps;
    a.each = s->channels / s->groups; a.drop = drop;
    const bool params = d_weight || d_bias;
    if (mode == NORM_ROWS) plan_rows(s, ctx->n_sms, backward, rows_vec_width(m, n_matrices, s), &p);
    else if (mode == NORM_TILES) plan_samples(s, ctx->n_sms, backward, vec_width(m, n_matrices, s->dtype, s->rows, a.each), &p, &a);
    // (what this plan wants, which is what mg_group_norm_workspace says or less: planning for every alignment again took 230 us for 4,096 samples)
    if (workspace_bytes < p.bytes || (!workspace && p.bytes))
        return mg_fail(ctx, MG_ERR_CAPACITY, "the workspace is smaller than mg_group_norm_workspace says");
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    if (mode == NORM_ROWS) {
        a.parts = params ? reinterpret_cast<float*>(ws) : nullptr;
        const RowLaunch l{p.vec, p.nv, p.cut, backward, p.grid, p.shape};
        MG_BY_TYPE(s->dtype, launch_rows<T>(l, a, st));
        ctx->launches++;
    } else if (mode == NORM_TILES) {
        a.fan_count = reinterpret_cast<uint32_t*>(ws + p.at_fan_count);
        a.sample_count = reinterpret_cast<uint32_t*>(ws + p.at_sample_count);
        a.tile_parts = reinterpret_cast<float*>(ws + p.at_tile_parts);
        a.fan_parts = reinterpret_cast<float*>(ws + p.at_fan_parts);
        a.group_parts = reinterpret_cast<float*>(ws + p.at_group_parts);
        a.parts = params ? reinterpret_cast<float*>(ws + p.at_parts) : nullptr;
        if (p.cleared) MG_CUDA(ctx, cudaMemsetAsync(ws, 0, p.cleared, st));
        bool empty = false;
        if (!a.equal) {
            int2* table = reinterpret_cast<int2*>(ws + p.at_table);
            TableArgs t;
            t.n = 0;
            int32_t tile = 0, first = 0;
            for (int32_t i = 0; i <= a.samples; ++i) {
                const int2 e = make_int2((int)s->sample_offsets[i], tile);
                if (i < a.samples) empty = empty || s->sample_offsets[i + 1] == s->sample_offsets[i];
                if (i < a.samples) tile += (int32_t)((s->sample_offsets[i + 1] - s->sample_offsets[i] + a.tile_rows - 1) / a.tile_rows);
                if (a.samples <= kInlineSamples) { a.inl[i] = e; continue; }
                t.at[t.n++] = e;
                if (t.n == kSamplesPerLaunch || i == a.samples) {
                    k_norm_table<<<1, 256, 0, st>>>(t, table + first);
                    ctx->launches++;
                    first += t.n; t.n = 0;
                }
            }
            if (a.samples > kInlineSamples) a.table = table;
        }
        if (empty && !backward && !p.block_grid) {
            k_norm_empty<<<std::min(a.samples, ctx->n_sms), 256, 0, st>>>(a);
            ctx->launches++;
        }
        if (a.tiles > 0 || p.block_grid) {
            const TileLaunch l{p.vec, p.sums_vec, backward, p.block_grid, p.cluster};
            MG_BY_TYPE(s->dtype, launch_tiles<T>(l, a, st));
            ctx->launches += p.block_grid ? 1 : 2;
        }
    }
    if (backward && params) {
        const int64_t columns = 2 * (int64_t)s->channels;
        const unsigned blocks = (unsigned)((columns + 31) / 32);
        const float* parts = a.parts;
        int64_t n = p.n_parts;
        if (n > kParamParts) {
            float* slices = reinterpret_cast<float*>(ws + p.at_slices);
            launch_chained(dim3(blocks, (unsigned)kParamSlices), kParamThreads, st, k_norm_params, parts, n, columns, slices, (float*)nullptr, (float*)nullptr);
            ctx->launches++;
            parts = slices; n = kParamSlices;
        }
        launch_chained(dim3(blocks), kParamThreads, st, k_norm_params, parts, n, columns, (float*)nullptr, d_weight, d_bias);
        ctx->launches++;
    }
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
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
    const Matrix m[2] = {{"x", x, x_stride, false}, {"y", y, y_stride, true}};
    const int vec = vec_width(m, 2, dtype, rows, channels);
    // Vectors to a thread at a time; narrower ones in pieces of 32 lanes, 8 / vec of them to a warp.  Blocks of fp32 vectors, bound by the memory, do one turn
    // and make room for the next: 543,000 rows of 256 took 179 us in eight blocks to an SM, 162 so.  What computes for longer makes several turns of its
    // blocks' first divisions: 150,001 fp16 rows of 768 93 us in one turn, 87 so.
    const bool wide = vec == 8, f32 = dtype == MG_DTYPE_F32;
    const int64_t per_block = wide ? (f32 ? 2 : 4) * kNormThreads : (int64_t)kNormWarps * (8 / vec), items = wide ? rows * (channels / vec) : rows * ((channels + 32 * vec - 1) / (32 * vec));
    const int64_t blocks = (items + per_block - 1) / per_block;
    MG_BY_TYPE(dtype, launch_dropout<T>(vec, x, x_stride, y, y_stride, rows, channels, d, (int)std::min<int64_t>(blocks, mg_grid(ctx, wide ? (f32 ? 128 : 16) : 10)), (cudaStream_t)stream));
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

extern "C" int mg_group_norm_workspace(mg_ctx* ctx, const mg_norm_spec* spec, int backward, size_t* bytes) {
    if (!ctx) return MG_ERR_ARG;
    if (!bytes) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    if (int rc = check_norm(ctx, spec)) return rc;
    *bytes = call_workspace(spec, ctx->n_sms, backward != 0);
    return MG_OK;
}

extern "C" int mg_group_norm(mg_ctx* ctx, const mg_norm_spec* spec, const void* x, int64_t x_stride, void* y, int64_t y_stride, float* mean, float* rstd,
                             void* workspace, size_t workspace_bytes, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    DropArgs drop;
    if (int rc = check_norm_call(ctx, spec, x, x_stride, nullptr, 0, false, y, y_stride, mean, rstd, workspace, &drop)) return rc;
    const Matrix m[2] = {{"x", x, x_stride, false}, {"y", y, y_stride, true}};
    return run_norm(ctx, spec, m, 2, false, mean, rstd, nullptr, nullptr, drop, workspace, workspace_bytes, (cudaStream_t)stream);
}

extern "C" int mg_group_norm_backward(mg_ctx* ctx, const mg_norm_spec* spec, const void* x, int64_t x_stride, const void* d_y, int64_t d_y_stride,
                                      const float* mean, const float* rstd, void* d_x, int64_t d_x_stride, float* d_weight, float* d_bias,
                                      void* workspace, size_t workspace_bytes, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    DropArgs drop;
    if (int rc = check_norm_call(ctx, spec, x, x_stride, d_y, d_y_stride, true, d_x, d_x_stride, mean, rstd, workspace, &drop, d_weight, d_bias)) return rc;
    const Matrix m[3] = {{"x", x, x_stride, false}, {"d_y", d_y, d_y_stride, false}, {"d_x", d_x, d_x_stride, true}};
    return run_norm(ctx, spec, m, 3, true, const_cast<float*>(mean), const_cast<float*>(rstd), d_weight, d_bias, drop, workspace, workspace_bytes, (cudaStream_t)stream);
}
