// Rows by id: the lookup with its scale, the places of equal ids brought together by a radix sort, the gradient summed up by them.
#include "mg_norm.cuh"
#include "mg_rows_plan.cuh"

namespace {

constexpr int kRowThreads = 256;

__device__ __forceinline__ int64_t id_at(const void* ids, int is_i64, int64_t i) {
    return is_i64 ? static_cast<const int64_t*>(ids)[i] : (int64_t)static_cast<const int32_t*>(ids)[i];
}

template <typename T> __device__ __forceinline__ float to_float(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// a warp to a row
template <typename T, typename O>
__global__ void k_embedding(const T* table, int64_t table_stride, int64_t n_rows, int32_t dim, const void* ids, int ids_are_i64, int64_t n, float scale, O* y, int64_t y_stride) {
    const int lane = threadIdx.x & 31;
    for (int64_t i = (int64_t)blockIdx.x * (kRowThreads / 32) + threadIdx.x / 32; i < n; i += (int64_t)gridDim.x * (kRowThreads / 32)) {
        const int64_t id = id_at(ids, ids_are_i64, i);
        const bool row = id >= 0 && id < n_rows;
        for (int32_t c = lane; c < dim; c += 32) y[i * y_stride + c] = row ? from_float<O>(scale * to_float(table[id * table_stride + c])) : from_float<O>(0.f);
    }
}

// ---- groups of equal ids ---------------------------------------------------------------------------------------------

__global__ void k_id_keys(const void* ids, int ids_are_i64, int64_t n, int64_t n_rows, uint32_t* keys, int32_t* order) {
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t id = id_at(ids, ids_are_i64, i);
        keys[i] = id >= 0 && id < n_rows ? (uint32_t)id : (uint32_t)n_rows;
        order[i] = (int32_t)i;
    }
}

// how many of each digit a tile has, digit after digit
__global__ void __launch_bounds__(kSortThreads) k_sort_count(const uint32_t* keys, int64_t n, int shift, int64_t tiles, uint32_t* hist) {
    __shared__ uint32_t sh[kSortBins];
    sh[threadIdx.x] = 0;
    __syncthreads();
    const int64_t lo = (int64_t)blockIdx.x * kSortTile, hi = min(lo + kSortTile, n);
    for (int64_t i = lo + threadIdx.x; i < hi; i += kSortThreads) atomicAdd(&sh[keys[i] >> shift & (kSortBins - 1)], 1u);
    __syncthreads();
    hist[threadIdx.x * tiles + blockIdx.x] = sh[threadIdx.x];
}

// what stands before each entry; by one block
__global__ void __launch_bounds__(1024) k_sort_scan(uint32_t* v, int64_t n) {
    __shared__ uint32_t warps[32];
    uint32_t before = 0;
    for (int64_t lo = 0; lo < n; lo += 1024) {
        const int64_t i = lo + threadIdx.x;
        const uint32_t own = i < n ? v[i] : 0u, inc = warp_incl_scan(own);
        if ((threadIdx.x & 31) == 31) warps[threadIdx.x / 32] = inc;
        __syncthreads();
        uint32_t at = before + inc - own, total = 0;
        for (int w = 0; w < 32; ++w) {
            if (w < (int)threadIdx.x / 32) at += warps[w];
            total += warps[w];
        }
        if (i < n) v[i] = at;
        before += total;
        __syncthreads();
    }
}

// a tile's keys to their places, equal digits in the order in which they stand: 32 at a time, by one warp after the other
__global__ void __launch_bounds__(kSortThreads) k_sort_place(const uint32_t* keys, const int32_t* order, int64_t n, int shift, int64_t tiles, const uint32_t* hist, uint32_t* keys_to, int32_t* order_to) {
    __shared__ uint32_t at[kSortBins];
    at[threadIdx.x] = hist[threadIdx.x * tiles + blockIdx.x];
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const int64_t lo = (int64_t)blockIdx.x * kSortTile, hi = min(lo + kSortTile, n);
    if (threadIdx.x >= 32) return;
    for (int64_t j = lo; j < hi; j += 32) {
        const bool ok = j + lane < hi;
        const uint32_t key = ok ? keys[j + lane] : 0u, digit = ok ? key >> shift & (kSortBins - 1) : kSortBins;
        const uint32_t peers = __match_any_sync(0xFFFFFFFFu, digit);
        if (ok) {
            const uint32_t to = at[digit] + __popc(peers & ((1u << lane) - 1u));
            keys_to[to] = key;
            order_to[to] = order[j + lane];
        }
        __syncwarp();
        if (ok && lane == __ffs(peers) - 1) at[digit] += __popc(peers);
        __syncwarp();
    }
}

__device__ __forceinline__ bool is_head(const uint32_t* keys, int64_t i, uint32_t none) { return keys[i] != none && (i == 0 || keys[i - 1] != keys[i]); }

__global__ void __launch_bounds__(kSortThreads) k_group_count(const uint32_t* keys, int64_t n, uint32_t none, uint32_t* heads) {
    const int64_t lo = (int64_t)blockIdx.x * kSortTile, hi = min(lo + kSortTile, n);
    __shared__ uint32_t total;
    if (threadIdx.x == 0) total = 0;
    __syncthreads();
    uint32_t mine = 0;
    for (int64_t i = lo + threadIdx.x; i < hi; i += kSortThreads) mine += is_head(keys, i, none);
    atomicAdd(&total, mine);
    __syncthreads();
    if (threadIdx.x == 0) heads[blockIdx.x] = total;
}

__global__ void __launch_bounds__(kSortThreads) k_group_write(const uint32_t* keys, int64_t n, uint32_t none, const uint32_t* heads, int ids_are_i64, void* group_ids, int32_t* starts, int32_t* n_groups) {
    __shared__ uint32_t warps[kSortThreads / 32];
    const int64_t lo = (int64_t)blockIdx.x * kSortTile, hi = min(lo + kSortTile, n);
    uint32_t before = n > 0 ? heads[blockIdx.x] : 0u;
    for (int64_t j = lo; j < hi; j += kSortThreads) {
        const int64_t i = j + threadIdx.x;
        const bool head = i < hi && is_head(keys, i, none);
        const uint32_t votes = __ballot_sync(0xFFFFFFFFu, head);
        if ((threadIdx.x & 31) == 0) warps[threadIdx.x / 32] = __popc(votes);
        __syncthreads();
        uint32_t g = before + __popc(votes & ((1u << (threadIdx.x & 31)) - 1u));
        for (int w = 0; w < kSortThreads / 32; ++w) {
            if (w < (int)threadIdx.x / 32) g += warps[w];
            before += warps[w];
        }
        if (head) {
            starts[g] = (int32_t)i;
            if (ids_are_i64) static_cast<int64_t*>(group_ids)[g] = keys[i];
            else static_cast<int32_t*>(group_ids)[g] = (int32_t)keys[i];
        }
        // the end of the last group: where the ids that are no rows begin, or behind all
        if (i < n && i < hi && keys[i] != none && (i + 1 == n || keys[i + 1] == none)) { starts[g + head] = (int32_t)i + 1; *n_groups = (int32_t)(g + head); }
        __syncthreads();
    }
    if (blockIdx.x == 0 && threadIdx.x == 0 && (n == 0 || keys[0] == none)) { starts[0] = 0; *n_groups = 0; }
}

// ---- sums by group ---------------------------------------------------------------------------------------------------

template <typename T>
__global__ void k_rows_zero(T* out, int64_t stride, int64_t rows, int32_t dim) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int32_t c = threadIdx.x; c < dim; c += blockDim.x) out[r * stride + c] = from_float<T>(0.f);
}

// a warp to a group
template <typename T, typename O>
__global__ void k_group_sums(const T* d_y, int64_t d_y_stride, int64_t n, int64_t n_rows, int32_t dim, float scale, const int32_t* order, const void* group_ids, int ids_are_i64,
                             const int32_t* starts, const int32_t* n_groups, int into, O* out, int64_t out_stride) {
    const int lane = threadIdx.x & 31;
    const int64_t groups = min((int64_t)*n_groups, min(n, n_rows));
    for (int64_t g = (int64_t)blockIdx.x * (kRowThreads / 32) + threadIdx.x / 32; g < groups; g += (int64_t)gridDim.x * (kRowThreads / 32)) {
        const int64_t id = id_at(group_ids, ids_are_i64, g), row = into == MG_ROWS_COMPACT ? g : id;
        if (id < 0 || id >= n_rows) continue;
        const int64_t lo = max(starts[g], 0), hi = min((int64_t)starts[g + 1], n);
        for (int32_t c = lane; c < dim; c += 32) {
            float part[3] = {0.f, 0.f, 0.f};   // of 64 places, of 64 of these, of all: no value goes through hundreds of additions
            for (int64_t i = lo; i < hi; ++i) {
                const int64_t at = order[i];
                if (at >= 0 && at < n) part[0] += to_float(d_y[at * d_y_stride + c]);
                if ((i - lo) % 64 == 63) { part[1] += part[0]; part[0] = 0.f; }
                if ((i - lo) % 4096 == 4095) { part[2] += part[1]; part[1] = 0.f; }
            }
            float s = (part[0] + part[1] + part[2]) * scale;
            O* to = out + row * out_stride + c;
            if (into == MG_ROWS_ADD) s += to_float(*to);
            *to = from_float<O>(s);
        }
    }
}

}  // namespace

extern "C" int mg_embedding(mg_ctx* ctx, const void* table, int64_t table_stride, int table_dtype, int64_t n_rows, int32_t dim, const void* ids, int ids_are_i64,
                            int64_t n, float scale, void* y, int64_t y_stride, int y_dtype, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_lookup(ctx, table, table_stride, table_dtype, n_rows, dim, ids, ids_are_i64, n, scale, y, y_stride, y_dtype)) return rc;
    if (n == 0) return MG_OK;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const int grid = (int)std::min<int64_t>((n + kRowThreads / 32 - 1) / (kRowThreads / 32), mg_grid(ctx, 8));
    MG_BY_TYPE(table_dtype, using From = T; MG_BY_TYPE(y_dtype, (k_embedding<From, T><<<grid, kRowThreads, 0, (cudaStream_t)stream>>>(static_cast<const From*>(table), table_stride, n_rows, dim, ids, ids_are_i64, n, scale, static_cast<T*>(y), y_stride))));
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

extern "C" int mg_id_groups_workspace(mg_ctx* ctx, int64_t n, int64_t n_rows, size_t* bytes) {
    if (!ctx) return MG_ERR_ARG;
    if (!bytes) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    static const int32_t some = 0;
    if (int rc = check_ids(ctx, &some, 0, n, n_rows)) return rc;
    *bytes = plan_groups(n, n_rows).bytes;
    return MG_OK;
}

extern "C" int mg_id_groups(mg_ctx* ctx, const void* ids, int ids_are_i64, int64_t n, int64_t n_rows, int32_t* order, void* group_ids, int32_t* starts,
                            int32_t* n_groups, void* workspace, size_t workspace_bytes, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_groups(ctx, ids, ids_are_i64, n, n_rows, order, group_ids, starts, n_groups, workspace, workspace_bytes)) return rc;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const cudaStream_t st = (cudaStream_t)stream;
    const GroupPlan p = plan_groups(n, n_rows);
    char* ws = static_cast<char*>(workspace);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(ws + p.at_keys[0]), reinterpret_cast<uint32_t*>(ws + p.at_keys[1])};
    int32_t* spare = reinterpret_cast<int32_t*>(ws + p.at_order);
    uint32_t *hist = reinterpret_cast<uint32_t*>(ws + p.at_hist), *heads = reinterpret_cast<uint32_t*>(ws + p.at_heads);
    const int tiles = (int)p.tiles;
    int at = 0;
    if (tiles) {
        // (the last pass ends in the caller's array)
        int32_t* by[2] = {p.passes % 2 ? spare : order, p.passes % 2 ? order : spare};
        k_id_keys<<<std::min(tiles * 16, mg_grid(ctx, 8)), 256, 0, st>>>(ids, ids_are_i64, n, n_rows, keys[0], by[0]);
        for (int pass = 0; pass < p.passes; ++pass, at ^= 1) {
            k_sort_count<<<tiles, kSortThreads, 0, st>>>(keys[at], n, pass * kSortBits, tiles, hist);
            k_sort_scan<<<1, 1024, 0, st>>>(hist, (int64_t)tiles * kSortBins);
            k_sort_place<<<tiles, kSortThreads, 0, st>>>(keys[at], by[at], n, pass * kSortBits, tiles, hist, keys[at ^ 1], by[at ^ 1]);
            ctx->launches += 3;
        }
        k_group_count<<<tiles, kSortThreads, 0, st>>>(keys[at], n, (uint32_t)n_rows, heads);
        k_sort_scan<<<1, 1024, 0, st>>>(heads, tiles);
        ctx->launches += 3;
    }
    k_group_write<<<std::max(tiles, 1), kSortThreads, 0, st>>>(keys[at], n, (uint32_t)n_rows, heads, ids_are_i64, group_ids, starts, n_groups);
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

extern "C" int mg_embedding_backward_workspace(mg_ctx* ctx, int64_t n, int64_t n_rows, int32_t dim, size_t* bytes) {
    if (!ctx) return MG_ERR_ARG;
    if (!bytes) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    static const int32_t some = 0;
    if (int rc = check_ids(ctx, &some, 0, n, n_rows)) return rc;
    if (dim < 1 || dim > 1 << 24) return mg_fail(ctx, MG_ERR_ARG, "the width of a row must be in [1, 2^24]");
    *bytes = sums_workspace(n, n_rows, dim);
    return MG_OK;
}

extern "C" int mg_embedding_backward(mg_ctx* ctx, const void* d_y, int64_t d_y_stride, int d_y_dtype, int64_t n, int64_t n_rows, int32_t dim, float scale,
                                     const int32_t* order, const void* group_ids, int ids_are_i64, const int32_t* starts, const int32_t* n_groups, int into,
                                     void* out, int64_t out_stride, int out_dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_sums(ctx, d_y, d_y_stride, d_y_dtype, n, n_rows, dim, scale, order, group_ids, ids_are_i64, starts, n_groups, into, out, out_stride, out_dtype, workspace, workspace_bytes)) return rc;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const cudaStream_t st = (cudaStream_t)stream;
    const int64_t most = std::min(n, n_rows);
    if (into == MG_ROWS_TABLE && n_rows > 0) {
        MG_BY_TYPE(out_dtype, (k_rows_zero<T><<<(int)std::min<int64_t>(n_rows, mg_grid(ctx, 8)), 256, 0, st>>>(static_cast<T*>(out), out_stride, n_rows, dim)));
        ctx->launches++;
    }
    if (most > 0) {
        const int grid = (int)std::min<int64_t>((most + kRowThreads / 32 - 1) / (kRowThreads / 32), mg_grid(ctx, 8));
        MG_BY_TYPE(d_y_dtype, using From = T; MG_BY_TYPE(out_dtype, (k_group_sums<From, T><<<grid, kRowThreads, 0, st>>>(static_cast<const From*>(d_y), d_y_stride, n, n_rows, dim, scale, order, group_ids, ids_are_i64, starts, n_groups, into, static_cast<T*>(out), out_stride))));
        ctx->launches++;
    }
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}
