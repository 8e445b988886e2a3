// Rows by id: the lookup with its scale, the places of equal ids brought together by a radix sort, the gradient summed up by them.
#include "mg_rows_plan.cuh"
#include "mg_rows_sums.cuh"

namespace {

using namespace mgrows;

constexpr int kRowThreads = 256;

// 543,000 fp32 rows of 128 out of two million: 90 us for 502 MB, 86 % of the copy's rate; the memory bounds it.  (A warp to a row: 157.)
// A warp to a tile of up to 32 looked-up rows: an id to each lane, then the rows' vectors numbered through, so that no lane is without one where a row's vectors are
// not a multiple of 32, U of them on their way.
struct LookupArgs {
    const void* table; int64_t table_stride, n_rows;
    const void* ids; int ids_are_i64;
    int64_t n; float scale;
    void* y; int64_t y_stride;
    int32_t vecs, rows;       // vectors to a row, rows to a tile
    uint32_t reciprocal;      // of vecs (two or more), in units of 2^-32, rounded up: t / vecs = t reciprocal / 2^32 for t < rows vecs
};
template <typename T, typename O, int VEC, int U>
__global__ void __launch_bounds__(kRowThreads) k_embedding(const __grid_constant__ LookupArgs a) {
    const int lane = threadIdx.x & 31;
    const int64_t base = ((int64_t)blockIdx.x * (kRowThreads / 32) + threadIdx.x / 32) * a.rows;
    if (base >= a.n) return;
    const int rows = (int)min((int64_t)a.rows, a.n - base);
    int64_t id = -1;
    if (lane < rows) id = id_at(a.ids, a.ids_are_i64, base + lane);
    const int32_t own = id >= 0 && id < a.n_rows ? (int32_t)id : -1;
    const int32_t items = rows * a.vecs;
    for (int32_t t0 = 0; t0 < items; t0 += 32 * U) {
        Raw<T, VEC> raw[U];
        int32_t row[U], vec[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t t = t0 + u * 32 + lane;
            row[u] = a.rows == 1 ? 0 : a.vecs == 1 ? t : (int32_t)__umulhi((uint32_t)t, a.reciprocal);
            vec[u] = t - row[u] * a.vecs;
            const int32_t from = __shfl_sync(0xFFFFFFFFu, own, row[u] & 31);
            if (t < items && from >= 0) raw[u].load(static_cast<const T*>(a.table) + from * a.table_stride + (int64_t)vec[u] * VEC);
            else raw[u].zero();
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t0 + u * 32 + lane < items) {
                float f[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = raw[u].get(e) * a.scale;
                Raw<O, VEC> out;
                out.put(f);
                out.store(static_cast<O*>(a.y) + (base + row[u]) * a.y_stride + (int64_t)vec[u] * VEC);
            }
    }
}

constexpr int kSortPolls = 1 << 20;   // (a poll is an L2 round trip: far beyond any legitimate wait)

template <int PER>
void launch_sort(mg_ctx* ctx, const GroupPlan& p, const void* ids, int ids_are_i64, int64_t n, int64_t n_rows, int32_t* order, int32_t* group_of, void* group_ids, int32_t* starts,
                 int32_t* n_groups, char* ws, cudaStream_t st) {
    const uint32_t none = (uint32_t)n_rows;
    SortShared* s = reinterpret_cast<SortShared*>(ws);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(ws + p.at_keys[0]), reinterpret_cast<uint32_t*>(ws + p.at_keys[1])};
    int32_t* spare = reinterpret_cast<int32_t*>(ws + p.at_order);
    const unsigned tiles = (unsigned)p.tiles;
    int at = 0;
    k_sort_hist<<<(unsigned)std::min<int64_t>((n + kSortThreads - 1) / kSortThreads, mg_grid(ctx, 4)), kSortThreads, 0, st>>>(ids, ids_are_i64, n, none, p.passes, p.bits, s);
    // (the last pass ends in the caller's array)
    int32_t* by[2] = {p.passes % 2 ? spare : order, p.passes % 2 ? order : spare};
    for (int pass = 0; pass < p.passes; ++pass, at ^= 1) {
        uint64_t* states = reinterpret_cast<uint64_t*>(ws + p.at_states) + (size_t)pass * p.tiles * kSortBins;
        mgnorm::launch_chained(dim3(tiles), kSortThreads, st, pass ? k_sort_pass<PER, false> : k_sort_pass<PER, true>, ids, ids_are_i64, (const uint32_t*)keys[at], (const int32_t*)by[at], n, none, pass,
                               p.bits, s, states, keys[at ^ 1], by[at ^ 1], kSortPolls);
    }
    // (few tiles, since each waits for those before: 543,000 ids 55 -> 52 us)
    constexpr int kGroupPer = PER == 4 ? 4 : 16;
    mgnorm::launch_chained(dim3((unsigned)((n + kSortThreads * kGroupPer - 1) / (kSortThreads * kGroupPer))), kSortThreads, st, k_sort_groups<kGroupPer>, (const uint32_t*)keys[at], n, none, s, reinterpret_cast<uint64_t*>(ws + p.at_chain), ids_are_i64, group_ids, starts, group_of,
                           n_groups, kSortPolls);
    ctx->launches += 2 + p.passes;
}

int pow2_up(int64_t v) { int p = 1; while (p < v) p *= 2; return p; }

// Elements to an access: as many as make 16 bytes (8 where types of two and four bytes meet), or half or a quarter of that, as the rows' width and where they begin allow.
// (500,000 bf16 rows of 100 of a million by 8 bytes 51 us, one element at a time 112; their gradient 194 and 331.)
int row_vec(const void* a, int64_t a_stride, int a_dtype, int64_t a_rows, const void* b, int64_t b_stride, int b_dtype, int64_t b_rows, int32_t dim) {
    int vec = a_dtype != MG_DTYPE_F32 && b_dtype != MG_DTYPE_F32 ? 8 : 4;
    const auto fits = [&](const void* p, int64_t stride, int dtype, int64_t rows) {
        return reinterpret_cast<uintptr_t>(p) % (uintptr_t)(vec * elem_size(dtype)) == 0 && (rows <= 1 || stride % vec == 0);
    };
    while (vec > 1 && !(dim % vec == 0 && fits(a, a_stride, a_dtype, a_rows) && fits(b, b_stride, b_dtype, b_rows))) vec /= 2;
    return vec;
}

template <typename T, typename O>
void launch_lookup(const LookupArgs& a, int vec, unsigned grid, cudaStream_t st) {
    if constexpr (sizeof(T) == 2 && sizeof(O) == 2)
        if (vec == 8) { k_embedding<T, O, 8, 4><<<grid, kRowThreads, 0, st>>>(a); return; }
    if (vec == 4) k_embedding<T, O, 4, 4><<<grid, kRowThreads, 0, st>>>(a);
    else if (vec == 2) k_embedding<T, O, 2, 8><<<grid, kRowThreads, 0, st>>>(a);
    else k_embedding<T, O, 1, 8><<<grid, kRowThreads, 0, st>>>(a);
}

template <typename T, typename O>
void launch_sums(SumArgs a, int vec, int64_t zero_blocks, cudaStream_t st) {
    const int each = std::max(vec, 4), lanes = std::min(32, std::max(4, pow2_up((a.dim + each - 1) / each))), columns = lanes * each;   // (columns to a lane)
    a.chunk_blocks = (int32_t)(((int64_t)a.chunks * lanes + kSumThreads - 1) / kSumThreads);
    const dim3 grid((unsigned)(a.chunk_blocks + zero_blocks), (unsigned)((a.dim + columns - 1) / columns));
    const auto go = [&](auto kernel, auto of_long) { mgnorm::launch_chained(grid, kSumThreads, st, a.chunk > kSumChain ? of_long : kernel, a, lanes); };
    if constexpr (sizeof(T) == 2 && sizeof(O) == 2)
        if (vec == 8) { go(k_chunk_sums<T, O, 8, 1, 4, false>, k_chunk_sums<T, O, 8, 1, 4, true>); return; }
    if (vec == 4) go(k_chunk_sums<T, O, 4, 1, 4, false>, k_chunk_sums<T, O, 4, 1, 4, true>);
    else if (vec == 2) go(k_chunk_sums<T, O, 2, 2, 4, false>, k_chunk_sums<T, O, 2, 2, 4, true>);
    else go(k_chunk_sums<T, O, 1, 4, 2, false>, k_chunk_sums<T, O, 1, 4, 2, true>);
}

}  // namespace

extern "C" int mg_embedding(mg_ctx* ctx, const void* table, int64_t table_stride, int table_dtype, int64_t n_rows, int32_t dim, const void* ids, int ids_are_i64,
                            int64_t n, float scale, void* y, int64_t y_stride, int y_dtype, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_lookup(ctx, table, table_stride, table_dtype, n_rows, dim, ids, ids_are_i64, n, scale, y, y_stride, y_dtype)) return rc;
    if (n == 0) return MG_OK;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const int vec = row_vec(table, table_stride, table_dtype, n_rows, y, y_stride, y_dtype, n, dim);
    LookupArgs a{table, table_stride, n_rows, ids, ids_are_i64, n, scale, y, y_stride, dim / vec, 32, 0};
    // rows to a tile: as few as give every multiprocessor 32 warps, and one where the rows' vectors could not be told apart by a product (or are many anyway)
    while (a.rows > 1 && (a.vecs > 1024 || n < (int64_t)ctx->n_sms * 32 * a.rows)) a.rows /= 2;
    a.reciprocal = (uint32_t)((1ull << 32) / (uint64_t)a.vecs + 1);
    const unsigned grid = (unsigned)((n + (int64_t)a.rows * (kRowThreads / 32) - 1) / ((int64_t)a.rows * (kRowThreads / 32)));
    MG_BY_TYPE(table_dtype, using From = T; MG_BY_TYPE(y_dtype, (launch_lookup<From, T>(a, vec, grid, (cudaStream_t)stream))));
    ctx->launches++;
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

extern "C" int mg_id_groups_workspace(mg_ctx* ctx, int64_t n, int64_t n_rows, size_t* bytes) {
    if (!ctx) return MG_ERR_ARG;
    if (!bytes) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    static const int32_t some = 0;
    if (int rc = check_ids(ctx, &some, 0, n, n_rows)) return rc;
    *bytes = plan_groups(n, n_rows, ctx->n_sms).bytes;
    return MG_OK;
}

extern "C" int mg_id_groups(mg_ctx* ctx, const void* ids, int ids_are_i64, int64_t n, int64_t n_rows, int32_t* order, int32_t* group_of, void* group_ids,
                            int32_t* starts, int32_t* n_groups, void* workspace, size_t workspace_bytes, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_groups(ctx, ids, ids_are_i64, n, n_rows, order, group_of, group_ids, starts, n_groups, workspace, workspace_bytes)) return rc;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const cudaStream_t st = (cudaStream_t)stream;
    const GroupPlan p = plan_groups(n, n_rows, ctx->n_sms);
    if (!p.passes) {
        k_sort_small<<<1, kSmallIds, 0, st>>>(ids, ids_are_i64, (int32_t)n, (uint32_t)n_rows, order, group_of, group_ids, starts, n_groups);
        ctx->launches++;
        MG_CUDA(ctx, cudaGetLastError());
        return MG_OK;
    }
    char* ws = static_cast<char*>(workspace);
    MG_CUDA(ctx, cudaMemsetAsync(ws, 0, p.cleared, st));
    (p.per == 4 ? launch_sort<4> : launch_sort<8>)(ctx, p, ids, ids_are_i64, n, n_rows, order, group_of, group_ids, starts, n_groups, ws, st);
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}

extern "C" int mg_embedding_backward_workspace(mg_ctx* ctx, int64_t n, int64_t n_rows, int32_t dim, size_t* bytes) {
    if (!ctx) return MG_ERR_ARG;
    if (!bytes) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    static const int32_t some = 0;
    if (int rc = check_ids(ctx, &some, 0, n, n_rows)) return rc;
    if (dim < 1 || dim > 1 << 22) return mg_fail(ctx, MG_ERR_ARG, "the width of a row must be in [1, 2^22]");
    *bytes = sums_workspace(n, n_rows, dim, ctx->n_sms);
    return MG_OK;
}

extern "C" int mg_embedding_backward(mg_ctx* ctx, const void* d_y, int64_t d_y_stride, int d_y_dtype, int64_t n, int64_t n_rows, int32_t dim, float scale,
                                     const int32_t* order, const int32_t* group_of, const void* group_ids, int ids_are_i64, const int32_t* starts,
                                     const int32_t* n_groups, int into, void* out, int64_t out_stride, int out_dtype, void* workspace, size_t workspace_bytes, void* stream) {
    if (!ctx) return MG_ERR_ARG;
    if (int rc = check_sums(ctx, d_y, d_y_stride, d_y_dtype, n, n_rows, dim, scale, order, group_of, group_ids, ids_are_i64, starts, n_groups, into, out, out_stride, out_dtype, workspace, workspace_bytes)) return rc;
    DeviceScope on(ctx->device);
    MG_CUDA(ctx, on.err);
    const cudaStream_t st = (cudaStream_t)stream;
    const SumPlan p = plan_sums(n, n_rows, dim, ctx->n_sms);
    char* ws = static_cast<char*>(workspace);
    // (rows to a block that writes zeros: 128 KB of them, fewer where blocks would be fewer than four to a multiprocessor, 32 at least)
    const int64_t much = (128 << 10) / ((int64_t)dim * elem_size(out_dtype)), few = (n_rows + mg_grid(ctx, 4) - 1) / mg_grid(ctx, 4);
    const int zero_rows = (int)std::min<int64_t>(std::max<int64_t>(std::min(much, few), 32) / 32 * 32, kMostZeroRows);
    const SumArgs a{d_y, d_y_stride, n, n_rows, dim, scale, order, group_of, starts, n_groups, group_ids, ids_are_i64, into, out, out_stride, p.chunk, p.chunks,
                    reinterpret_cast<float*>(ws), p.pitch, reinterpret_cast<int32_t*>(ws + p.at_begun), 0, zero_rows,
                    row_vec(out, out_stride, out_dtype, n_rows, out, out_stride, out_dtype, n_rows, dim)};
    int64_t zero_blocks = into == MG_ROWS_TABLE ? (n_rows + zero_rows - 1) / zero_rows : 0;
    if (zero_blocks && (!p.chunks || n_rows * dim * elem_size(out_dtype) > 32ll << 20)) {
        MG_BY_TYPE(out_dtype, mgnorm::launch_chained(dim3((unsigned)zero_blocks), kSumThreads, st, k_zero_others<T>, a));
        ctx->launches++;
        zero_blocks = 0;
    }
    if (p.chunks > 0) {
        const int vec = row_vec(d_y, d_y_stride, d_y_dtype, n, out, out_stride, out_dtype, n_rows, dim);
        MG_BY_TYPE(d_y_dtype, using From = T; MG_BY_TYPE(out_dtype, (launch_sums<From, T>(a, vec, zero_blocks, st))));
        MG_BY_TYPE(out_dtype, mgnorm::launch_chained(dim3((unsigned)std::min(p.chunks, mg_grid(ctx, 1)), (unsigned)((dim + 127) / 128)), kJoinThreads, st, k_join_shares<T>, a));
        ctx->launches += 2;
    }
    MG_CUDA(ctx, cudaGetLastError());
    return MG_OK;
}
