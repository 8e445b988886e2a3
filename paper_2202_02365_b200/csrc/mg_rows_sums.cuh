// The gradient of looked-up rows: sums over the places of each id, in an order that goes by the places alone.
//
// The sorted places are cut into chunks.  A part of a warp goes along a chunk's places, adds up rows and writes a sum where the id changes; an id that begins in the chunk and
// ends no more than a chunk's length on is followed to its end, so that most ids are summed up in one go.  Of an id with more places than a chunk has, every chunk leaves
// its share in the workspace, and a second kernel adds the shares up.  No float is added atomically.  543,000 fp32 rows of 128 into 433,750: 100 us for 504 MB, 5.0 TB/s, the shares 7; bound by
// the latency of rows that lie anywhere, with 24 warps to an SM that have four to eight rows each on their way.
#pragma once

#include "mg_norm.cuh"
#include "mg_rows_sort.cuh"

namespace mgrows {

constexpr int kSumThreads = 256, kJoinThreads = 1024;
// Places whose rows are added up in fp32 one behind the other; the sums of so many each are added up in 64 bits.  With 256 shares to a warp and 32 warps, no value goes through more than
// 480 additions in fp32, however many places an id has.  (A multiple of every number of lanes.)
constexpr int kSumChain = 192;

struct SumArgs {
    const void* d_y; int64_t d_y_stride, n, n_rows;
    int32_t dim; float scale;
    const int32_t *order, *group_of, *starts, *n_groups; const void* group_ids; int ids_are_i64;
    int into;
    void* out; int64_t out_stride;
    int32_t chunk, chunks;        // places to a chunk
    float* shares; int32_t pitch; // [chunks][2][pitch]: of the id that the chunk begins within, of the one that goes on behind it
    int32_t* begun;               // [chunks]: the group that begins in the chunk and has shares, -1
    int32_t chunk_blocks, zero_rows;   // blocks of the sums; rows to a block of those that write zeros
    int32_t zero_vec;             // ... elements at a time
};

template <typename O, int VEC>
__device__ __forceinline__ void write_sum(const SumArgs& a, int64_t row, int32_t c, float (&s)[VEC]) {
    O* to = static_cast<O*>(a.out) + row * a.out_stride + c;
    Raw<O, VEC> raw;
    if (a.into == MG_ROWS_ADD) {
        raw.load(to);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[e] = fmaf(s[e], a.scale, raw.get(e));
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[e] *= a.scale;
    }
    raw.put(s);
    raw.store(to);
}

// Zeros into the rows of the table that no id names: a block finds the named ones among its rows, marks them in shared memory and writes the others.  Tables of up to 32 MB by blocks
// behind those of the sums, in one launch (14,824 rows of 100: 49 us, by a kernel of its own 53); larger ones by the kernel of its own, of which an SM holds more blocks
// (300,007 bf16 rows of 768: 199 us, with the sums 217).
constexpr int kMostZeroRows = 2048;
template <typename O>
__device__ __forceinline__ void zero_others(const SumArgs& a, int64_t block) {
    __shared__ uint32_t named[kMostZeroRows / 32];
    __shared__ int64_t sh_first;
    const int64_t r0 = block * a.zero_rows, r1 = min(r0 + a.zero_rows, a.n_rows);
    const int64_t groups = max((int64_t)0, min((int64_t)*a.n_groups, min(a.n, a.n_rows)));
    if (threadIdx.x < kMostZeroRows / 32) named[threadIdx.x] = 0;
    if (threadIdx.x < 32) {
        // the first group whose id is r0 or more, 32 probes at a time
        int64_t lo = 0, hi = groups;
        while (lo < hi) {
            const int64_t step = (hi - lo + 31) / 32, at = lo + step * threadIdx.x;
            const uint32_t below = __ballot_sync(0xFFFFFFFFu, at < hi && id_at(a.group_ids, a.ids_are_i64, at) < r0);
            const int k = __popc(below);   // the probes up to it lie below
            hi = min(hi, k < 32 ? lo + step * k : hi);
            lo = k ? lo + step * (k - 1) + 1 : lo;
            if (k == 0) hi = lo;
        }
        if (threadIdx.x == 0) sh_first = lo;
    }
    __syncthreads();
    for (int64_t g = sh_first + threadIdx.x; g < min(groups, sh_first + a.zero_rows); g += kSumThreads) {
        const int64_t id = id_at(a.group_ids, a.ids_are_i64, g);
        if (id >= r0 && id < r1) atomicOr(&named[(id - r0) >> 5], 1u << ((id - r0) & 31));
    }
    __syncthreads();
    const auto write = [&](auto zero, int width) {
        zero.zero();
        const int vecs = a.dim / width, lanes = min(kSumThreads, 1 << (31 - __clz(vecs)));
        const int sub = (int)threadIdx.x & (lanes - 1);
        for (int64_t r = r0 + threadIdx.x / lanes; r < r1; r += kSumThreads / lanes) {
            if (named[(r - r0) >> 5] >> ((r - r0) & 31) & 1) continue;
            O* to = static_cast<O*>(a.out) + r * a.out_stride;
            for (int v = sub; v < vecs; v += lanes) zero.store(to + v * width);
        }
    };
    constexpr int VEC = 16 / sizeof(O);
    if (a.zero_vec == VEC) write(Raw<O, VEC>(), VEC);
    else if (a.zero_vec == VEC / 2) write(Raw<O, VEC / 2>(), VEC / 2);
    else write(Raw<O, 1>(), 1);
}

template <typename O>
__global__ void __launch_bounds__(kSumThreads) k_zero_others(const __grid_constant__ SumArgs a) {
    chain_wait();
    chain_start();
    zero_others<O>(a, blockIdx.x);
}

// `lanes` lanes to a chunk, NV vectors of its rows to a lane, U rows on their way while U others are added up; blockIdx.y: which of the rows' columns.
// What a chunk has to know of its neighbours is asked for beside its first places, and of its first and last ids beside its first rows.
// LONG: chunks of more than kSumChain places, which few calls have (more than some 1.4 million ids, or of 1.4 GB in fp32): a million bf16 rows of 1,024 434 us, without 419, and the others
// would lose as much.
template <typename T, typename O, int VEC, int NV, int U, bool LONG>
__global__ void __launch_bounds__(kSumThreads, 3) k_chunk_sums(const __grid_constant__ SumArgs a, int lanes) {
    chain_wait();
    chain_start();
    if ((int32_t)blockIdx.x >= a.chunk_blocks) {
        if (blockIdx.y == 0) zero_others<O>(a, (int64_t)blockIdx.x - a.chunk_blocks);
        return;
    }
    const int sub = (int)threadIdx.x & (lanes - 1);
    const int32_t chunk = (int32_t)((blockIdx.x * (int64_t)kSumThreads + threadIdx.x) / lanes);
    const int32_t c0 = ((int32_t)blockIdx.y * NV * lanes + sub) * VEC, step = lanes * VEC;
    const uint32_t peers = lanes == 32 ? 0xFFFFFFFFu : ((1u << lanes) - 1u) << ((int)(threadIdx.x & 31) & ~(lanes - 1));
    if (chunk >= a.chunks) return;
    const int64_t lo = (int64_t)chunk * a.chunk, hi = min(lo + a.chunk, a.n);
    const int32_t groups = *a.n_groups;
    const bool some = groups > 0 && groups <= min(a.n, a.n_rows);
    const auto group_at = [&](int64_t i) { return min(max(a.group_of[i], -1), groups - 1); };
    int32_t place = -1, group = -1, next_place = -1, next_group = -1;   // of the lane, in this batch of `lanes` places and the next
    int32_t first = -1, came = -1, last = -1;                            // groups: of the first place, of the one before, of the last
    if (some) {
        if (lo + sub < a.n) { place = a.order[lo + sub]; group = group_at(lo + sub); }
        first = group_at(lo); last = group_at(hi - 1);
        if (lo > 0) came = group_at(lo - 1);
    }
    const uint32_t from_stride = (uint32_t)(a.d_y_stride * (int64_t)sizeof(T));   // (below 2^31)
    const auto load = [&](Raw<T, VEC> (&raw)[U][NV], int32_t of, int at) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t i = __shfl_sync(peers, of, (at + u) & (lanes - 1), lanes);
            const T* const row = reinterpret_cast<const T*>(static_cast<const char*>(a.d_y) + (uint64_t)(uint32_t)i * from_stride) + c0;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if ((uint32_t)i < (uint32_t)a.n && c0 + v * step < a.dim) raw[u][v].load(row + v * step);
                else raw[u][v].zero();
            }
        }
    };
    Raw<T, VEC> one[U][NV], two[U][NV];
    load(one, place, 0);
    // an id that began before the chunk and is no longer than one is left to whom it began with; one that begins here, to its end; longer ones leave a share
    int32_t before = -1, behind = -1, skip = -1;
    int64_t end = hi;
    if (first >= 0 && came == first) {
        if (a.starts[first + 1] - a.starts[first] > a.chunk) before = first;
        else skip = first;
    }
    if (last >= 0 && last != before && last != skip) {
        const int64_t until = min((int64_t)a.starts[last + 1], a.n);
        if (until - a.starts[last] > a.chunk) { if (until > hi) behind = last; }
        else end = max(until, hi);
    }
    if (!some) end = lo;
    if (sub == 0 && blockIdx.y == 0) a.begun[chunk] = behind;
    float acc[NV][VEC];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[v][e] = 0.f;
    __shared__ double put_away[LONG ? NV * VEC : 1][LONG ? kSumThreads : 1];   // the sum of an id's places up to the last kSumChain
    bool has_put = false;
    const auto put = [&]() {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                double& to = put_away[v * VEC + e][threadIdx.x];
                to = (has_put ? to : 0.) + (double)acc[v][e];
                acc[v][e] = 0.f;
            }
        has_put = true;
    };
    int32_t cur = -1, cur_row = -1;
    const auto flush = [&]() {
        if (LONG && has_put) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[v][e] = (float)(put_away[v * VEC + e][threadIdx.x] + (double)acc[v][e]);
            has_put = false;
        }
        if (cur >= 0 && cur != skip) {
            const bool share = cur == before || cur == behind;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int32_t c = c0 + v * step;
                if (c >= a.dim) continue;
                if (share) {
                    float* to = a.shares + ((int64_t)chunk * 2 + (cur == behind)) * a.pitch + c;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) to[e] = acc[v][e];
                } else if (cur_row >= 0) write_sum<O, VEC>(a, cur_row, c, acc[v]);
            }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < VEC; ++e) acc[v][e] = 0.f;
    };
    const auto row_of = [&](int32_t g) -> int32_t {
        const int64_t row = g < 0 ? -1 : a.into == MG_ROWS_COMPACT ? g : id_at(a.group_ids, a.ids_are_i64, g);
        return row < a.n_rows ? (int32_t)row : -1;
    };
    int32_t row = row_of(group);
    const auto ask = [&](int64_t p) {   // for a batch's places
        next_place = next_group = -1;
        if (p + sub < end) { next_place = a.order[p + sub]; next_group = group_at(p + sub); }
    };
    ask(lo + lanes);
    const auto add = [&](const Raw<T, VEC> (&raw)[U][NV], int left, int at) {   // the batch's places at .., as far as they are among its first `left`
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t g = __shfl_sync(peers, group, (at + u) & (lanes - 1), lanes);
            if (at + u < left) {
                if (g != cur) {
                    flush();
                    cur = g;
                    cur_row = __shfl_sync(peers, row, (at + u) & (lanes - 1), lanes);
                }
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[v][e] += raw[u][v].get(e);
            }
        }
    };
    // (a batch is a multiple of 2 U places, or these are all of it)
    for (int64_t p = lo; p < end; p += lanes) {
        const int32_t after = next_place;   // places of the batch behind this one
        const int left = (int)min(end - p, (int64_t)lanes);
        for (int at = 0; at < lanes; at += 2 * U) {
            if (lanes >= 2 * U) load(two, place, at + U);
            add(one, left, at);
            const bool more = at + 2 * U < lanes;
            load(one, more ? place : after, more ? at + 2 * U : 0);
            if (lanes >= 2 * U) add(two, left, at + U);
        }
        if (LONG && ((uint32_t)(p - lo) + (uint32_t)lanes) % kSumChain == 0) put();
        place = next_place; group = next_group;
        row = row_of(group);
        ask(p + 2 * lanes);
    }
    flush();
}

// The shares of the ids that begin in a chunk and go on behind it: a block looks at every gridDim.x-th chunk; 32 lanes of four columns.  Up to 32 shares are added up by a warp, more
// by 32 warps that each take a stretch of the chunks that the id spans.  (The chunks, 8,192 at most, are one round of eight multiprocessors or more.  Without the loop and its
// barriers the compiler has fewer shares on their way: a million ids of 64 columns into three rows 116 us, so 103.)
constexpr int kWarpShares = 32;
struct Spanned { int32_t chunk, shares, row; };   // the chunk that the id begins in
__device__ __forceinline__ Spanned spanned(const SumArgs& a, int32_t chunk) {
    const int32_t g = a.begun[chunk];
    const int64_t end = min((int64_t)a.starts[g + 1], a.n), row = a.into == MG_ROWS_COMPACT ? g : id_at(a.group_ids, a.ids_are_i64, g);
    return {chunk, min((int32_t)((end - 1) / a.chunk), a.chunks - 1) - chunk + 1, row < a.n_rows ? (int32_t)row : -1};
}
// (of 8,192 shares, the most that there are, a warp has 256)
__device__ __forceinline__ float4 add_shares(const SumArgs& a, int32_t chunk, int32_t lo, int32_t hi, int32_t c) {
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c >= a.dim) return s;
    constexpr int U = 8;
    for (int32_t i0 = lo; i0 < hi; i0 += U) {
        float4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)   // (the first chunk's is the share of an id that begins there)
            v[u] = i0 + u < hi ? *reinterpret_cast<const float4*>(a.shares + ((int64_t)(chunk + i0 + u) * 2 + (i0 + u == 0)) * a.pitch + c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int u = 0; u < U; ++u) { s.x += v[u].x; s.y += v[u].y; s.z += v[u].z; s.w += v[u].w; }
    }
    return s;
}
template <typename O>
__device__ __forceinline__ void write_joined(const SumArgs& a, int64_t row, int32_t c, const float4& s) {
    if (row < 0) return;
    const float all[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < a.dim) {
            float one[1] = {all[e]};
            write_sum<O, 1>(a, row, c + e, one);
        }
}
template <typename O>
__global__ void __launch_bounds__(kJoinThreads) k_join_shares(const __grid_constant__ SumArgs a) {
    constexpr int W = kJoinThreads / 32;
    __shared__ float4 part[W][32];
    __shared__ Spanned few[kJoinThreads], many[kJoinThreads];   // (their order does not matter: each id's sum is its own)
    __shared__ int32_t n_few, n_many;
    chain_wait();
    chain_start();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t c = ((int32_t)blockIdx.y * 32 + lane) * 4;
    for (int32_t c0 = (int32_t)blockIdx.x; c0 < a.chunks; c0 += (int32_t)gridDim.x * kJoinThreads) {
        if (threadIdx.x == 0) n_few = n_many = 0;
        __syncthreads();
        const int64_t mine = c0 + (int64_t)threadIdx.x * gridDim.x;
        if (mine < a.chunks && a.begun[mine] >= 0) {
            const Spanned s = spanned(a, (int32_t)mine);
            if (s.shares <= kWarpShares) few[atomicAdd(&n_few, 1)] = s;
            else many[atomicAdd(&n_many, 1)] = s;
        }
        __syncthreads();
        for (int f = warp; f < n_few; f += W) write_joined<O>(a, few[f].row, c, add_shares(a, few[f].chunk, 0, few[f].shares, c));
        for (int f = 0; f < n_many; ++f) {
            const Spanned s = many[f];
            part[warp][lane] = add_shares(a, s.chunk, (int32_t)((int64_t)s.shares * warp / W), (int32_t)((int64_t)s.shares * (warp + 1) / W), c);
            __syncthreads();
            if (warp == 0) {
                float4 t = part[0][lane];
                for (int w = 1; w < W; ++w) { const float4 o = part[w][lane]; t.x += o.x; t.y += o.y; t.z += o.z; t.w += o.w; }
                write_joined<O>(a, s.row, c, t);
            }
            __syncthreads();
        }
        __syncthreads();   // (the counters are set back behind the warps that read them)
    }
}

}  // namespace mgrows
