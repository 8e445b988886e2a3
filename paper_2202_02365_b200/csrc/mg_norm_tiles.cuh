// Group norm of samples of several rows, in two passes: tiles of rows are summed up by channel, the last block of a sample's brings its sums
// together, and a launch later the tiles' results are computed.  No block waits for another.  A launch does the sums of one window of samples and
// the results of the window before, so that both passes keep the memory busy together and the second finds its rows in L2.
#pragma once

#include "mg_norm_rows.cuh"

namespace mgnorm {

constexpr int kFan = 32;             // tiles whose sums one block brings together; then as many of those
constexpr int kInlineSamples = 64;   // samples whose place is handed over in the kernel's parameters

struct TileArgs : NormArgs {
    // samples: equal ones, or a table of (first row, first tile), one entry more than samples
    int32_t samples = 0, equal = 0;
    int64_t rows_per_sample = 0;
    int32_t tiles_per_sample = 0;
    const int2* table = nullptr;     // null: `inl`
    int2 inl[kInlineSamples + 1];
    // tiles: tile_rows rows, each in `chunks` runs of (256 or fewer) vectors
    int32_t tile_rows = 0, chunks = 0, tx = 0;   // tx: log2 of the threads along a row
    // this launch: sums of tiles from sums_tile on in the first sums_blocks blocks, results of those from result_tile on in the others
    int32_t sums_tile = 0, sums_blocks = 0, result_tile = 0, result_tiles = 0, reversed = 0;
    // workspace
    uint32_t* fan_count = nullptr;   // cleared: sums that have arrived, by kFan tiles of a sample ...
    uint32_t* sample_count = nullptr;   // ... and by sample
    float* tile_parts = nullptr;     // [tiles][2][channels]
    float* fan_parts = nullptr;      // [tiles / kFan + samples][2][channels]
    float* group_parts = nullptr;    // backward: mean of dz w, mean of dz w hat: [samples][2][groups]
};

struct Tile {
    int32_t tile, sample, first, tiles;   // its number among all; the sample's first tile and how many it has
    int64_t row0, row1, sample_rows;
};

__device__ __forceinline__ int2 sample_entry(const TileArgs& a, int32_t s) { return a.table ? a.table[s] : a.inl[s]; }

// the sample and the rows of a tile
__device__ __forceinline__ void locate_tile(const TileArgs& a, int32_t tile, Tile* t) {
    t->tile = tile;
    int64_t s0, s1;
    if (a.equal) {
        t->sample = tile / a.tiles_per_sample;
        t->first = t->sample * a.tiles_per_sample;
        t->tiles = a.tiles_per_sample;
        s0 = t->sample * a.rows_per_sample; s1 = s0 + a.rows_per_sample;
    } else {
        int32_t l = 0, h = a.samples;
        while (h - l > 1) {
            const int32_t mid = (l + h) >> 1;
            if (sample_entry(a, mid).y <= tile) l = mid; else h = mid;
        }
        const int2 e = sample_entry(a, l), f = sample_entry(a, l + 1);
        t->sample = l; t->first = e.y; t->tiles = f.y - e.y;
        s0 = e.x; s1 = f.x;
    }
    t->row0 = s0 + (int64_t)(tile - t->first) * a.tile_rows;
    t->row1 = min(s1, t->row0 + a.tile_rows);
    t->sample_rows = s1 - s0;
}

// Mean and sum of squares about it of two sets (Chan, Golub and LeVeque 1979)
__device__ __forceinline__ void merge_moments(float& n, float& m, float& q, float nb, float mb, float qb) {
    const float all = n + nb, f = all > 0.f ? __fdividef(nb, all) : 0.f, d = mb - m;
    m = fmaf(d, f, m);
    q += fmaf(d * n * f, d, qb);   // (a first set, n = 0: no square of its mean)
    n = all;
}

// What a thread has of its channels: forward the mean and the squares about it over n rows, backward two sums
template <int VEC> struct Pair { float n; float u[VEC], v[VEC]; };

template <int VEC, bool BACKWARD>
__device__ __forceinline__ void merge(Pair<VEC>& a, float nb, const float (&u)[VEC], const float (&v)[VEC]) {
    if (BACKWARD) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) { a.u[e] += u[e]; a.v[e] += v[e]; }
    } else {
        const float all = a.n + nb, f = all > 0.f ? __fdividef(nb, all) : 0.f, g = a.n * f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float d = u[e] - a.u[e];
            a.u[e] = fmaf(d, f, a.u[e]);
            a.v[e] += fmaf(d * g, d, v[e]);   // (a first set, g = 0: no square of its mean)
        }
        a.n = all;
    }
}

// Sums of a tile: every thread has one vector of the channels and every n_ty-th row, K rows in flight; then the block's threads are brought together.
template <typename T, int VEC, bool BACKWARD, int K>
__device__ __forceinline__ void tile_sums(const TileArgs& a, const Tile& t, int32_t c, bool in, int ty, int n_ty, float mean, float rstd, const float (&w)[VEC],
                                          const float (&b)[VEC], Pair<VEC>& p) {
    p.n = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) p.u[e] = p.v[e] = 0.f;
    if (!in) return;
    const int64_t x_step = (int64_t)n_ty * a.x_stride, d_step = (int64_t)n_ty * a.d_y_stride;
    const T* x = static_cast<const T*>(a.x) + (t.row0 + ty) * a.x_stride + c;
    const T* d_y = static_cast<const T*>(a.d_y) + (BACKWARD ? (t.row0 + ty) * a.d_y_stride + c : 0);
    const int32_t rows = (int32_t)(t.row1 - t.row0);
    for (int32_t r = ty; r < rows; r += K * n_ty) {
        Raw<T, VEC> raw[K], rd[BACKWARD ? K : 1];
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (r + k * n_ty < rows) {
                raw[k].load(x + k * x_step);
                if (BACKWARD) rd[k].load(d_y + k * d_step);
            }
        if constexpr (BACKWARD) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (r + k * n_ty >= rows) break;
                float h[VEC], d[VEC];
                grad_vector<T, VEC>(a, raw[k], rd[k], a.drop.on ? drop_key(a.drop, t.row0 + r + k * n_ty) : 0, c, mean, rstd, w, b, h, d);
#pragma unroll
                for (int e = 0; e < VEC; ++e) { p.u[e] = fmaf(d[e], h[e], p.u[e]); p.v[e] += d[e]; }
            }
            d_y += K * d_step;
        } else {
            float u[VEC], v[VEC];
            if (r + (K - 1) * n_ty < rows) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    u[e] = raw[0].get(e); v[e] = 0.f;
#pragma unroll
                    for (int k = 1; k < K; ++k) u[e] += raw[k].get(e);
                    u[e] *= 1.f / K;
#pragma unroll
                    for (int k = 0; k < K; ++k) { const float d = raw[k].get(e) - u[e]; v[e] = fmaf(d, d, v[e]); }
                }
                merge<VEC, false>(p, (float)K, u, v);
            } else {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    if (r + k * n_ty >= rows) break;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) { u[e] = raw[k].get(e); v[e] = 0.f; }
                    merge<VEC, false>(p, 1.f, u, v);
                }
            }
        }
        x += K * x_step;
    }
}

// lanes with the same channels
template <int VEC, bool BACKWARD>
__device__ __forceinline__ void lane_pairs(Pair<VEC>& p, int threads_x) {
    const int lane = threadIdx.x & 31;
    for (int o = threads_x; o < 32; o <<= 1) {
        float u[VEC], v[VEC];
        const float n = __shfl_xor_sync(0xFFFFFFFFu, p.n, o);
#pragma unroll
        for (int e = 0; e < VEC; ++e) { u[e] = __shfl_xor_sync(0xFFFFFFFFu, p.u[e], o); v[e] = __shfl_xor_sync(0xFFFFFFFFu, p.v[e], o); }
        if (!BACKWARD && (lane & o)) {   // (the lower lane's set first on both sides, so that both have the same)
            Pair<VEC> q;
            q.n = n;
#pragma unroll
            for (int e = 0; e < VEC; ++e) { q.u[e] = u[e]; q.v[e] = v[e]; u[e] = p.u[e]; v[e] = p.v[e]; }
            const float mine = p.n;
            merge<VEC, BACKWARD>(q, mine, u, v);
            p = q;
        } else merge<VEC, BACKWARD>(p, n, u, v);
    }
}

// The block's threads with the same channels, into `out` ([2][channels], the chunk's channels of it)
template <int VEC, bool BACKWARD>
__device__ __forceinline__ void block_pairs(const TileArgs& a, Pair<VEC>& p, float* smem, int tx, int32_t chunk0, float* out) {
    const int threads_x = 1 << a.tx, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    lane_pairs<VEC, BACKWARD>(p, threads_x);
    const int across = threads_x < 32 ? kNormThreads / 32 : kNormThreads / threads_x;   // sets of a channel that are left
    const int set = threads_x < 32 ? warp : threadIdx.x >> a.tx, width = threads_x * VEC;
    float* su = smem;                          // [across][width], across * width <= kNormThreads * VEC
    float* sv = smem + kNormThreads * VEC;
    float* sn = smem + 2 * kNormThreads * VEC;   // [across]
    __syncthreads();
    if (threads_x >= 32 || lane < threads_x) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) { su[set * width + tx * VEC + e] = p.u[e]; sv[set * width + tx * VEC + e] = p.v[e]; }
        if (tx == 0) sn[set] = p.n;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < width; i += kNormThreads) {
        const int32_t c = chunk0 + i;
        if (c >= a.channels) break;
        float u = su[i], v = sv[i], n = sn[0];
        for (int s = 1; s < across; ++s) {
            if (BACKWARD) { u += su[s * width + i]; v += sv[s * width + i]; }
            else merge_moments(n, u, v, sn[s], su[s * width + i], sv[s * width + i]);
        }
        __stcg(out + c, u);
        __stcg(out + a.channels + c, v);
    }
}

// sums of `n` sets that lie one behind the other, rows_of(i) rows each, into `out` and, where it is given, `shared` ([2][stride]); V channels a
// thread at a time, B sets in flight
template <bool BACKWARD, int NT, int V, int B, typename Rows>
__device__ __forceinline__ void merge_parts(const TileArgs& a, const float* parts, int32_t n, Rows rows_of, float* out, int tid, float* shared, int stride) {
    const int64_t step = 2 * (int64_t)a.channels;
    for (int32_t c = tid * V; c < a.channels; c += NT * V) {
        float u[V], v[V], m = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) u[e] = v[e] = 0.f;
        for (int32_t i0 = 0; i0 < n; i0 += B) {
            float pu[B][V], pv[B][V];
#pragma unroll
            for (int k = 0; k < B; ++k)
                if (i0 + k < n) {
                    const float* from = parts + (i0 + k) * step + c;
                    if constexpr (V == 4) {
                        const float4 x = __ldcg(reinterpret_cast<const float4*>(from)), y = __ldcg(reinterpret_cast<const float4*>(from + a.channels));
                        pu[k][0] = x.x; pu[k][1] = x.y; pu[k][2] = x.z; pu[k][3] = x.w;
                        pv[k][0] = y.x; pv[k][1] = y.y; pv[k][2] = y.z; pv[k][3] = y.w;
                    } else { pu[k][0] = __ldcg(from); pv[k][0] = __ldcg(from + a.channels); }
                }
#pragma unroll
            for (int k = 0; k < B; ++k)
                if (i0 + k < n) {
                    if (BACKWARD) {
#pragma unroll
                        for (int e = 0; e < V; ++e) { u[e] += pu[k][e]; v[e] += pv[k][e]; }
                    } else {
                        const float nb = rows_of(i0 + k), all = m + nb, f = __fdividef(nb, all), g = m * f;   // (no set is empty)
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const float d = pu[k][e] - u[e];
                            u[e] = fmaf(d, f, u[e]);
                            v[e] += fmaf(d * g, d, pv[k][e]);
                        }
                        m = all;
                    }
                }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
            __stcg(out + c + e, u[e]);
            __stcg(out + a.channels + c + e, v[e]);
            if (shared) { shared[c + e] = u[e]; shared[stride + c + e] = v[e]; }
        }
    }
}

// the groups' values from the channels' of a whole sample: a warp per group
template <bool BACKWARD, int NT>
__device__ __forceinline__ void finish_sample(const TileArgs& a, int32_t sample, float rows, const float* part) {
    const int lane = threadIdx.x & 31;
    const float n = rows * (float)a.each;
    for (int32_t g = threadIdx.x >> 5; g < a.groups; g += NT / 32) {
        float u = 0.f, v = 0.f;
        for (int32_t c = g * a.each + lane; c < (g + 1) * a.each; c += 32) {
            if (BACKWARD) {
                const float w = a.weight ? a.weight[c] : 1.f;
                u = fmaf(w, __ldcg(part + c), u); v = fmaf(w, __ldcg(part + a.channels + c), v);
            } else u += __ldcg(part + c);
        }
        u = row_sum(u, 5); v = row_sum(v, 5);
        if (BACKWARD) {
            if (lane == 0) {
                __stcg(a.group_parts + ((int64_t)sample * 2) * a.groups + g, v / n);        // mean of dz w
                __stcg(a.group_parts + ((int64_t)sample * 2 + 1) * a.groups + g, u / n);    // mean of dz w hat
            }
            continue;
        }
        const float mean = u / (float)a.each;
        for (int32_t c = g * a.each + lane; c < (g + 1) * a.each; c += 32) {
            const float d = __ldcg(part + c) - mean;
            v += fmaf(d * d, rows, __ldcg(part + a.channels + c));
        }
        v = row_sum(v, 5);
        if (lane == 0) {
            __stcg(a.mean + (int64_t)sample * a.groups + g, mean);
            __stcg(a.rstd + (int64_t)sample * a.groups + g, rsqrtf(v / n + a.eps));
        }
    }
}

// A tile's sums are written: the last of kFan tiles brings theirs together, the last of those the sample's.
template <bool BACKWARD>
__device__ __forceinline__ void arrive(const TileArgs& a, const Tile& t, int32_t* sh_last) {
    const int32_t in_sample = t.tile - t.first, fan = in_sample / kFan, fans = (t.tiles + kFan - 1) / kFan, fan_tiles = min(kFan, t.tiles - fan * kFan);
    const int64_t fan_id = t.first / kFan + t.sample + fan;   // (blocks of kFan tiles of all samples before lie below)
    __syncthreads();
    if (threadIdx.x == 0) {   // (what the block's threads wrote before they met is announced with it)
        __threadfence();
        *sh_last = atomicAdd(a.fan_count + fan_id, 1u) + 1u == (uint32_t)(fan_tiles * a.chunks);
        __threadfence();
    }
    __syncthreads();
    if (!*sh_last) return;
    const int64_t step = 2 * (int64_t)a.channels;
    float* fan_part = a.fan_parts + fan_id * step;
    const auto tile_rows = [&](int32_t i) { return (float)min((int64_t)a.tile_rows, t.sample_rows - ((int64_t)fan * kFan + i) * a.tile_rows); };
    float* whole = BACKWARD ? a.parts + t.sample * step : a.fan_parts + (t.first / kFan + t.sample) * step;   // the sample's channels
    merge_parts<BACKWARD, kNormThreads, 1, 8>(a, a.tile_parts + ((int64_t)t.first + fan * kFan) * step, fan_tiles, tile_rows, fans == 1 ? whole : fan_part, threadIdx.x, nullptr, 0);
    __syncthreads();
    if (fans > 1) {
        if (threadIdx.x == 0) {
            __threadfence();
            *sh_last = atomicAdd(a.sample_count + t.sample, 1u) + 1u == (uint32_t)fans;
            __threadfence();
        }
        __syncthreads();
        if (!*sh_last) return;
        const auto fan_rows = [&](int32_t i) { return (float)min((int64_t)kFan * a.tile_rows, t.sample_rows - (int64_t)i * kFan * a.tile_rows); };
        merge_parts<BACKWARD, kNormThreads, 1, 8>(a, a.fan_parts + (t.first / kFan + t.sample) * step, fans, fan_rows, whole, threadIdx.x, nullptr, 0);
        __syncthreads();
    }
    finish_sample<BACKWARD, kNormThreads>(a, t.sample, (float)t.sample_rows, whole);
}

template <int VEC>
__device__ __forceinline__ void load_params(const float* p, int32_t c, float without, float (&o)[VEC]) {
    if constexpr (VEC >= 4) if (p && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
        for (int q = 0; q < VEC; q += 4) {
            const float4 f = *reinterpret_cast<const float4*>(p + c + q);
            o[q] = f.x; o[q + 1] = f.y; o[q + 2] = f.z; o[q + 3] = f.w;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) o[e] = p ? p[c + e] : without;
}

template <typename T, int VEC, bool BACKWARD, int K, int U, int MINB>
__global__ void __launch_bounds__(kNormThreads, MINB) k_norm_tiles(const __grid_constant__ TileArgs a) {
    __shared__ __align__(16) float smem[2 * kNormThreads * VEC + kNormWarps];
    __shared__ int32_t sh_flag;
    const int tx = threadIdx.x & ((1 << a.tx) - 1), ty = threadIdx.x >> a.tx, n_ty = kNormThreads >> a.tx;
    const bool sums = (int32_t)blockIdx.x < a.sums_blocks;
    const int32_t item = (int32_t)blockIdx.x - (sums ? 0 : a.sums_blocks), tile = item / a.chunks, chunk = item - tile * a.chunks;
    Tile t;
    locate_tile(a, sums ? a.sums_tile + tile : a.result_tile + (a.reversed ? a.result_tiles - 1 - tile : tile), &t);
    const int32_t chunk0 = chunk * (VEC << a.tx), c = chunk0 + tx * VEC;
    const bool in = c < a.channels;
    const int64_t stat = (int64_t)t.sample * a.groups + (in ? c / a.each : 0);
    float w[VEC], b[VEC], mean = 0.f, rstd = 0.f;
    if (BACKWARD || !sums) {
        load_params<VEC>(in ? a.weight : nullptr, c, 1.f, w);
        load_params<VEC>(in ? a.bias : nullptr, c, 0.f, b);
        mean = a.mean[stat]; rstd = a.rstd[stat];
    }
    if (sums) {
        Pair<VEC> p;
        tile_sums<T, VEC, BACKWARD, K>(a, t, c, in, ty, n_ty, mean, rstd, w, b, p);
        block_pairs<VEC, BACKWARD>(a, p, smem, tx, chunk0, a.tile_parts + 2 * (int64_t)t.tile * a.channels);
        arrive<BACKWARD>(a, t, &sh_flag);
        return;
    }
    if (!in) return;
    float s1 = 0.f, s2 = 0.f;
    if (BACKWARD) {
        const int64_t at_group = (int64_t)t.sample * 2 * a.groups + c / a.each;
        s1 = a.group_parts[at_group]; s2 = a.group_parts[at_group + a.groups];
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] *= rstd;
    }
    const int64_t x_step = (int64_t)n_ty * a.x_stride, d_step = (int64_t)n_ty * a.d_y_stride, out_step = (int64_t)n_ty * a.out_stride;
    const T* x = static_cast<const T*>(a.x) + (t.row0 + ty) * a.x_stride + c;
    const T* d_y = static_cast<const T*>(a.d_y) + (BACKWARD ? (t.row0 + ty) * a.d_y_stride + c : 0);
    T* out = static_cast<T*>(a.out) + (t.row0 + ty) * a.out_stride + c;
    const int32_t rows = (int32_t)(t.row1 - t.row0);
    for (int32_t r = ty; r < rows; r += U * n_ty) {
        Raw<T, VEC> raw[U], rd[BACKWARD ? U : 1];
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (r + k * n_ty < rows) {
                raw[k].load(x + k * x_step);
                if (BACKWARD) rd[k].load(d_y + k * d_step);
            }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (r + k * n_ty >= rows) break;
            const uint64_t key = a.drop.on ? drop_key(a.drop, t.row0 + r + k * n_ty) : 0;
            float f[VEC];
            if constexpr (BACKWARD) {
                float h[VEC];
                grad_vector<T, VEC>(a, raw[k], rd[k], key, c, mean, rstd, w, b, h, f);
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = rstd * fmaf(-h[e], s2, fmaf(f[e], w[e], -s1));
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = fmaf(raw[k].get(e) - mean, w[e], b[e]);
                act_values<VEC>(a.act, f);
                if (a.drop.on) {
                    Keep<VEC> keep;
                    keep.draw(a.drop, key, (uint32_t)c);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) f[e] = keep(a.drop, e) ? f[e] * a.drop.factor : 0.f;
                }
            }
            raw[k].put(f);
            raw[k].store(out + k * out_step);
        }
        x += U * x_step; out += U * out_step;
        if (BACKWARD) d_y += U * d_step;
    }
}

// Samples without rows have no tiles: their statistics (backward: their parts of the weight's and bias's gradients) are zero.
template <typename = void>
__global__ void k_norm_empty(const __grid_constant__ TileArgs a, int backward) {
    for (int32_t s = blockIdx.x; s < a.samples; s += gridDim.x) {
        if (sample_entry(a, s).x != sample_entry(a, s + 1).x) continue;
        if (!backward) for (int32_t g = threadIdx.x; g < a.groups; g += blockDim.x) { a.mean[(int64_t)s * a.groups + g] = 0.f; a.rstd[(int64_t)s * a.groups + g] = 0.f; }
        else for (int32_t c = threadIdx.x; c < 2 * a.channels; c += blockDim.x) a.parts[2 * (int64_t)s * a.channels + c] = 0.f;
    }
}

// what a translation unit of its own per row type launches
struct RowLaunch { int vec, nv; bool general, backward; int grid; RowShape shape; };
struct TileLaunch { int vec; bool backward; int64_t grid; };
template <typename T> void launch_dropout(int vec, const void* x, int64_t x_stride, void* y, int64_t y_stride, int64_t rows, int32_t channels, const DropArgs& d, int grid, cudaStream_t st);
template <typename T> void launch_rows(const RowLaunch& l, const NormArgs& a, cudaStream_t st);
template <typename T> void launch_tiles(const TileLaunch& l, const TileArgs& a, cudaStream_t st);

}  // namespace mgnorm
