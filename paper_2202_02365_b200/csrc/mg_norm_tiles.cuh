// Group norm of samples of several rows.
//
// What fits: a block, or a cluster of blocks, sums a sample up and computes its results in one launch (k_norm_block; k_norm_wide for many short samples that it
// does not take).  The rest: two launches.  Tiles of rows are summed up, the last block of a sample's tiles brings its sums together (no block waits for
// another), and the second launch computes the results from the rows once more.  It reads most of them from memory again: of 185 MB and more 93 to 100 % come
// from DRAM, of 93 MB 75 to 98, of 67 MB of fp16 maps 37 to 65; to begin with the tiles that were summed up last takes the same time to half a percent.  Sums are
// means and squares about them, merged pairwise by Chan, Golub and LeVeque's formulas: a mean that is k deviations from zero costs the variance the digits
// of k, not of its square; for the gradient, plain sums of dz and dz hat.
//
// The bytes bound it: x twice and y once (backward x and d_y twice, d_x once).  543,000 rows of 256 fp32 channels in 24 samples, with a ReLU and a dropout,
// take 270 us for 1.67 GB, 6.2 TB/s; the gradient, with a GELU and a keyed dropout, 512 us for 2.78 GB, 5.4 TB/s: its slopes and masks are computed twice.
// (One persistent launch with the rows kept in shared memory until their sample's sums were there, or read again as soon as they were, took
// 1.4 to 3.9 times as long: every tile waits for round trips through L2 that nothing hides.  So did launches over a few samples at a time, whose rows
// stay in L2: six of the 24 a call 334 us, one a call 641.)
#pragma once

#include "mg_norm_rows.cuh"

namespace mgnorm {

constexpr int kFan = 32;             // tiles whose sums one block brings together; then as many of those
constexpr int kInlineSamples = 64;   // samples whose place is handed over in the kernel's parameters

// how a launch's blocks lie on a tile: 2^tx threads along a row, the channels in `chunks` runs of as many vectors
struct TileShape { int32_t tx = 0, chunks = 0; };

struct TileArgs : NormArgs {
    // samples: equal ones, or a table of (first row, first tile), one entry more than samples
    int32_t samples = 0, equal = 0;
    int64_t rows_per_sample = 0;
    int32_t tiles_per_sample = 0;
    const int2* table = nullptr;     // null: `inl`
    int2 inl[kInlineSamples + 1];
    int32_t tile_rows = 0, tiles = 0;
    int32_t parts_of_tile = 1, part_rows = 0;   // results: a tile's rows by several blocks
    TileShape sums, results;
    int32_t run = 0;                 // channels of a run, for the sums
    // workspace
    uint32_t* fan_count = nullptr;      // cleared: sums that have arrived, by kFan tiles of a sample ...
    uint32_t* sample_count = nullptr;   // ... and by sample
    float* tile_parts = nullptr;     // [tiles][chunks][2][groups]: mean and squares about it, or (backward) sums of dz w hat and dz w
    float* fan_parts = nullptr;      // [tiles / kFan + samples][2][groups]
    float* group_parts = nullptr;    // backward: mean of dz w, mean of dz w hat: [samples][2][groups]
    // (parts: the tiles' sums by channel)
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

// x - mean and dz = dropout(dy) act' of a vector, for the statistics of one sample: wr = weight rstd
template <typename T, int VEC>
__device__ __forceinline__ void centred_grad(const TileArgs& a, const Raw<T, VEC>& rx, const Raw<T, VEC>& rd, uint64_t key, int32_t c, float mean, float rstd,
                                             const float (&wr)[VEC], const float* sb, float (&xc)[VEC], float (&d)[VEC]) {
    float n[VEC], b[VEC];
    Params<VEC, 8, true>::read(sb, b);
#pragma unroll
    for (int e = 0; e < VEC; ++e) { xc[e] = rx.get(e) - mean; n[e] = fmaf(xc[e], wr[e], b[e]); d[e] = rd.get(e); }
    act_slopes<VEC>(a.act, d, n, b, [&](int e) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) if (i == e) x = rx.get(i);
        return ((double)x - (double)mean) * (double)rstd * (double)(a.weight ? a.weight[c + e] : 1.f) + (double)(a.bias ? a.bias[c + e] : 0.f);
    });
    drop_vector<VEC>(a.drop, key, c, d);
}

// Sums of a tile: every thread has one vector of the channels and every n_ty-th row, K rows on their way; then the block's threads are brought
// together.  Forward: the mean of K rows first, then the squares about it, then the two sets of moments as one.
template <typename T, int VEC, bool BACKWARD, int K>
__device__ __forceinline__ void tile_sums(const TileArgs& a, const Tile& t, int32_t c, bool in, int ty, int n_ty, float mean, float rstd, const float* swr,
                                          const float* sb, Pair<VEC>& p) {
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
        uint64_t key = 0;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (r + k * n_ty < rows) {
                raw[k].load(x + k * x_step);
                if (BACKWARD) rd[k].load(d_y + k * d_step);
            }
        // (a single row's key with the row: behind its arrival it would be waited for once more.  More rows' are too many registers.)
        if (BACKWARD && K == 1 && a.drop.on) key = drop_key(a.drop, t.row0 + r);
        x += K * x_step;
        if (BACKWARD) d_y += K * d_step;
        if constexpr (BACKWARD) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (r + k * n_ty >= rows) break;
                float xc[VEC], d[VEC], wr[VEC];
                Params<VEC, 8, true>::read(swr, wr);
                if (K > 1 && a.drop.on) key = drop_key(a.drop, t.row0 + r + k * n_ty);
                centred_grad<T, VEC>(a, raw[k], rd[k], key, c, mean, rstd, wr, sb, xc, d);
#pragma unroll
                for (int e = 0; e < VEC; ++e) { p.u[e] = fmaf(d[e], xc[e], p.u[e]); p.v[e] += d[e]; }
            }
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
    }
    if (BACKWARD) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) p.u[e] *= rstd;
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

template <int VEC> __device__ __forceinline__ void put_shared(float* s, const float (&v)[VEC]) {
    if constexpr (VEC % 4 == 0) {
#pragma unroll
        for (int e = 0; e < VEC; e += 4) *reinterpret_cast<float4*>(s + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[e] = v[e];
    }
}

// The block's threads with the same channels: su[i], sv[i] become channel i's of the run (su, sv: [256 * VEC], sn: [kNormWarps or the sets])
template <int VEC, bool BACKWARD>
__device__ __forceinline__ void block_pairs(Pair<VEC>& p, float* su, float* sv, float* sn, int log_x, int32_t channels) {
    const int threads_x = 1 << log_x, tx = threadIdx.x & (threads_x - 1), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    lane_pairs<VEC, BACKWARD>(p, threads_x);
    const int across = threads_x < 32 ? kNormWarps : kNormThreads / threads_x;   // sets of a channel that are left
    const int set = threads_x < 32 ? warp : threadIdx.x >> log_x, width = threads_x * VEC;
    if (threads_x >= 32 || lane < threads_x) {
        put_shared<VEC>(su + set * width + tx * VEC, p.u);
        put_shared<VEC>(sv + set * width + tx * VEC, p.v);
        if (tx == 0) sn[set] = p.n;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < min(width, channels); i += kNormThreads) {   // (a thread reads and writes its channel's column alone)
        float u = su[i], v = sv[i], n = sn[0];
        if (across == 1) break;
        for (int s = 1; s < across; ++s) {
            if (BACKWARD) { u += su[s * width + i]; v += sv[s * width + i]; }
            else merge_moments(n, u, v, sn[s], su[s * width + i], sv[s * width + i]);
        }
        su[i] = u; sv[i] = v;
    }
    __syncthreads();
}

// threads that share a group, of one warp, where `threads` work on `groups`
__device__ __forceinline__ int group_threads(int groups, int threads) {
    int per = 1;
    while (per < 32 && 2 * per * groups <= threads) per *= 2;
    return per;
}

// channels that a run [c0, c1) and a group have in common
__device__ __forceinline__ int32_t shared_channels(const TileArgs& a, int32_t g, int32_t c0, int32_t c1) { return max(0, min(c1, (g + 1) * a.each) - max(c0, g * a.each)); }

// a run's groups from its channels, to put(g, u, v): mean and squares about it, or sums of dz w hat and dz w
template <bool BACKWARD, typename Put>
__device__ __forceinline__ void run_groups(const TileArgs& a, const float* su, const float* sv, int32_t c0, int32_t c1, float rows, Put put) {
    const int32_t g_lo = c0 / a.each, n_g = (c1 - 1) / a.each - g_lo + 1;
    const int per = group_threads(n_g, kNormThreads), sub = threadIdx.x % per;
    for (int32_t q = 0; q < n_g; q += kNormThreads / per) {   // (all threads of a warp go round together)
        const int32_t g = g_lo + q + threadIdx.x / per, lo = max(c0, g * a.each), hi = q + (int)threadIdx.x / per < n_g ? min(c1, (g + 1) * a.each) : 0;
        float u = 0.f, v = 0.f;
        for (int32_t c = lo + sub; c < hi; c += per) {
            if (BACKWARD) {
                const float w = a.weight ? a.weight[c] : 1.f;
                u = fmaf(w, su[c - c0], u); v = fmaf(w, sv[c - c0], v);
            } else u += su[c - c0];
        }
        for (int o = 1; o < per; o <<= 1) { u += __shfl_xor_sync(0xFFFFFFFFu, u, o); if (BACKWARD) v += __shfl_xor_sync(0xFFFFFFFFu, v, o); }
        if (!BACKWARD) {
            u /= (float)max(hi - lo, 1);
            for (int32_t c = lo + sub; c < hi; c += per) { const float d = su[c - c0] - u; v += fmaf(d * rows, d, sv[c - c0]); }
            for (int o = 1; o < per; o <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        }
        if (sub == 0 && lo < hi) put(g, u, v);
    }
}

// `n` sets of the groups' values, fetch(i, g, u, v), of values_of(i, g) values each (none: the set is not there), to `use(g, u, v)`
template <bool BACKWARD, typename Values, typename Fetch, typename Use>
__device__ __forceinline__ void merge_sets(const TileArgs& a, int32_t n, Values values_of, Fetch fetch, Use use) {
    const int per = group_threads(a.groups, kNormThreads), sub = threadIdx.x % per;
    constexpr int B = 4;   // sets on their way at a time
    for (int32_t g0 = 0; g0 < a.groups; g0 += kNormThreads / per) {
        const int32_t g = min(g0 + (int)threadIdx.x / per, a.groups - 1);
        float m = 0.f, u = 0.f, v = 0.f;
        for (int32_t i0 = sub; i0 < n; i0 += B * per) {
            float pu[B], pv[B], pn[B];
#pragma unroll
            for (int k = 0; k < B; ++k) {
                const int32_t i = min(i0 + k * per, n - 1);
                pn[k] = i0 + k * per < n ? values_of(i, g) : 0.f;
                fetch(i, g, pu[k], pv[k]);
            }
#pragma unroll
            for (int k = 0; k < B; ++k) {
                if (pn[k] == 0.f) continue;
                if (BACKWARD) { u += pu[k]; v += pv[k]; }
                else merge_moments(m, u, v, pn[k], pu[k], pv[k]);
            }
        }
        for (int o = 1; o < per; o <<= 1) {
            const float mb = __shfl_xor_sync(0xFFFFFFFFu, m, o), ub = __shfl_xor_sync(0xFFFFFFFFu, u, o), vb = __shfl_xor_sync(0xFFFFFFFFu, v, o);
            if (BACKWARD) { u += ub; v += vb; }
            else if (threadIdx.x & o) { float x = mb, y = ub, z = vb; merge_moments(x, y, z, m, u, v); m = x; u = y; v = z; }   // (the lower threads' set first)
            else merge_moments(m, u, v, mb, ub, vb);
        }
        if (sub == 0 && g0 + (int)threadIdx.x / per < a.groups) use(g, u, v);
    }
}

// A block's sums are written: the last of kFan tiles' brings theirs together, the last of those the sample's.
template <bool BACKWARD>
__device__ __forceinline__ void arrive(const TileArgs& a, const Tile& t, int32_t* sh_last) {
    const int32_t fan = (t.tile - t.first) / kFan, fans = (t.tiles + kFan - 1) / kFan, fan_tiles = min(kFan, t.tiles - fan * kFan), chunks = a.sums.chunks;
    const int64_t first_fan = t.first / kFan + t.sample;   // (those of all samples before lie below)
    const int64_t step = 2 * (int64_t)a.groups;
    const auto last = [&](uint32_t* counter, int32_t want) {
        __syncthreads();
        if (threadIdx.x == 0) {   // (what the block's threads wrote before they met is announced with it)
            __threadfence();
            *sh_last = atomicAdd(counter, 1u) + 1u == (uint32_t)want;
            __threadfence();
        }
        __syncthreads();
        return *sh_last != 0;
    };
    const float values = (float)t.sample_rows * (float)a.each;
    const auto finish = [&](int32_t g, float u, float v) {
        if (BACKWARD) {
            a.group_parts[t.sample * step + g] = v / values;               // mean of dz w
            a.group_parts[t.sample * step + a.groups + g] = u / values;    // mean of dz w hat
        } else {
            a.mean[(int64_t)t.sample * a.groups + g] = u;
            a.rstd[(int64_t)t.sample * a.groups + g] = rsqrtf(v / values + a.eps);
        }
    };
    if (!last(a.fan_count + first_fan + fan, fan_tiles * chunks)) return;
    float* fan_part = a.fan_parts + (first_fan + fan) * step;
    const auto tile_values = [&](int32_t i, int32_t g) {
        const int64_t rows = min((int64_t)a.tile_rows, t.sample_rows - ((int64_t)fan * kFan + i / chunks) * a.tile_rows);
        const int32_t c0 = i % chunks * a.run;
        return (float)rows * (float)(chunks == 1 ? a.each : shared_channels(a, g, c0, min(c0 + a.run, a.channels)));
    };
    const auto keep = [&](int32_t g, float u, float v) {
        if (fans == 1) finish(g, u, v);
        else { __stcg(fan_part + g, u); __stcg(fan_part + a.groups + g, v); }
    };
    const auto from = [&](const float* sets) { return [=](int32_t i, int32_t g, float& u, float& v) { u = __ldcg(sets + i * step + g); v = __ldcg(sets + i * step + step / 2 + g); }; };
    merge_sets<BACKWARD>(a, fan_tiles * chunks, tile_values, from(a.tile_parts + ((int64_t)t.first + fan * kFan) * chunks * step), keep);
    if (fans == 1 || !last(a.sample_count + t.sample, fans)) return;
    const auto fan_values = [&](int32_t i, int32_t) { return (float)min((int64_t)kFan * a.tile_rows, t.sample_rows - (int64_t)i * kFan * a.tile_rows) * (float)a.each; };
    merge_sets<BACKWARD>(a, fans, fan_values, from(a.fan_parts + first_fan * step), finish);
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

// weight rstd and bias of a block's run of channels, for the gradient: in shared memory, so that more blocks fit an SM's registers
__device__ __forceinline__ void share_params(const TileArgs& a, const Tile& t, float* swr, float* sb, int32_t c0, int32_t n) {
    for (int i = threadIdx.x; i < n; i += kNormThreads) {
        swr[i] = (a.weight ? a.weight[c0 + i] : 1.f) * a.rstd[(int64_t)t.sample * a.groups + (c0 + i) / a.each];
        sb[i] = a.bias ? a.bias[c0 + i] : 0.f;
    }
    __syncthreads();
}

// A launch that may begin while the one before it ends: nothing of that one's is read, nor anything written, before chain_wait.
__device__ __forceinline__ void chain_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }   // (the next one's blocks may come where there is room)
__device__ __forceinline__ void chain_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Bound by the latency of its loads: of 181,000 fp32 rows of 256, forward, 41 us for 185 MB (4.5 TB/s) with four rows of 16 bytes to a thread, four blocks
// to an SM; backward 92 us for 370 MB with a row of 32 bytes of x and of d_y, three blocks, 61 % of the issue slots busy.
template <typename T, int VEC, bool BACKWARD, int K, int MINB>
__global__ void __launch_bounds__(kNormThreads, MINB) k_norm_sums(const __grid_constant__ TileArgs a) {
    __shared__ __align__(16) float su[kNormThreads * VEC], sv[kNormThreads * VEC], sw[BACKWARD ? kNormThreads * VEC : 4], sb[BACKWARD ? kNormThreads * VEC : 4];
    __shared__ float sn[kNormThreads];
    __shared__ int32_t sh_last;
    const int tx = threadIdx.x & ((1 << a.sums.tx) - 1), ty = threadIdx.x >> a.sums.tx, n_ty = kNormThreads >> a.sums.tx;
    const int32_t tile = (int32_t)blockIdx.x / a.sums.chunks, chunk = (int32_t)blockIdx.x - tile * a.sums.chunks;
    Tile t;
    locate_tile(a, tile, &t);
    const int32_t c0 = chunk * a.run, c1 = min(c0 + a.run, a.channels), c = c0 + tx * VEC;
    const bool in = c < c1;
    float mean = 0.f, rstd = 0.f;
    if (BACKWARD) {
        const int64_t stat = (int64_t)t.sample * a.groups + (in ? c / a.each : 0);
        mean = a.mean[stat]; rstd = a.rstd[stat];
        share_params(a, t, sw, sb, c0, c1 - c0);
    }
    Pair<VEC> p;
    tile_sums<T, VEC, BACKWARD, K>(a, t, c, in, ty, n_ty, mean, rstd, sw + tx * VEC, sb + tx * VEC, p);
    chain_start();
    block_pairs<VEC, BACKWARD>(p, su, sv, sn, a.sums.tx, c1 - c0);
    if (BACKWARD && a.parts) {
        float* to = a.parts + 2 * (int64_t)tile * a.channels + c0;
        for (int i = threadIdx.x; i < c1 - c0; i += kNormThreads) { to[i] = su[i]; to[a.channels + i] = sv[i]; }
    }
    float* part = a.tile_parts + 2 * ((int64_t)tile * a.sums.chunks + chunk) * a.groups;
    run_groups<BACKWARD>(a, su, sv, c0, c1, (float)(t.row1 - t.row0), [&](int32_t g, float u, float v) { __stcg(part + g, u); __stcg(part + a.groups + g, v); });
    arrive<BACKWARD>(a, t, &sh_last);
}

// Results of a tile's rows: U rows on their way per thread.  Forward: w, b = weight rstd and bias; backward: from shared memory.
template <typename T, int VEC, bool BACKWARD, int U>
__device__ __forceinline__ void tile_results(const TileArgs& a, const Tile& t, int32_t c, int ty, int n_ty, float mean, float rstd, float s1, float s2,
                                             float (&w)[VEC], float (&b)[VEC], const float* swr, const float* sb) {
    const int64_t x_step = (int64_t)n_ty * a.x_stride, d_step = (int64_t)n_ty * a.d_y_stride, out_step = (int64_t)n_ty * a.out_stride;
    const T* x = static_cast<const T*>(a.x) + (t.row0 + ty) * a.x_stride + c;
    const T* d_y = static_cast<const T*>(a.d_y) + (BACKWARD ? (t.row0 + ty) * a.d_y_stride + c : 0);
    T* out = static_cast<T*>(a.out) + (t.row0 + ty) * a.out_stride + c;
    const int32_t rows = (int32_t)(t.row1 - t.row0);
    const float k1 = -s1 * rstd, k2 = -s2 * rstd * rstd;
    for (int32_t r = ty; r < rows; r += U * n_ty) {
        Raw<T, VEC> raw[U], rd[BACKWARD ? U : 1];
        uint64_t key = 0;
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (r + k * n_ty < rows) {
                raw[k].load(x + k * x_step);
                if (BACKWARD) rd[k].load(d_y + k * d_step);
            }
        if (U == 1 && a.drop.on) key = drop_key(a.drop, t.row0 + r);   // (as for the sums)
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (r + k * n_ty >= rows) break;
            float f[VEC];
            if (U > 1 && a.drop.on) key = drop_key(a.drop, t.row0 + r + k * n_ty);
            if constexpr (BACKWARD) {   // rstd (dz w - mean(dz w) - hat mean(dz w hat))
                float xc[VEC];
                Params<VEC, 8, true>::read(swr, w);
                centred_grad<T, VEC>(a, raw[k], rd[k], key, c, mean, rstd, w, sb, xc, f);
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = fmaf(f[e], w[e], fmaf(xc[e], k2, k1));
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = fmaf(raw[k].get(e) - mean, w[e], b[e]);
                act_values<VEC>(a.act, f);
                drop_vector<VEC>(a.drop, key, c, f);
            }
            raw[k].put(f);
            raw[k].store(out + k * out_step);
        }
        x += U * x_step; out += U * out_step;
        if (BACKWARD) d_y += U * d_step;
    }
}

template <typename T, int VEC, bool BACKWARD, int U, int MINB>
__global__ void __launch_bounds__(kNormThreads, MINB) k_norm_results(const __grid_constant__ TileArgs a) {
    __shared__ __align__(16) float sw[BACKWARD ? kNormThreads * VEC : 4], sb[BACKWARD ? kNormThreads * VEC : 4];
    const int tx = threadIdx.x & ((1 << a.results.tx) - 1), ty = threadIdx.x >> a.results.tx, n_ty = kNormThreads >> a.results.tx;
    const int32_t part = (int32_t)blockIdx.x / a.results.chunks, c0 = ((int32_t)blockIdx.x - part * a.results.chunks) * (VEC << a.results.tx), c = c0 + tx * VEC;
    Tile t;
    locate_tile(a, part / a.parts_of_tile, &t);
    t.row0 += (int64_t)(part % a.parts_of_tile) * a.part_rows;
    t.row1 = min(t.row1, t.row0 + a.part_rows);
    if (t.row0 >= t.row1) return;   // (a sample's last tile has fewer rows)
    if (BACKWARD) share_params(a, t, sw, sb, c0, min(VEC << a.results.tx, a.channels - c0));
    chain_start();
    chain_wait();
    if (c >= a.channels) return;
    const int32_t group = c / a.each;
    const float mean = a.mean[(int64_t)t.sample * a.groups + group], rstd = a.rstd[(int64_t)t.sample * a.groups + group];
    float s1 = 0.f, s2 = 0.f, w[VEC], b[VEC];
    if (BACKWARD) {
        s1 = a.group_parts[(int64_t)t.sample * 2 * a.groups + group]; s2 = a.group_parts[((int64_t)t.sample * 2 + 1) * a.groups + group];
    } else {
        load_params<VEC>(a.weight, c, 1.f, w);
        load_params<VEC>(a.bias, c, 0.f, b);
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] *= rstd;
    }
    tile_results<T, VEC, BACKWARD, U>(a, t, c, ty, n_ty, mean, rstd, s1, s2, w, b, sw + tx * VEC, sb + tx * VEC);
}

// Samples that a block, or a cluster of blocks, goes through twice by itself (its second look finds them in L1 or L2): one launch.  The blocks of a
// cluster take equal shares of the rows and read each other's sums from shared memory.
constexpr int kBlockChannels = 1024, kBlockGroups = 256, kMaxCluster = 16;

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ float peer_value(const float* mine, uint32_t rank) {   // the same place in another block's shared memory
    uint32_t at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

template <typename T, int VEC, bool BACKWARD, bool CLUSTER, int K>
__global__ void __launch_bounds__(kNormThreads, 2) k_norm_block(const __grid_constant__ TileArgs a) {
    __shared__ __align__(16) float su[kNormThreads * VEC], sv[kNormThreads * VEC], sw[BACKWARD ? kBlockChannels : 4], sb[BACKWARD ? kBlockChannels : 4], acc[BACKWARD ? 2 * kBlockChannels : 4];
    __shared__ float sn[kNormThreads], g1[kBlockGroups], g2[kBlockGroups], part1[CLUSTER ? kBlockGroups : 1], part2[CLUSTER ? kBlockGroups : 1];
    const int tx = threadIdx.x & ((1 << a.results.tx) - 1), ty = threadIdx.x >> a.results.tx, n_ty = kNormThreads >> a.results.tx;
    const int32_t c = tx * VEC, size = CLUSTER ? (int32_t)cluster_size() : 1, rank = CLUSTER ? (int32_t)cluster_rank() : 0;
    const bool in = c < a.channels;
    const int32_t group = in ? c / a.each : 0;
    bool read = false;   // the others' sums have been: they may write theirs anew, or end, when all have
    for (int i = threadIdx.x; BACKWARD && i < 2 * a.channels; i += kNormThreads) acc[i] = 0.f;
    for (int32_t s = (int32_t)blockIdx.x / size; s < a.samples; s += (int32_t)gridDim.x / size) {
        Tile t;
        t.sample = s;
        const int64_t row0 = a.equal ? s * a.rows_per_sample : sample_entry(a, s).x;
        t.sample_rows = a.equal ? a.rows_per_sample : sample_entry(a, s + 1).x - row0;
        const int64_t stat = (int64_t)s * a.groups;
        if (t.sample_rows == 0) {
            for (int32_t g = threadIdx.x; !BACKWARD && g < a.groups; g += kNormThreads) { a.mean[stat + g] = 0.f; a.rstd[stat + g] = 0.f; }
            continue;
        }
        const int64_t share = (t.sample_rows + size - 1) / size;
        const auto start = [&](int32_t r) { return min(r * share, t.sample_rows); };
        t.row0 = row0 + start(rank);
        t.row1 = row0 + start(rank + 1);
        float mean = 0.f, rstd = 0.f, w[VEC], b[VEC];
        __syncthreads();   // (shared memory has been read)
        if (BACKWARD) {
            mean = a.mean[stat + group]; rstd = a.rstd[stat + group];
            share_params(a, t, sw, sb, 0, a.channels);
        }
        Pair<VEC> p;
        tile_sums<T, VEC, BACKWARD, K>(a, t, c, in, ty, n_ty, mean, rstd, sw + c, sb + c, p);
        block_pairs<VEC, BACKWARD>(p, su, sv, sn, a.results.tx, a.channels);
        for (int i = threadIdx.x; BACKWARD && i < a.channels; i += kNormThreads) { acc[i] += su[i]; acc[a.channels + i] += sv[i]; }
        const float values = (float)t.sample_rows * (float)a.each;
        const auto finish = [&](int32_t g, float u, float v) {
            if (BACKWARD) { g1[g] = v / values; g2[g] = u / values; }
            else {
                g1[g] = u; g2[g] = rsqrtf(v / values + a.eps);
                if (rank == 0) { a.mean[stat + g] = u; a.rstd[stat + g] = g2[g]; }
            }
        };
        if (CLUSTER && read) cluster_wait();
        run_groups<BACKWARD>(a, su, sv, 0, a.channels, (float)(t.row1 - t.row0), [&](int32_t g, float u, float v) {
            if (!CLUSTER) finish(g, u, v);
            else { part1[g] = u; part2[g] = v; }
        });
        if constexpr (CLUSTER) {
            cluster_arrive();
            cluster_wait();
            merge_sets<BACKWARD>(a, size, [&](int32_t i, int32_t) { return (float)(start(i + 1) - start(i)) * (float)a.each; },
                                 [&](int32_t i, int32_t g, float& u, float& v) { u = peer_value(part1 + g, i); v = peer_value(part2 + g, i); }, finish);
            cluster_arrive();
            read = true;
        }
        __syncthreads();
        if (!in) continue;
        if (!BACKWARD) {
            mean = g1[group]; rstd = g2[group];
            load_params<VEC>(a.weight, c, 1.f, w);
            load_params<VEC>(a.bias, c, 0.f, b);
#pragma unroll
            for (int e = 0; e < VEC; ++e) w[e] *= rstd;
        }
        tile_results<T, VEC, BACKWARD, K>(a, t, c, ty, n_ty, mean, rstd, g1[group], g2[group], w, b, sw + c, sb + c);
    }
    if (CLUSTER && read) cluster_wait();
    if (!BACKWARD || !a.parts) return;
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.channels; i += kNormThreads) a.parts[2 * (int64_t)blockIdx.x * a.channels + i] = acc[i];
}

// Many short samples that k_norm_block does not take (more channels or groups than its shared memory has room for, or rows that alignment cuts into more
// than one run of vectors): a block goes through a sample by itself, run after run of its channels, twice.  What groups and channels add up to lies in
// memory, by block and not by sample: a group that a run's end cuts is added up in the sample's statistics (backward: in the block's own place), the
// gradients of weight and bias in the block's part.
template <int VEC> constexpr int kWideBlocks = VEC == 8 ? 2 : 3;   // per SM, backward: what registers leave room for

template <typename T, int VEC, bool BACKWARD, int K, int MINB>
__global__ void __launch_bounds__(kNormThreads, MINB) k_norm_wide(const __grid_constant__ TileArgs a) {
    __shared__ __align__(16) float su[kNormThreads * VEC], sv[kNormThreads * VEC], sw[BACKWARD ? kNormThreads * VEC : 4], sb[BACKWARD ? kNormThreads * VEC : 4];
    __shared__ float sn[kNormThreads];
    const int tx = threadIdx.x & ((1 << a.results.tx) - 1), ty = threadIdx.x >> a.results.tx, n_ty = kNormThreads >> a.results.tx;
    float* const sums = BACKWARD ? a.group_parts + 2 * (int64_t)blockIdx.x * a.groups : nullptr;
    float* const part = BACKWARD && a.parts ? a.parts + 2 * (int64_t)blockIdx.x * a.channels : nullptr;
    bool first = true;
    for (int32_t s = (int32_t)blockIdx.x; s < a.samples; s += (int32_t)gridDim.x) {
        Tile t;
        t.sample = s;
        t.row0 = a.equal ? s * a.rows_per_sample : sample_entry(a, s).x;
        t.row1 = a.equal ? t.row0 + a.rows_per_sample : sample_entry(a, s + 1).x;
        const int64_t stat = (int64_t)s * a.groups;
        const float rows = (float)(t.row1 - t.row0), values = rows * (float)a.each;
        if (t.row0 == t.row1) {
            for (int32_t g = threadIdx.x; !BACKWARD && g < a.groups; g += kNormThreads) { a.mean[stat + g] = 0.f; a.rstd[stat + g] = 0.f; }
            continue;
        }
        float* const u_at = BACKWARD ? sums : a.mean + stat;
        float* const v_at = BACKWARD ? sums + a.groups : a.rstd + stat;
        for (int32_t c0 = 0; c0 < a.channels; c0 += a.run) {
            const int32_t c1 = min(c0 + a.run, a.channels), c = c0 + tx * VEC;
            const bool in = c < c1;
            float mean = 0.f, rstd = 0.f;
            __syncthreads();   // (shared memory has been read)
            if (BACKWARD) {
                const int64_t at = stat + (in ? c / a.each : 0);
                mean = a.mean[at]; rstd = a.rstd[at];
                share_params(a, t, sw, sb, c0, c1 - c0);
            }
            Pair<VEC> p;
            tile_sums<T, VEC, BACKWARD, K>(a, t, c, in, ty, n_ty, mean, rstd, sw + tx * VEC, sb + tx * VEC, p);
            float pu[BACKWARD ? VEC : 1], pv[BACKWARD ? VEC : 1];   // (what the part has: on its way while the block's threads meet)
            if (BACKWARD && part) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int i = threadIdx.x + j * kNormThreads;
                    pu[j] = pv[j] = 0.f;
                    if (!first && i < c1 - c0) { pu[j] = part[c0 + i]; pv[j] = part[a.channels + c0 + i]; }
                }
            }
            block_pairs<VEC, BACKWARD>(p, su, sv, sn, a.results.tx, c1 - c0);
            if (BACKWARD && part) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int i = threadIdx.x + j * kNormThreads;
                    if (i < c1 - c0) { part[c0 + i] = pu[j] + su[i]; part[a.channels + c0 + i] = pv[j] + sv[i]; }
                }
            }
            run_groups<BACKWARD>(a, su, sv, c0, c1, rows, [&](int32_t g, float u, float v) {
                const int32_t before = c0 - g * a.each;   // channels of the group in the runs before
                if (before > 0) {
                    float n = rows * (float)before, m = u_at[g], q = v_at[g];
                    if (BACKWARD) { m += u; q += v; }
                    else merge_moments(n, m, q, rows * (float)shared_channels(a, g, c0, c1), u, v);
                    u = m; v = q;
                }
                u_at[g] = u; v_at[g] = v;
            });
        }
        __syncthreads();
        for (int32_t g = threadIdx.x; g < a.groups; g += kNormThreads) {
            if (BACKWARD) { const float u = u_at[g]; u_at[g] = v_at[g] / values; v_at[g] = u / values; }   // mean of dz w, mean of dz w hat
            else v_at[g] = rsqrtf(v_at[g] / values + a.eps);
        }
        __syncthreads();
        for (int32_t c0 = 0; c0 < a.channels; c0 += a.run) {
            const int32_t c = c0 + tx * VEC;
            if (BACKWARD && a.run < a.channels) {   // (a single run's are still there)
                __syncthreads();
                share_params(a, t, sw, sb, c0, min(a.run, a.channels - c0));
            }
            if (c >= min(c0 + a.run, a.channels)) continue;
            const int32_t group = c / a.each;
            float w[VEC], b[VEC];
            const float mean = a.mean[stat + group], rstd = a.rstd[stat + group];
            if (!BACKWARD) {
                load_params<VEC>(a.weight, c, 1.f, w);
                load_params<VEC>(a.bias, c, 0.f, b);
#pragma unroll
                for (int e = 0; e < VEC; ++e) w[e] *= rstd;
            }
            tile_results<T, VEC, BACKWARD, K>(a, t, c, ty, n_ty, mean, rstd, BACKWARD ? u_at[group] : 0.f, BACKWARD ? v_at[group] : 0.f, w, b, sw + tx * VEC, sb + tx * VEC);
        }
        first = false;
    }
    for (int32_t i = threadIdx.x; part && first && i < 2 * a.channels; i += kNormThreads) part[i] = 0.f;   // (none of its samples has a row)
}

// Samples without rows have no tiles: their statistics are zero.
template <typename = void>
__global__ void k_norm_empty(const __grid_constant__ TileArgs a) {
    for (int32_t s = blockIdx.x; s < a.samples; s += gridDim.x) {
        if (sample_entry(a, s).x != sample_entry(a, s + 1).x) continue;
        for (int32_t g = threadIdx.x; g < a.groups; g += blockDim.x) { a.mean[(int64_t)s * a.groups + g] = 0.f; a.rstd[(int64_t)s * a.groups + g] = 0.f; }
    }
}

// behind a launch of this file's in the same stream (an error is found by cudaGetLastError)
template <typename... P, typename... A>
void launch_chained(dim3 grid, int threads, cudaStream_t st, void (*kernel)(P...), A... args) {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t how = {};
    how.gridDim = grid; how.blockDim = dim3((unsigned)threads); how.stream = st;
    how.attrs = &attr; how.numAttrs = 1;
    cudaLaunchKernelEx(&how, kernel, args...);
}

// what a translation unit of its own per row type launches
struct RowLaunch { int vec, nv, cut; bool backward; int grid; RowShape shape; };
struct TileLaunch { int vec, sums_vec; bool backward; int block_grid, cluster; };   // block_grid: of k_norm_block, or (no blocks to a sample's cluster) of k_norm_wide, or 0
template <typename T> void launch_dropout(int vec, const void* x, int64_t x_stride, void* y, int64_t y_stride, int64_t rows, int32_t channels, const DropArgs& d, int grid, cudaStream_t st);
template <typename T> void launch_rows(const RowLaunch& l, const NormArgs& a, cudaStream_t st);
template <typename T> void launch_tiles(const TileLaunch& l, const TileArgs& a, cudaStream_t st);

}  // namespace mgnorm
