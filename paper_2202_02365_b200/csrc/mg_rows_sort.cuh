// The places of equal ids brought together: a radix sort of the ids by their places, eight bits at a time, each digit one kernel whose tiles look back at those
// before them.  All kernels for 543,000 ids of two million rows (three digits): 52 us, for 50,000 of 14,824 22; bound by launches and the waits for the tiles before.
#pragma once

#include "mg_norm_tiles.cuh"

namespace mgrows {

using mgnorm::chain_start;
using mgnorm::chain_wait;

constexpr int kSortThreads = 256, kSortWarps = kSortThreads / 32, kSortBits = 8, kSortBins = 1 << kSortBits, kMaxPasses = 4;

__device__ __forceinline__ int64_t id_at(const void* ids, int is_i64, int64_t i) {
    return is_i64 ? static_cast<const int64_t*>(ids)[i] : (int64_t)static_cast<const int32_t*>(ids)[i];
}
__device__ __forceinline__ uint32_t sort_key(const void* ids, int is_i64, int64_t i, uint32_t none) {
    const int64_t id = id_at(ids, is_i64, i);
    return id >= 0 && id < (int64_t)none ? (uint32_t)id : none;
}

// what the kernels of one call share, cleared before the first
struct SortShared {
    uint32_t hist[kMaxPasses][kSortBins];   // how often each digit occurs
    uint32_t ticket[kMaxPasses + 1];        // the next tile of a pass, of the groups
    uint32_t failed;                        // a bounded wait ran out
};

// Which lanes of the warp have the same digit (`ok`: that have one), by a vote for each of its bits: a match instruction takes some 70 cycles of an SM, where this takes six.
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, int bits, bool ok) {
    uint32_t peers = __ballot_sync(0xFFFFFFFFu, ok);
#pragma unroll
    for (int b = 0; b < kSortBits; ++b)
        if (b < bits) {
            const uint32_t votes = __ballot_sync(0xFFFFFFFFu, digit >> b & 1);
            peers &= digit >> b & 1 ? votes : ~votes;
        }
    return peers;
}

// (a warp whose digits are all the same adds them once: many of one id would wait for one another)
__global__ void __launch_bounds__(kSortThreads) k_sort_hist(const void* ids, int ids_are_i64, int64_t n, uint32_t none, int passes, int bits, SortShared* s) {
    __shared__ uint32_t sh[kMaxPasses][kSortBins];
    for (int p = 0; p < kMaxPasses; ++p) sh[p][threadIdx.x] = 0;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    constexpr int U = 4;
    for (int64_t j = (int64_t)blockIdx.x * kSortThreads * U; j < n; j += (int64_t)gridDim.x * kSortThreads * U) {
        uint32_t key[U];
#pragma unroll
        for (int u = 0; u < U; ++u) key[u] = j + u * kSortThreads + threadIdx.x < n ? sort_key(ids, ids_are_i64, j + u * kSortThreads + threadIdx.x, none) : 0u;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool ok = j + u * kSortThreads + threadIdx.x < n;
            for (int p = 0; p < passes; ++p) {
                const uint32_t digit = key[u] >> p * bits & ((1u << bits) - 1u), of_first = __shfl_sync(0xFFFFFFFFu, digit, 0);
                if (__all_sync(0xFFFFFFFFu, ok && digit == of_first)) { if (lane == 0) atomicAdd(&sh[p][digit], 32u); }
                else if (ok) atomicAdd(&sh[p][digit], 1u);
            }
        }
    }
    __syncthreads();
    for (int p = 0; p < passes; ++p)
        if (sh[p][threadIdx.x]) atomicAdd(&s->hist[p][threadIdx.x], sh[p][threadIdx.x]);
}

// One digit's pass: a tile's keys are ranked by digit, warp by warp and 32 at a time, laid out digit by digit in shared memory and written from there.  Where a digit's
// keys of this tile begin is the digit's first place, and what the tiles before it have of the digit: a word per tile and digit says the tile's own number, or that
// of all tiles up to it.  Tiles come from a counter, so those before are in running blocks and every wait ends; it is bounded all the same.
// (One word at a time: four at once, of which the later ones are mostly not there yet, took 38 us in the place of 35 for all the kernels of 150,001 ids, sixteen 57.)
constexpr uint64_t kOwn = 1ull << 32, kTotal = 2ull << 32;

template <int PER, bool FIRST>
__global__ void __launch_bounds__(kSortThreads) k_sort_pass(const void* ids, int ids_are_i64, const uint32_t* keys, const int32_t* places, int64_t n, uint32_t none, int pass, int bits,
                                                            SortShared* s, uint64_t* states, uint32_t* keys_to, int32_t* places_to, int max_polls) {
    constexpr int TILE = kSortThreads * PER;
    __shared__ uint32_t counts[kSortWarps][kSortBins];
    __shared__ uint32_t tile_base[kSortBins], warp_tot[kSortWarps];
    __shared__ int64_t glob_base[kSortBins];   // of the digit's keys in the output, less its first place in the tile
    __shared__ uint32_t stage_key[TILE];
    __shared__ int32_t stage_place[TILE];
    __shared__ uint32_t sh_tile;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, shift = pass * bits;
    const uint32_t mask = (1u << bits) - 1u;
    chain_wait();
    chain_start();
    if (threadIdx.x == 0) sh_tile = atomicAdd(&s->ticket[pass], 1u);
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) counts[w][threadIdx.x] = 0;
    __syncthreads();
    const int64_t tile = sh_tile, base = tile * TILE;
    const int tile_n = (int)min((int64_t)TILE, n - base);
    uint32_t key[PER], rank[PER];
    int32_t place[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int at = (warp * PER + k) * 32 + lane;
        key[k] = 0; place[k] = 0;
        if (at < tile_n) {
            if (FIRST) { key[k] = sort_key(ids, ids_are_i64, base + at, none); place[k] = (int32_t)(base + at); }
            else { key[k] = keys[base + at]; place[k] = places[base + at]; }
        }
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const bool ok = (warp * PER + k) * 32 + lane < tile_n;
        const uint32_t digit = key[k] >> shift & mask, peers = same_digit(digit, bits, ok);
        const int leader = __ffs(peers) - 1;
        uint32_t old = 0;
        if (ok && lane == leader) { old = counts[warp][digit]; counts[warp][digit] = old + __popc(peers); }
        old = __shfl_sync(0xFFFFFFFFu, old, leader);
        rank[k] = old + __popc(peers & ((1u << lane) - 1u));
        __syncwarp();
    }
    __syncthreads();
    // thread = digit: what the warps before have of it, the tile's number, told to the tiles behind
    uint32_t own = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) { const uint32_t c = counts[w][threadIdx.x]; counts[w][threadIdx.x] = own; own += c; }
    volatile uint64_t* state = states + threadIdx.x;
    if (tile > 0) state[tile * kSortBins] = kOwn | own;
    else state[0] = kTotal | own;
    const uint32_t all = s->hist[pass][threadIdx.x], inc = warp_incl_scan(own), all_inc = warp_incl_scan(all);
    __shared__ uint32_t warp_all[kSortWarps];
    if (lane == 31) { warp_tot[warp] = inc; warp_all[warp] = all_inc; }
    __syncthreads();
    uint32_t in_tile = inc - own, before = 0;
    int64_t first = (int64_t)(all_inc - all);
    for (int w = 0; w < warp; ++w) { in_tile += warp_tot[w]; first += warp_all[w]; }
    bool known = tile == 0;
    int polls = 0;
    for (int64_t back = tile - 1; !known && polls < max_polls;) {
        const uint64_t told = state[back * kSortBins];
        if (!(told >> 32)) { ++polls; continue; }
        before += (uint32_t)told;
        known = (told & kTotal) != 0;   // (tile 0 says so)
        --back;
        polls = 0;
    }
    if (!known) atomicExch(&s->failed, 1u);
    if (tile > 0) state[tile * kSortBins] = kTotal | (uint64_t)(before + own);
    first += before;
    tile_base[threadIdx.x] = in_tile;
    glob_base[threadIdx.x] = first - in_tile;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if ((warp * PER + k) * 32 + lane < tile_n) {
            const uint32_t digit = key[k] >> shift & mask, at = tile_base[digit] + counts[warp][digit] + rank[k];
            stage_key[at] = key[k];
            stage_place[at] = place[k];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < tile_n; i += kSortThreads) {
        const uint32_t k = stage_key[i];
        const int64_t to = glob_base[k >> shift & mask] + i;
        if (to >= 0 && to < n) { keys_to[to] = k; places_to[to] = stage_place[i]; }   // (always, unless a wait ran out)
    }
}

// Where the sorted ids change: groups are numbered through, a tile looking back for how many there are before it.
template <int PER>
__global__ void __launch_bounds__(kSortThreads) k_sort_groups(const uint32_t* keys, int64_t n, uint32_t none, SortShared* s, uint64_t* states, int ids_are_i64, void* group_ids, int32_t* starts,
                                                              int32_t* group_of, int32_t* n_groups, int max_polls) {
    constexpr int TILE = kSortThreads * PER;
    __shared__ uint32_t warp_tot[kSortWarps], sh_tile, sh_before;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const auto say = [&](int32_t count) {   // -1 where a wait has run out, here or in the sort, or does so later
        volatile int32_t* to = n_groups;
        *to = count;
        __threadfence();
        if (*reinterpret_cast<volatile uint32_t*>(&s->failed)) *to = -1;
    };
    chain_wait();
    chain_start();
    if (threadIdx.x == 0) sh_tile = atomicAdd(&s->ticket[kMaxPasses], 1u);
    __syncthreads();
    const int64_t tile = sh_tile, base = tile * TILE + warp * PER * 32;
    uint32_t key[PER], heads[PER], mine = 0;
    uint32_t last = base > 0 && base - 1 < n ? keys[base - 1] : none;   // (the id before the first is like none; a group of `none` is not one)
#pragma unroll
    for (int k = 0; k < PER; ++k) key[k] = base + k * 32 + lane < n ? keys[base + k * 32 + lane] : none;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        uint32_t prev = __shfl_up_sync(0xFFFFFFFFu, key[k], 1);
        if (lane == 0) prev = last;
        last = __shfl_sync(0xFFFFFFFFu, key[k], 31);
        heads[k] = __ballot_sync(0xFFFFFFFFu, key[k] != none && (prev != key[k] || base + k * 32 + lane == 0));
        mine += __popc(heads[k]);
    }
    if (lane == 0) warp_tot[warp] = mine;
    __syncthreads();
    if (warp == 0) {
        uint32_t total = 0;
        for (int w = 0; w < kSortWarps; ++w) total += warp_tot[w];
        bool gave_up = false;
        const uint32_t before = chain_tiles(states, (int32_t)tile, 1ull << 34, 0u, total, max_polls, &gave_up);
        if (lane == 0) sh_before = before;
        if (__any_sync(0xFFFFFFFFu, gave_up) && lane == 0) {   // (each lane waits for a tile of its own)
            atomicExch(&s->failed, 1u);
            __threadfence();
            *reinterpret_cast<volatile int32_t*>(n_groups) = -1;
        }
    }
    __syncthreads();
    uint32_t g = sh_before;   // groups that begin before the place
    for (int w = 0; w < warp; ++w) g += warp_tot[w];
    const int64_t room = min(n, (int64_t)none);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int64_t i = base + k * 32 + lane;
        const uint32_t to = g + __popc(heads[k] & (0xFFFFFFFFu >> (31 - lane)));   // ... up to the place itself
        g += __popc(heads[k]);
        if (i >= n) continue;
        group_of[i] = key[k] != none ? (int32_t)to - 1 : -1;
        if (key[k] == none) continue;
        if ((heads[k] >> lane & 1) && (int64_t)to <= room) {
            starts[to - 1] = (int32_t)i;
            if (ids_are_i64) static_cast<int64_t*>(group_ids)[to - 1] = key[k];
            else static_cast<int32_t*>(group_ids)[to - 1] = (int32_t)key[k];
        }
        if (i + 1 == n || keys[i + 1] == none) {   // the last place of the last group
            if ((int64_t)to <= room) starts[to] = (int32_t)i + 1;
            say((int32_t)to);
        }
    }
    if (tile == 0 && threadIdx.x == 0 && keys[0] == none) { starts[0] = 0; say(0); }
}

// All of it in one block: few ids, whose sort by several kernels is launches and waits.  An id with its place below it to a thread, sorted by a bitonic network: steps within a
// warp by shuffles, others through shared memory.  1,000 ids 7 us, where the kernels above take 19; 4,000, four to a thread, took 44 (one SM's instructions), so they are not taken.
constexpr int kSmallIds = 1024;
__global__ void __launch_bounds__(kSmallIds) k_sort_small(const void* ids, int ids_are_i64, int32_t n, uint32_t none, int32_t* order, int32_t* group_of, void* group_ids, int32_t* starts,
                                                          int32_t* n_groups) {
    __shared__ uint64_t item[kSmallIds];
    __shared__ uint32_t warp_tot[32];
    const int32_t i = threadIdx.x;
    uint64_t v = i < n ? (uint64_t)sort_key(ids, ids_are_i64, i, none) << 32 | (uint32_t)i : ~0ull;
    for (int32_t k = 2; k <= kSmallIds; k *= 2)
        for (int32_t j = k / 2; j; j /= 2) {
            uint64_t other;
            if (j >= 32) {
                __syncthreads();
                item[i] = v;
                __syncthreads();
                other = item[i ^ j];
            } else other = __shfl_xor_sync(0xFFFFFFFFu, (unsigned long long)v, j);
            v = ((i & j) == 0) == ((i & k) == 0) ? min(v, other) : max(v, other);
        }
    __syncthreads();
    item[i] = v;
    __syncthreads();
    // groups, as in k_sort_groups
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t key = i < n ? (uint32_t)(v >> 32) : none;
    const uint32_t heads = __ballot_sync(0xFFFFFFFFu, key != none && (i == 0 || (uint32_t)(item[i - 1] >> 32) != key));
    if (lane == 0) warp_tot[warp] = __popc(heads);
    __syncthreads();
    uint32_t to = __popc(heads & (0xFFFFFFFFu >> (31 - lane)));   // groups that begin up to the place
    for (int w = 0; w < warp; ++w) to += warp_tot[w];
    if (i == 0 && key == none) { starts[0] = 0; *n_groups = 0; }
    if (i >= n) return;
    order[i] = (int32_t)(uint32_t)v;
    group_of[i] = key != none ? (int32_t)to - 1 : -1;
    if (key == none) return;
    if (heads >> lane & 1) {
        starts[to - 1] = i;
        if (ids_are_i64) static_cast<int64_t*>(group_ids)[to - 1] = key;
        else static_cast<int32_t*>(group_ids)[to - 1] = (int32_t)key;
    }
    if (i + 1 == n || (uint32_t)(item[i + 1] >> 32) == none) { starts[to] = i + 1; *n_groups = (int32_t)to; }
}

}  // namespace mgrows
