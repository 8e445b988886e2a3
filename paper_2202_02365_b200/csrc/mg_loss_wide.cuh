// Wide rows of logits, forward: a block or a cluster of them goes along a row, whose vectors every thread has brought to places of its own in shared memory some rounds ahead:
// no registers wait for them, and no thread for another's.  8,192 bf16 rows of 32,000 against a teacher's 64 pairs: 91 us (5.8 TB/s), more where one follows the other at a lower clock;
// 4,096 of 50,257 with twenty best 109 to 119 (by box and clock), without 72 to 74.  Bound by instructions: five to seven a value (two for the conversion and the largest, one exponential at 16 a cycle and SM, sums in pairs)
// and 300 to 1,000 a warp and row.  Measured and taken back: vectors in registers, eight of them to a thread in segments (119; 143 with twenty best), the same by blocks that stay and ask for
// the next row's vectors early (141 - 230).
#pragma once

#include <float.h>

#include <cooperative_groups.h>

#include "mg_loss.cuh"

namespace mgloss {

constexpr int kWideThreads = 128, kWideLeastThreads = 64, kWideMostThreads = 1024;
constexpr int kWideAhead = 6;                      // vectors of a thread that are on their way (12 KB of a block of 128; with ten blocks to an SM more than the memory's latency asks for)
constexpr int kWideRoom = 512, kWideTrim = 64;     // pairs of vectors, and classes, that may be among the best: room; how many classes are cut down to the best again

// (places in shared memory by their 32-bit addresses)
__device__ __forceinline__ void copy_ahead(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ uint4 copied(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// blocks to an SM: 40 warps of the usual ones, 32 of the small
constexpr int wide_blocks(int threads) { return threads == kWideThreads ? 10 : threads == kWideLeastThreads ? 16 : 1; }

// packed values of one type: two halves to a word, or a float
template <typename T> struct Word {
    static constexpr int N = sizeof(T) == 4 ? 1 : 2;
    static __device__ __forceinline__ uint32_t least() { return sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00FC00u : 0xFF80FF80u; }   // -infinity
    static __device__ __forceinline__ uint32_t max(uint32_t a, uint32_t b) {   // (not a NaN where there is a number)
        if constexpr (sizeof(T) == 4) return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
        else {
            uint32_t r;
            if constexpr (std::is_same<T, __half>::value) asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
            else asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
            return r;
        }
    }
    static __device__ __forceinline__ void floats(uint32_t w, float* lo, float* hi) {
        if constexpr (std::is_same<T, __half>::value) {
            const float2 f = __half22float2(reinterpret_cast<const __half2&>(w));
            *lo = f.x; *hi = f.y;
        } else {
            *lo = __uint_as_float(w << 16); *hi = __uint_as_float(w & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ float largest(uint32_t w) {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w);
        else {
            float lo, hi;
            floats(w, &lo, &hi);
            return fmaxf(lo, hi);
        }
    }
};

// One thread's part of a row's sums, as it goes along, about a value that none of its own lies far above: where one comes that is more than 2^8 times as likely, what it has
// is scaled down.  (About the largest value itself, almost every vector early in a row would scale one lane's sums down.)
constexpr float kFarAbove = 8.f;
template <bool WEIGHTED> struct Running {
    float max = kNegInf;
    Pair sum = {0}, weighted = {0}, minus_max = {0};
    __device__ __forceinline__ void raise(float m, float scale2) {
        if (!((m - max) * scale2 > kFarAbove)) return;   // (a first number is infinitely far above)
        if (max != kNegInf) {
            const float by = (max - m) * scale2, f = fast_exp2(by);
            const Pair ff = pair(f, f);
            // sum 2^(y + by) (y + by)
            if (WEIGHTED) weighted = f == 0.f ? Pair{0} : mul2(ff, fma2(sum, pair(by, by), weighted));   // (0 times infinity, where `by` is that large)
            sum = mul2(ff, sum);
        }
        max = m;
        minus_max = pair(-m, -m);
    }
    __device__ __forceinline__ void add(float a, float b, Pair scale2) {
        const Pair y = mul2(add2(pair(a, b), minus_max), scale2);
        float y0, y1;
        split(y, &y0, &y1);
        const Pair e = pair(fast_exp2(y0), fast_exp2(y1));
        sum = add2(sum, e);
        if (WEIGHTED) weighted = fma2(e, pair(fmaxf(y0, kLeast), fmaxf(y1, kLeast)), weighted);
    }
    __device__ __forceinline__ RowSums both() const {
        float a, b, c, d;
        split(sum, &a, &b);
        split(weighted, &c, &d);
        return {max, a + b, c + d};
    }
};

// Sums about different values brought together about the largest of these: over the lanes of a warp, or over the first COUNT of them.
template <bool WEIGHTED, int COUNT>
__device__ __forceinline__ RowSums over_warp(RowSums a, float scale2) {
    const float m = warp_max(a.max), by = (a.max - m) * scale2;
    // (a part without a class has no sum; one with a NaN alone keeps it)
    const float f = a.max == kNegInf ? 1.f : fast_exp2(by);
    if (WEIGHTED) a.weighted = f == 0.f || a.max == kNegInf ? 0.f : f * fmaf(a.sum, by, a.weighted);   // sum 2^(y + by) (y + by)
    return {m, lanes_sum<COUNT>(a.sum * f), WEIGHTED ? lanes_sum<COUNT>(a.weighted) : 0.f};
}

// (ROOM: without best classes, none)
template <int THREADS, int ROOM> struct WideShared {
    static constexpr int WARPS = THREADS / 32;
    float max[WARPS], sum[WARPS], weighted[WARPS], scratch[WARPS];
    float all[3];                  // of the block: what others of its cluster read
    int n, n_best;                 // pairs of vectors, classes that may be among the best; more than there is room for: the best are found one by one
    float first[32], bound;        // the largest values of the threads' first vectors, a few of each warp; what lies below is not among the best (as far as is known)
    int32_t pairs[ROOM];
    uint64_t room[ROOM];           // a class and its value
    uint64_t best[MG_MAX_TOP], warp_best[WARPS];
};

// The `top` best of the keys to `best`, the best first (every thread; behind a barrier, and before one): each key's rank is counted, by up to eight neighbouring threads.
template <int THREADS>
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, int32_t top, uint64_t* best) {
    int share = 1;
    while (share < 8 && n * share * 2 <= THREADS) share *= 2;
    const int sub = (int)threadIdx.x & (share - 1);
    for (int i0 = 0; i0 < n; i0 += THREADS / share) {
        const int i = i0 + (int)threadIdx.x / share;
        const uint64_t key = i < n ? keys[i] : ~0ull;
        int rank = 0;
        if (i < n)
#pragma unroll 4
            for (int j = sub; j < n; j += share) rank += keys[j] > key;
        for (int o = 1; o < share; o *= 2) rank += __shfl_xor_sync(0xFFFFFFFFu, rank, o);
        if (i < n && sub == 0 && rank < top) best[rank] = key;
    }
}

// A value that no more than a few of the row's lie above, and `top` do not lie below: the top-th largest of the few largest that each warp's threads have found in their
// first vectors.  (full: warps all of whose threads have one.)
template <int THREADS, int ROOM>
__device__ __forceinline__ float first_bound(float own, int full, int32_t top, WideShared<THREADS, ROOM>* sh) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, use = max(min(full, 32), 1), each = min(32 / use, (top + use - 1) / use + 1);
    if (full <= 0 || each * use < top) {
        if (threadIdx.x == 0) sh->bound = kNegInf;
        __syncthreads();
        return kNegInf;
    }
    if (warp < use) {
        float left = own;
        for (int k = 0; k < each; ++k) {
            const float most = warp_max(left);
            const uint32_t holders = __ballot_sync(0xFFFFFFFFu, left == most);
            if (lane == __ffs(holders) - 1) left = kNegInf;
            if (lane == 0) sh->first[warp * each + k] = most;
        }
    }
    __syncthreads();
    if (warp == 0) {
        const float v = lanes_sorted<32>(lane < each * use ? sh->first[lane] : kNegInf);
        if (lane == top - 1) sh->bound = v;
    }
    __syncthreads();
    return sh->bound;
}

// the largest value of a vector, of each half of its words
template <typename T>
__device__ __forceinline__ uint32_t largest_of(const uint4& w) { return Word<T>::max(Word<T>::max(w.x, w.y), Word<T>::max(w.z, w.w)); }

// A row's part `part` of 2^parts_log2: its classes are vectors [lo, hi) of the cut, the first part's the edges too.  `meanwhile` is called when the first vectors are on their way.
// On return thread 0 .. all have the part's sums, and sh->best the part's best classes (zero where it has fewer).
template <typename T, int THREADS, int ROOM, bool WEIGHTED, bool EDGES, typename F>
__device__ __forceinline__ RowSums go_along(const T* x, int32_t classes, float scale2, int part, int parts_log2, int32_t top, WideShared<THREADS, ROOM>* sh, uint4* ring, F meanwhile) {
    constexpr int VEC = 16 / sizeof(T), WARPS = THREADS / 32;
    const Cut<VEC> cut(x, sizeof(T), classes);
    const int32_t lo = (int32_t)((int64_t)cut.vecs * part >> parts_log2), hi = (int32_t)((int64_t)cut.vecs * (part + 1) >> parts_log2);
    const int32_t count = hi - lo, rounds = (count + THREADS - 1) / THREADS;
    const char* from = reinterpret_cast<const char*>(x + cut.head) + ((int64_t)lo + (int32_t)threadIdx.x) * 16;
    constexpr uint32_t kStep = THREADS * 16, kRing = kWideAhead * kStep;
    const uint32_t first = (uint32_t)__cvta_generic_to_shared(ring) + threadIdx.x * 16, last = first + kRing;
#pragma unroll
    for (int i = 0; i < kWideAhead; ++i) {
        if (i * THREADS + (int32_t)threadIdx.x < count) copy_ahead(first + i * kStep, from + i * kStep);
        copies_end();
    }
    from += kRing;
    const bool has_edge = EDGES && part == 0 && (int)threadIdx.x < cut.edges;
    const Pair scales = pair(scale2, scale2);
    Running<WEIGHTED> run;
    float least = kNegInf;      // what lies below is not among the best
    float edge = kNegInf;
    if (has_edge) edge = to_float(x[cut.edge(threadIdx.x)]);
    meanwhile();
    if (top) {
        uint32_t all = Word<T>::least();
        copies_wait<0>();
#pragma unroll
        for (int i = 0; i < kWideAhead; ++i)
            if (i * THREADS + (int32_t)threadIdx.x < count) all = Word<T>::max(all, largest_of<T>(copied(first + i * kStep)));
        if (threadIdx.x == 0) { sh->n = 0; sh->n_best = 0; }
        least = first_bound<THREADS>(fmaxf(Word<T>::largest(all), edge), min(count / 32, WARPS), top, sh);
        least = fmaxf(least, -FLT_MAX);   // (classes that are not allowed come in by themselves, where the others are too few)
    }
    if (EDGES) {
        run.raise(edge, scale2);
        run.add(edge, kNegInf, scales);
    }
    const auto add = [&](const uint4& raw) {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int k = 0; k < 4; k += 3 - Word<T>::N) {
            float a, b;
            if constexpr (sizeof(T) == 4) { a = __uint_as_float(w[k]); b = __uint_as_float(w[k + 1]); }
            else Word<T>::floats(w[k], &a, &b);
            run.add(a, b, scales);
        }
    };
    // Which of the last 32 pairs of the thread's vectors may hold one of the best: their classes are collected behind these, by whichever threads.
    uint32_t flags = 0;
    const auto collect = [&](int32_t pair0) {
        for (; flags; flags &= flags - 1) {
            const int at = atomicAdd(&sh->n, 1);
            if (at < ROOM) sh->pairs[at] = (pair0 + __ffs(flags) - 1) * (2 * THREADS) + (int32_t)threadIdx.x;
        }
        __syncthreads();
        const int n = sh->n;
        if (n > ROOM) { if (threadIdx.x == 0) sh->n_best = ROOM + 1; }
        else
            for (int e = threadIdx.x; e < 2 * n; e += THREADS) {
                const int32_t v = sh->pairs[e >> 1] + (e & 1) * THREADS;
                if (v >= count) continue;
                const int32_t c = cut.head + (lo + v) * VEC;
                Raw<T, VEC> raw;
                raw.load(x + c);
                uint32_t some = 0;
#pragma unroll
                for (int k = 0; k < VEC; ++k) some |= (raw.get(k) >= least ? 1u : 0u) << k;
                for (; some; some &= some - 1) {
                    const int at = atomicAdd(&sh->n_best, 1);
                    if (at < ROOM) sh->room[at] = key_of(to_float(x[c + __ffs(some) - 1]), c + __ffs(some) - 1);
                }
            }
        __syncthreads();
    };
    uint32_t slot = first;
    int32_t i = 0;
    // two rounds at a time, as long as every thread has a vector in both
    for (const int32_t whole = count / THREADS; i + 2 <= whole; i += 2) {
        copies_wait<kWideAhead - 2>();
        const uint4 one = copied(slot), two = copied(slot + kStep);
        const float m = Word<T>::largest(Word<T>::max(largest_of<T>(one), largest_of<T>(two)));
        if (top && m >= least) flags |= 1u << (i / 2 % 32);
        run.raise(m, scale2);
        add(one);
        add(two);
        if (i + kWideAhead + 2 <= whole) {
            copy_ahead(slot, from);
            copy_ahead(slot + kStep, from + kStep);
        } else {
            const int32_t v = (i + kWideAhead) * THREADS + (int32_t)threadIdx.x;
            if (v < count) copy_ahead(slot, from);
            if (v + THREADS < count) copy_ahead(slot + kStep, from + kStep);
        }
        copies_end();
        copies_end();   // (a group for each round, as at the beginning and the end)
        from += 2 * kStep;
        slot += 2 * kStep;
        if (slot == last) slot = first;
        // long rows: behind 16, 32 and every 64 rounds, so that the bound keeps up with the row
        if (top && rounds > 32 && (i == 14 || i == 30 || i % 64 == 62) && i + 2 < rounds) {
            collect(i / 64 * 32);
            const int n = sh->n_best;
            if (n > kWideTrim && n <= ROOM) {
                rank_keys<THREADS>(sh->room, n, top, sh->best);
                __syncthreads();
                if ((int)threadIdx.x < top) sh->room[threadIdx.x] = sh->best[threadIdx.x];
                least = fmaxf(least, value_of((uint32_t)(sh->best[top - 1] >> 32)));
                if (threadIdx.x == 0) sh->bound = least;
            }
            __syncthreads();
            if (threadIdx.x == 0) { sh->n = 0; if (n > kWideTrim && n <= ROOM) sh->n_best = top; }
            __syncthreads();
        }
    }
    for (int32_t v = i * THREADS + (int32_t)threadIdx.x; i < rounds; ++i, v += THREADS) {
        copies_wait<kWideAhead - 1>();
        if (v < count) {
            const uint4 one = copied(slot);
            const float m = Word<T>::largest(largest_of<T>(one));
            if (top && m >= least) flags |= 1u << (i / 2 % 32);
            run.raise(m, scale2);
            add(one);
            if (v + kWideAhead * THREADS < count) copy_ahead(slot, from);
        }
        copies_end();
        from += kStep;
        slot += kStep;
        if (slot == last) slot = first;
    }
    // over the block, in an order that does not change
    RowSums r = over_warp<WEIGHTED, 32>(run.both(), scale2);
    if ((threadIdx.x & 31) == 0) { sh->max[threadIdx.x / 32] = r.max; sh->sum[threadIdx.x / 32] = r.sum; if (WEIGHTED) sh->weighted[threadIdx.x / 32] = r.weighted; }
    __syncthreads();
    if (threadIdx.x < 32) {
        const int w = threadIdx.x;
        r = {kNegInf, 0.f, 0.f};
        if (w < WARPS) r = {sh->max[w], sh->sum[w], WEIGHTED ? sh->weighted[w] : 0.f};
        r = over_warp<WEIGHTED, WARPS>(r, scale2);
        if (w == 0) { sh->all[0] = r.max; sh->all[1] = r.sum; sh->all[2] = r.weighted; }
    }
    if (top) {
        if (has_edge && edge >= least) {
            const int at = atomicAdd(&sh->n_best, 1);
            if (at < ROOM) sh->room[at] = key_of(edge, cut.edge(threadIdx.x));
        }
        collect((rounds - 1) / 64 * 32);
    }
    __syncthreads();
    r = {sh->all[0], sh->all[1], sh->all[2]};
    return r;
}

// The best of the part one by one, each a pass over it.
template <typename T, int THREADS>
__device__ __noinline__ void best_one_by_one(const T* x, int32_t classes, int part, int parts_log2, int32_t top, WideShared<THREADS, kWideRoom>* sh) {
    constexpr int VEC = 16 / sizeof(T), WARPS = THREADS / 32;
    const Cut<VEC> cut(x, sizeof(T), classes);
    const int32_t lo = (int32_t)((int64_t)cut.vecs * part >> parts_log2), hi = (int32_t)((int64_t)cut.vecs * (part + 1) >> parts_log2);
    uint64_t last = ~0ull;
    for (int k = 0; k < top; ++k) {
        uint64_t best = 0;
        for (int32_t c = cut.head + lo * VEC + (int32_t)threadIdx.x; c < cut.head + hi * VEC; c += THREADS) {
            const uint64_t key = key_of(to_float(x[c]), c);
            if (key < last && key > best) best = key;
        }
        if (part == 0 && (int)threadIdx.x < cut.edges) {
            const int32_t c = cut.edge(threadIdx.x);
            const uint64_t key = key_of(to_float(x[c]), c);
            if (key < last && key > best) best = key;
        }
        best = lanes_max<32>(best);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh->warp_best[threadIdx.x / 32] = best;
        __syncthreads();
        last = sh->warp_best[0];
        for (int w = 1; w < WARPS; ++w) last = max(last, sh->warp_best[w]);
        if (threadIdx.x == 0) sh->best[k] = last;   // (zero where the part has fewer classes)
        if (last == 0) last = 1;
    }
}

// The best of the part where its candidates are fewer than `top` or more than there is room for.  `anew`: the classes above the bound are looked for once more; where these have no
// room either, since values rise along the row, above one that goes by all of it.  What is still missing are the first of the classes at the bound: of those that are not allowed,
// where all others are too few.  4,096 bf16 rows of 50,257 equal values with twenty best 209 us (one by one
// 3,066), with ten classes allowed 92, fp32 rows that rise along their whole length 1,180.  Else (hundreds of NaN) one by one.
template <typename T, int THREADS>
__device__ __noinline__ void best_about_bound(const T* x, int32_t classes, int part, int parts_log2, int32_t top, bool anew, WideShared<THREADS, kWideRoom>* sh) {
    constexpr int VEC = 16 / sizeof(T), WARPS = THREADS / 32;
    const Cut<VEC> cut(x, sizeof(T), classes);
    const int32_t lo = (int32_t)((int64_t)cut.vecs * part >> parts_log2), hi = (int32_t)((int64_t)cut.vecs * (part + 1) >> parts_log2);
    const bool has_edge = part == 0 && (int)threadIdx.x < cut.edges;
    const float edge = has_edge ? to_float(x[cut.edge(threadIdx.x)]) : kNegInf;
    float bound = anew ? sh->bound : kNegInf;
    for (int go = 0; anew && go < 2; ++go) {
        __syncthreads();
        if (go) {
            float most = fmaxf(edge, kNegInf);   // (no NaN)
            for (int32_t v = lo + (int32_t)threadIdx.x; v < hi; v += THREADS) {
                Raw<T, VEC> raw;
                raw.load(x + cut.head + v * VEC);
#pragma unroll
                for (int k = 0; k < VEC; ++k) most = fmaxf(most, raw.get(k));
            }
            bound = first_bound<THREADS>(most, min((hi - lo) / 32, WARPS), top, sh);
        }
        if (threadIdx.x == 0) sh->n_best = 0;
        __syncthreads();
        const auto take = [&](float value, int32_t c) {
            const int at = atomicAdd(&sh->n_best, 1);
            if (at < kWideRoom) sh->room[at] = key_of(value, c);
        };
        for (int32_t v = lo + (int32_t)threadIdx.x; v < hi; v += THREADS) {
            Raw<T, VEC> raw;
            const int32_t c = cut.head + v * VEC;
            raw.load(x + c);
            uint32_t some = 0;
#pragma unroll
            for (int k = 0; k < VEC; ++k) some |= (raw.get(k) <= bound ? 0u : 1u) << k;   // (a NaN is above all)
            for (; some; some &= some - 1) take(to_float(x[c + __ffs(some) - 1]), c + __ffs(some) - 1);
        }
        if (has_edge && !(edge <= bound)) take(edge, cut.edge(threadIdx.x));
        __syncthreads();
        if (sh->n_best <= kWideRoom) break;
    }
    int have = sh->n_best;
    if (have > kWideRoom) return best_one_by_one<T, THREADS>(x, classes, part, parts_log2, top, sh);
    rank_keys<THREADS>(sh->room, have, top, sh->best);
    const uint32_t order = order_of(bound);
    const int32_t head = part == 0 ? cut.head : 0, inner = (hi - lo) * VEC, total = inner + (part == 0 ? cut.edges : 0);
    for (int32_t p0 = 0; p0 < total && have < top; p0 += THREADS) {
        const int32_t p = p0 + (int32_t)threadIdx.x, c = p < head ? p : p < head + inner ? cut.head + lo * VEC + (p - head) : p - inner + cut.vecs * VEC;
        const bool is = p < total && order_of(to_float(x[c])) == order;
        const uint32_t mask = __ballot_sync(0xFFFFFFFFu, is);
        if ((threadIdx.x & 31) == 0) sh->warp_best[threadIdx.x / 32] = __popc(mask);
        __syncthreads();
        int rank = have + __popc(mask & ((1u << (threadIdx.x & 31)) - 1));
        for (int w = 0; w < WARPS; ++w) {
            const int n = (int)sh->warp_best[w];
            have += n;
            if (w < (int)threadIdx.x / 32) rank += n;
        }
        if (is && rank < top) sh->best[rank] = (uint64_t)order << 32 | (uint32_t)~c;
        __syncthreads();
    }
    if ((int)threadIdx.x >= have && (int)threadIdx.x < top) sh->best[threadIdx.x] = 0;   // (the part has fewer classes)
}

// the parts' sums, in rank 0's hands
template <bool WEIGHTED, int THREADS, int ROOM>
__device__ __forceinline__ RowSums over_cluster(RowSums r, int parts, float scale2, WideShared<THREADS, ROOM>* sh) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    if (cluster.block_rank() == 0) {
        const int p = threadIdx.x & 31;
        r = {kNegInf, 0.f, 0.f};
        if (p < parts) {
            const float* from = cluster.map_shared_rank(sh->all, p);
            r = {from[0], from[1], from[2]};
        }
        r = over_warp<WEIGHTED, 16>(r, scale2);
        r = {r.max, __shfl_sync(0xFFFFFFFFu, r.sum, 0), __shfl_sync(0xFFFFFFFFu, r.weighted, 0)};
    }
    return r;
}

template <typename T, int THREADS, bool EDGES>
__global__ void __launch_bounds__(THREADS, wide_blocks(THREADS)) k_scores_wide(const __grid_constant__ ScoreArgs a, int parts_log2) {
    namespace cg = cooperative_groups;
    __shared__ WideShared<THREADS, kWideRoom> sh;
    extern __shared__ __align__(16) uint4 ring[];   // kWideAhead vectors of each thread
    const int parts = 1 << parts_log2;
    const int64_t r = blockIdx.x >> parts_log2;
    const int part = (int)(blockIdx.x & (unsigned)(parts - 1));
    const T* x = static_cast<const T*>(a.x) + r * a.stride;
    int32_t label = -1;
    float at_label = 0.f;
    RowSums s = go_along<T, THREADS, kWideRoom, true, EDGES>(x, a.classes, a.scale2, part, parts_log2, a.top, &sh, ring, [&] {
        if (threadIdx.x == 0 && part == 0 && a.log_prob) {
            label = class_at(a.labels, a.labels_are_i64, r, a.classes);
            if (label >= 0) at_label = to_float(x[label]);
        }
    });
    if (a.top) {
        const int n = sh.n_best;
        const bool anew = n > kWideRoom || !(s.sum < __builtin_huge_valf());
        if (!anew && n >= a.top) rank_keys<THREADS>(sh.room, n, a.top, sh.best);
        else best_about_bound<T, THREADS>(x, a.classes, part, parts_log2, a.top, anew, &sh);
        __syncthreads();
    }
    if (parts > 1) s = over_cluster<true>(s, parts, a.scale2, &sh);
    if (part == 0) {
        if (a.top && parts > 1) {
            cg::cluster_group cluster = cg::this_cluster();
            const int n = parts * a.top;      // (MG_MAX_TOP from each of 16 blocks: there is room)
            for (int i = threadIdx.x; i < n; i += THREADS) sh.room[i] = cluster.map_shared_rank(sh.best, i / a.top)[i % a.top];
            __syncthreads();
            rank_keys<THREADS>(sh.room, n, a.top, sh.best);
            __syncthreads();
        }
        if (threadIdx.x < 32) {
            const RowResult res(s, a.scale);
            if (threadIdx.x == 0) {
                if (a.lse) a.lse[r] = res.lse;
                if (a.entropy) a.entropy[r] = res.entropy;
                if (a.log_prob) a.log_prob[r] = label >= 0 ? res.log_p(at_label) : 0.f;
                if (a.row_sums) a.row_sums[r] = res.sums();
            }
            if ((int)threadIdx.x < a.top) {
                const uint64_t key = sh.best[threadIdx.x];
                if (a.top_ids) a.top_ids[r * a.top + threadIdx.x] = class_of(key);
                if (a.top_log_probs) a.top_log_probs[r * a.top + threadIdx.x] = res.log_p(value_of((uint32_t)(key >> 32)));
            }
        }
    }
    if (parts > 1) cg::this_cluster().sync();   // (nobody leaves while its memory is read)
}

// Over the first `warps` warps of a block, in their hands; barrier 1 is theirs.
__device__ __forceinline__ void some_warps_meet(int warps) {
    if (warps > 1) asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
    else __syncwarp();
}
template <typename F>
__device__ __forceinline__ float over_warps(float v, int warps, float* scratch, F f) {
    v = over_lanes<32>(v, f);
    if (warps == 1) return v;
    some_warps_meet(warps);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x / 32] = v;
    some_warps_meet(warps);
    v = scratch[0];
    for (int w = 1; w < warps; ++w) v = f(v, scratch[w]);
    return v;
}

// The warps that deal with a teacher's pairs: a pair to a thread, up to 256 threads, or as many as a block has; more pairs go round.
constexpr int kTeacherThreads = 256;
template <int THREADS> __device__ __forceinline__ int teacher_warps(const TeacherArgs& t) { return (min(t.entries, THREADS) + 31) / 32; }

// A teacher's row, by these warps: `above` [entries] in shared memory gets the values less `shift` (-infinity: not a pair), at_class the logits of their classes, where
// `wanted(class)`.  Each thread deals with the same pairs throughout.  A pair's probability is exp(above) part, its logarithm above - log_sum.
struct TeacherRow { float part, log_sum, mass; };   // mass: the probabilities' sum
template <int THREADS, typename T, typename F>
__device__ __forceinline__ TeacherRow teacher_row(const TeacherArgs& t, int64_t r, const T* x, int32_t classes, float scale, int warps, float* scratch, float* above, float* at_class, int32_t* c, F wanted) {
    float m = kNegInf;
    for (int k = threadIdx.x; k < t.entries; k += THREADS) {
        const int32_t of = class_at(t.ids, t.ids_are_i64, r * t.ids_stride + k, classes);
        const float v = of >= 0 ? scale * float_at(t.values, t.dtype, r * t.values_stride + k) : kNegInf;
        at_class[k] = of >= 0 && wanted(of) ? to_float(x[of]) : 0.f;
        above[k] = v;
        if (c) c[k] = of;
        m = fmaxf(m, v);
    }
    const float shift = t.lse ? t.lse[r] : centre(over_warps(m, warps, scratch, [](float a, float b) { return fmaxf(a, b); }));
    float sum = 0.f;
    for (int k = threadIdx.x; k < t.entries; k += THREADS) {
        above[k] = above_shift(above[k], shift);   // (what is no pair stays -infinity)
        sum += expf(above[k]);                     // (0 of -infinity)
    }
    sum = over_warps(sum, warps, scratch, [](float a, float b) { return a + b; });
    if (t.lse) return {1.f, 0.f, sum};
    return {sum == 0.f ? 0.f : 1.f / sum, logf(sum), sum == 0.f ? 0.f : sum * (1.f / sum)};
}

template <typename T, int THREADS, bool EDGES>
__global__ void __launch_bounds__(THREADS, wide_blocks(THREADS)) k_distill_wide(const __grid_constant__ ScoreArgs a, const __grid_constant__ TeacherArgs t, float* loss, int parts_log2) {
    namespace cg = cooperative_groups;
    __shared__ WideShared<THREADS, 1> sh;
    extern __shared__ __align__(16) uint4 ring[];   // kWideAhead vectors of each thread
    __shared__ float above[MG_MAX_TEACHER], at_class[MG_MAX_TEACHER];
    const int parts = 1 << parts_log2;
    const int64_t r = blockIdx.x >> parts_log2;
    const int part = (int)(blockIdx.x & (unsigned)(parts - 1));
    const T* x = static_cast<const T*>(a.x) + r * a.stride;
    constexpr int TEACHERS = THREADS < kTeacherThreads ? THREADS : kTeacherThreads;
    const int warps = teacher_warps<TEACHERS>(t);
    const bool teaches = part == 0 && (int)threadIdx.x < warps * 32;
    TeacherRow teacher{0.f, 0.f, 0.f};   // (while the row's first vectors are on their way)
    RowSums s = go_along<T, THREADS, 1, false, EDGES>(x, a.classes, a.scale2, part, parts_log2, 0, &sh, ring, [&] {
        if (teaches) teacher = teacher_row<TEACHERS>(t, r, x, a.classes, a.scale, warps, sh.scratch, above, at_class, nullptr, [](int32_t) { return true; });
    });
    if (parts > 1) s = over_cluster<false>(s, parts, a.scale2, &sh);
    if (teaches) {
        const RowResult res(s, a.scale);
        float v = 0.f;
        for (int k = threadIdx.x; k < t.entries; k += TEACHERS) {
            const float q = expf(above[k]) * teacher.part;
            if (q != 0.f) v = fmaf(q, (above[k] - teacher.log_sum) - res.log_p(at_class[k]), v);
        }
        v = over_warps(v, warps, sh.scratch, [](float a, float b) { return a + b; });
        if (threadIdx.x == 0) {
            loss[r] = v;
            if (a.lse) a.lse[r] = res.lse;
            if (a.row_sums) a.row_sums[r] = res.sums();
        }
    }
    if (parts > 1) cg::this_cluster().sync();
}

}  // namespace mgloss
