// Group norm of samples of many rows whose rows are whole 16-byte pieces: one block per SM keeps tiles of rows in a ring of shared-memory slots
// that asynchronous copies fill.  A tile's sums are taken, the tile stays where it is until its sample's statistics are there, and the result
// is computed from it: the rows are read once where the samples under way fit the SMs' shared memory together (28 MB), and again (from L2, or
// from memory) where they do not.
//
// Every tile comes from one counter and belongs to the block that took it.  No block waits before it has taken what it can: a tile whose slot is
// wanted for another's sums is given up, and read again later.  So the blocks need not run at the same time, and every sample's sums arrive;
// the waits are bounded all the same.
//
// Warps 0 .. 15 work on commands (sums of a tile, result of a tile); warp 16 decides what comes next, takes tiles and starts copies; warps 17 .. 19
// take the finished sums in turn, hand them to the other blocks and bring those of a sample together.  The last four spend their time waiting
// for round trips through L2, about a microsecond each, which the first sixteen so do not see.
#pragma once

#include "mg_norm_tiles.cuh"
#include "mg_tcgen05.cuh"

namespace mgnorm {

constexpr int kRingThreads = 512, kRingWarps = kRingThreads / 32, kRingBlock = kRingThreads + 128;
constexpr int kRingSlots = 16, kRingCmds = 16;
constexpr int kRingHands = 3, kRingSums = 2 * kRingHands;   // warps that finished sums go to; tiles whose sums may wait for them
constexpr int kRingFifo = 1280;             // tiles that a block has taken and not finished: more than a sample has (kFan * kFan), so that the oldest
                                            // one's sample has been taken whole when it is full
constexpr int kRingSharedBytes = 227 << 10;

enum { CMD_SUMS = 0, CMD_RESULT = 1, CMD_EXIT = 2 };
enum { PART_FIRST = 1, PART_LAST = 2 };     // of a tile's pieces (a tile of one slot is one piece)

struct RingCmd {
    int32_t kind, slot, rows, part;
    int32_t wait;            // 0: the slot is filled; else 1 + the parity of its copy
    int32_t tile, sample, pad;
    int64_t row0;
};

struct RingArgs : TileArgs {
    int32_t total = 0;       // tiles
    int32_t slots = 0;
    int32_t sub_rows = 0;    // rows of a slot
    int32_t fan = 0;         // tiles whose sums are brought together at once
    int32_t hold = 0;        // tiles are of one slot, and stay in it
    int32_t patience = 0;    // polls before a slot is given up
    int32_t slot_bytes = 0, d_y_at = 0, keys_at = 0;   // of a slot; where dy's rows and the keys start in it
    // (tile_parts and fan_parts: [..][2][groups]; parts: the tiles' sums by channel)
};

struct RingShared {
    uint64_t full[kRingSlots], cmd_full[kRingCmds], cmd_done[kRingCmds];
    RingCmd cmd[kRingCmds];
    volatile int32_t passed[kRingHands];    // commands that a hand is through with ...
    volatile int32_t taken[kRingHands];     // ... and its finished sums among them
    volatile int32_t failed;
    int32_t held[kRingSlots];               // the tile that a slot keeps; -1: free, -2: in use
    int32_t fifo[kRingFifo];
};

// shared memory: RingShared, ring_pairs' scratch, the finished sums by channel ([kRingSums][2][channels]), the slots
__host__ __device__ constexpr int ring_scratch_at() { return (int)(sizeof(RingShared) + 127) / 128 * 128; }
__host__ __device__ constexpr int ring_sums_at(int vec) { return ring_scratch_at() + ((kRingThreads * vec + kRingWarps) * (int)sizeof(float) + 127) / 128 * 128; }
__host__ __device__ constexpr int ring_fixed_bytes(int vec, int channels) { return ring_sums_at(vec) + (kRingSums * 2 * channels * (int)sizeof(float) + 127) / 128 * 128; }

__device__ __forceinline__ void ring_sync() { asm volatile("bar.sync 1, 512;" ::: "memory"); }
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {   // (does not wait: mbarrier.try_wait may, for microseconds)
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(tc::smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}

__device__ __forceinline__ void ring_fail(const RingArgs& a, RingShared* sh) {
    sh->failed = 1;
    tc::report(a.status, kRoleNorm);
}

// the next command; longer than the block that gives it out waits for anything
__device__ __forceinline__ bool ring_next(RingShared* sh, int at, int parity) {
    if (tc::mbar_try_wait(&sh->cmd_full[at], parity)) return true;
    const long long t0 = clock64();
    while (!tc::mbar_try_wait(&sh->cmd_full[at], parity))
        if (clock64() - t0 > 8 * tc::kWaitCycles) return false;
    return true;
}

// how a sample's tiles are brought together
struct Fans { int64_t first_id; int32_t n; };
__device__ __forceinline__ Fans fans_of(const RingArgs& a, const Tile& t) { return {(int64_t)(t.first / a.fan + t.sample), (t.tiles + a.fan - 1) / a.fan}; }

// ---- warp 16 ----------------------------------------------------------------------------
// (all lanes go the same way: what may differ between them is read by one and handed round)
template <typename T, bool BACKWARD>
struct RingLead {
    const RingArgs& a;
    RingShared* sh;
    char* slots;
    const int lane;
    int head = 0, tail = 0, sums = 0;
    uint32_t phases = 0;                     // parity of each slot's next copy
    long long last = 0;

    __device__ __forceinline__ RingLead(const RingArgs& a_, RingShared* sh_, char* slots_) : a(a_), sh(sh_), slots(slots_), lane(threadIdx.x & 31) {}
    __device__ __forceinline__ int one(int v) const { return __shfl_sync(0xFFFFFFFFu, v, 0); }
    __device__ __forceinline__ void emit(const RingCmd& c) {
        if (lane == 0) {
            sh->cmd[head % kRingCmds] = c;
            asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(tc::smem_u32(&sh->cmd_full[head % kRingCmds])) : "memory");
        }
        ++head;
        last = clock64();
    }
    __device__ __forceinline__ void set_held(int slot, int32_t v) {
        __syncwarp();
        if (lane == 0) sh->held[slot] = v;
        __syncwarp();
    }
    // copies of `rows` rows into the slot; 1 + the parity to wait for
    __device__ __forceinline__ int load(int slot, int64_t row0, int32_t rows) {
        char* to = slots + (int64_t)slot * a.slot_bytes;
        uint64_t* bar = &sh->full[slot];
        const int64_t row_bytes = (int64_t)a.channels * sizeof(T);
        if (lane == 0) tc::mbar_expect_tx(bar, (uint32_t)(rows * row_bytes) * (BACKWARD ? 2 : 1));
        __syncwarp();
        for (int q = 0; q < (BACKWARD ? 2 : 1); ++q) {
            const char* from = static_cast<const char*>(q ? a.d_y : a.x);
            const int64_t stride = (q ? a.d_y_stride : a.x_stride) * (int64_t)sizeof(T);
            char* at = to + (q ? a.d_y_at : 0);
            if (stride == row_bytes) {
                if (lane == 0) tc::bulk_load(at, from + row0 * row_bytes, (uint32_t)(rows * row_bytes), bar);
            } else {
                for (int32_t r = lane; r < rows; r += 32) tc::bulk_load(at + r * row_bytes, from + (row0 + r) * stride, (uint32_t)row_bytes, bar);
            }
        }
        if (a.drop.on && a.drop.keys) {
            for (int32_t r = lane; r < rows; r += 32)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(tc::smem_u32(to + a.keys_at + 8 * r)), "l"(a.drop.keys + row0 + r) : "memory");
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(tc::smem_u32(bar)) : "memory");
        }
        const int wait = 1 + (int)(phases >> slot & 1u);
        phases ^= 1u << slot;
        return wait;
    }
    __device__ __forceinline__ void completions() {   // slots of finished commands
        while (tail < head && one(lane == 0 ? (int)mbar_test(&sh->cmd_done[tail % kRingCmds], tail / kRingCmds & 1) : 0)) {
            if (lane == 0) {
                const RingCmd& c = sh->cmd[tail % kRingCmds];
                if (c.kind == CMD_RESULT || !a.hold) sh->held[c.slot] = -1;
            }
            __syncwarp();
            ++tail;
            last = clock64();
        }
    }
    __device__ __forceinline__ bool gave_up() { return one(lane == 0 ? (int)(sh->failed || clock64() - last > tc::kWaitCycles) : 0); }
    __device__ __forceinline__ bool room() {
        return head - tail < kRingCmds && __all_sync(0xFFFFFFFFu, lane >= kRingHands || head - sh->passed[lane < kRingHands ? lane : 0] < kRingCmds);
    }
    // may the sums of another tile be waiting? (its hand is through with those before the last but one)
    __device__ __forceinline__ bool sums_room() { return one(lane == 0 ? (int)(sums / kRingHands - sh->taken[sums % kRingHands] < kRingSums / kRingHands) : 0); }
    // the slot that keeps tile `v`, or is free (-1), or -1
    __device__ __forceinline__ int slot_with(int32_t v) {
        const uint32_t with = __ballot_sync(0xFFFFFFFFu, lane < a.slots && sh->held[lane & (kRingSlots - 1)] == v);
        return with ? __ffs(with) - 1 : -1;
    }
    __device__ __forceinline__ bool ready(int32_t sample) {
        const bool r = one(lane == 0 ? (int)*reinterpret_cast<volatile uint32_t*>(a.ready + sample) : 0);
        if (r) __threadfence();
        return r;
    }
    __device__ __forceinline__ void work() {
        int fifo_head = 0, fifo_tail = 0, known_ready = -1, newest = -1, ticket = 0, tickets_left = 0, waited = 0, since = 0;
        int64_t result_row = -1, sums_row = -1;   // where a tile of several pieces goes on
        bool more = true, have_oldest = false;
        Tile oldest, taken;
        last = clock64();
        while (true) {
            completions();
            if (gave_up()) { if (lane == 0) ring_fail(a, sh); break; }   // (copies under way are waited for by the commands that want them)
            if (!room()) continue;
            if (!have_oldest && fifo_head != fifo_tail) {
                locate_tile(a, sh->fifo[fifo_head % kRingFifo], &oldest);
                have_oldest = true;
                result_row = oldest.row0;
            }
            const int free_slot = slot_with(-1);
            // another piece of a tile whose sums have been begun: its pieces come one behind the other, a thread keeps its sums between them
            // (the other way round, a new tile, only where there is no result to compute)
            const bool result = sums_row < 0 && have_oldest && known_ready == oldest.sample;
            if (result) {
                int slot = a.hold ? slot_with(oldest.tile) : -1;
                const bool kept = slot >= 0;
                if (!kept) slot = free_slot;
                if (slot >= 0) {
                    RingCmd c{CMD_RESULT, slot, 0, 0, 0, oldest.tile, oldest.sample, 0, result_row};
                    c.rows = (int32_t)min((int64_t)a.sub_rows, oldest.row1 - result_row);
                    if (!kept) c.wait = load(slot, result_row, c.rows);
                    set_held(slot, -2);
                    emit(c);
                    result_row += c.rows;
                    if (result_row == oldest.row1) { ++fifo_head; have_oldest = false; }
                    waited = 0;
                    continue;
                }
            }
            // has the oldest tile's sample come together?  It may have once all of it has been taken.  (Not before every fourth tile: a poll takes
            // as long as a tile's copy.)
            if (have_oldest && known_ready != oldest.sample && (free_slot < 0 || !more || (newest != oldest.sample && ++since >= 4))) {
                since = 0;
                if (ready(oldest.sample)) { known_ready = oldest.sample; continue; }
            }
            if (free_slot >= 0 && (sums_row >= 0 || (more && fifo_tail - fifo_head < kRingFifo && sums_room()))) {
                if (sums_row < 0) {
                    if (tickets_left == 0) {
                        tickets_left = a.total > 16 * (int)gridDim.x ? 2 : 1;
                        ticket = one(lane == 0 ? (int)atomicAdd(a.ticket, (uint32_t)tickets_left) : 0);
                    }
                    if (ticket >= a.total) { more = false; continue; }
                    locate_tile(a, ticket, &taken);
                    ++ticket; --tickets_left;
                    newest = taken.sample;
                    sums_row = taken.row0;
                }
                RingCmd c{CMD_SUMS, free_slot, (int32_t)min((int64_t)a.sub_rows, taken.row1 - sums_row), 0, 0, taken.tile, taken.sample, 0, sums_row};
                c.part = (sums_row == taken.row0 ? PART_FIRST : 0) | (sums_row + c.rows == taken.row1 ? PART_LAST : 0);
                c.wait = load(free_slot, c.row0, c.rows);
                set_held(free_slot, a.hold ? taken.tile : -2);
                emit(c);
                sums_row += c.rows;
                if (sums_row == taken.row1) {
                    sums_row = -1;
                    ++sums;
                    if (lane == 0) sh->fifo[fifo_tail % kRingFifo] = taken.tile;
                    __syncwarp();
                    ++fifo_tail;
                }
                waited = 0;
                continue;
            }
            if (!more && fifo_head == fifo_tail && head == tail) break;
            // every slot keeps a tile whose sample has not come together: the latest is given up for tiles that may be missing
            if (free_slot < 0 && more && a.hold && head == tail && ++waited > a.patience) {
                waited = 0;
                const int32_t mine = lane < a.slots ? sh->held[lane & (kRingSlots - 1)] : -2, latest = __reduce_max_sync(0xFFFFFFFFu, mine);
                const int give = slot_with(latest);
                if (latest >= 0 && give >= 0) set_held(give, -1);
            }
        }
        const long long t0 = clock64();
        while (!room() && one(lane == 0 ? (int)(clock64() - t0 < tc::kWaitCycles) : 0)) completions();
        if (head - tail < kRingCmds) emit(RingCmd{CMD_EXIT, 0, 0, 0, 0, 0, 0, 0, 0});
    }
};

// ---- warps 17 .. 19 ---------------------------------------------------------------------
// `n` sets of the groups' moments that lie one behind the other, values_of(i) values each, into `out`: lanes share a group where there are fewer than
// lanes, a lane's sets are on their way together
template <bool BACKWARD, typename Values>
__device__ __forceinline__ void hand_merge(const RingArgs& a, const float* parts, int32_t n, Values values_of, float* out) {
    const int lane = threadIdx.x & 31;
    const int64_t step = 2 * (int64_t)a.groups;
    int per = 1;
    while (per < 32 && 2 * per * a.groups <= 32) per *= 2;
    const int across = 32 / per, slice = lane / across;
    for (int32_t g0 = 0; g0 < a.groups; g0 += across) {
        const int32_t g = min(g0 + lane % across, a.groups - 1);
        float m = 0.f, u = 0.f, v = 0.f;
        constexpr int B = 8;
        for (int32_t i0 = slice; i0 < n; i0 += B * per) {
            float pu[B], pv[B];
#pragma unroll
            for (int k = 0; k < B; ++k) {
                const float* from = parts + min(i0 + k * per, n - 1) * step + g;
                pu[k] = __ldcg(from); pv[k] = __ldcg(from + a.groups);
            }
#pragma unroll
            for (int k = 0; k < B; ++k) {
                if (i0 + k * per >= n) break;
                if (BACKWARD) { u += pu[k]; v += pv[k]; }
                else merge_moments(m, u, v, values_of(i0 + k * per), pu[k], pv[k]);
            }
        }
        for (int o = across; o < 32; o <<= 1) {
            const float mb = __shfl_xor_sync(0xFFFFFFFFu, m, o), ub = __shfl_xor_sync(0xFFFFFFFFu, u, o), vb = __shfl_xor_sync(0xFFFFFFFFu, v, o);
            if (BACKWARD) { u += ub; v += vb; }
            else if (lane & o) { float x = mb, y = ub, z = vb; merge_moments(x, y, z, m, u, v); m = x; u = y; v = z; }   // (the lower lanes' set first)
            else merge_moments(m, u, v, mb, ub, vb);
        }
        if (slice == 0 && g0 + lane < a.groups) { __stcg(out + g, u); __stcg(out + a.groups + g, v); }
    }
}

template <bool BACKWARD>
__device__ __forceinline__ void ring_hand(const RingArgs& a, RingShared* sh, const float* sums, int hand) {
    const int lane = threadIdx.x & 31;
    const int64_t step = 2 * (int64_t)a.groups;
    const auto one = [](int v) { return __shfl_sync(0xFFFFFFFFu, v, 0); };
    int32_t seen = 0;   // tiles' sums among the commands
    for (int n = 0;; ++n) {
        const int at = n % kRingCmds, parity = n / kRingCmds & 1;
        if (!__all_sync(0xFFFFFFFFu, ring_next(sh, at, parity))) { ring_fail(a, sh); return; }
        const int32_t kind = sh->cmd[at].kind, part = sh->cmd[at].part, tile = sh->cmd[at].tile;
        if (kind == CMD_EXIT) return;
        const bool last = kind == CMD_SUMS && (part & PART_LAST), mine = last && seen % kRingHands == hand;
        if (mine && !__all_sync(0xFFFFFFFFu, tc::mbar_wait(&sh->cmd_done[at], parity))) ring_fail(a, sh);
        __syncwarp();
        if (lane == 0) sh->passed[hand] = n + 1;
        if (last) ++seen;
        if (!mine) continue;
        // the groups' sums from the channels'
        const float* u_c = sums + (seen - 1) % kRingSums * 2 * a.channels;
        const float* v_c = u_c + a.channels;
        Tile t;
        locate_tile(a, tile, &t);
        const Fans f = fans_of(a, t);
        const float rows = (float)(t.row1 - t.row0);
        float* out = a.tile_parts + tile * step;
        int per = 1;   // lanes of a group
        while (per < 32 && 2 * per * a.groups <= 32) per *= 2;
        for (int32_t g0 = 0; g0 < a.groups; g0 += 32 / per) {
            const int32_t g = g0 + lane / per, c0 = g * a.each, c1 = g < a.groups ? c0 + a.each : 0;
            float u = 0.f, v = 0.f;
            if (BACKWARD) {
                for (int32_t c = c0 + lane % per; c < c1; c += per) {
                    const float w = a.weight ? a.weight[c] : 1.f;
                    u = fmaf(w, u_c[c], u); v = fmaf(w, v_c[c], v);
                }
            } else {
                for (int32_t c = c0 + lane % per; c < c1; c += per) u += u_c[c];
            }
            for (int o = 1; o < per; o <<= 1) { u += __shfl_xor_sync(0xFFFFFFFFu, u, o); if (BACKWARD) v += __shfl_xor_sync(0xFFFFFFFFu, v, o); }
            if (!BACKWARD) {
                u /= (float)a.each;
                for (int32_t c = c0 + lane % per; c < c1; c += per) { const float d = u_c[c] - u; v += fmaf(d * rows, d, v_c[c]); }
                for (int o = 1; o < per; o <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
            }
            if (lane % per == 0 && g < a.groups) { __stcg(out + g, u); __stcg(out + a.groups + g, v); }
        }
        if (BACKWARD && a.parts) {   // (the channels are a multiple of four)
            float4* to = reinterpret_cast<float4*>(a.parts + 2 * (int64_t)tile * a.channels);
            for (int32_t c = lane; c < a.channels / 2; c += 32) to[c] = reinterpret_cast<const float4*>(u_c)[c];
        }
        __syncwarp();
        if (lane == 0) sh->taken[hand] = (seen - 1) / kRingHands + 1;
        // the last of `fan` tiles brings theirs together, the last of those the sample's
        const int32_t fan = (tile - t.first) / a.fan, fan_tiles = min(a.fan, t.tiles - fan * a.fan);
        const auto count = [&](uint32_t* counter, int32_t want) {
            __syncwarp();
            int32_t full = 0;
            if (lane == 0) {
                __threadfence();
                full = atomicAdd(counter, 1u) + 1u == (uint32_t)want;
                __threadfence();
            }
            full = one(full);
            __syncwarp();
            return full != 0;
        };
        if (!count(a.fan_count + f.first_id + fan, fan_tiles)) continue;
        float* fan_parts = a.fan_parts + f.first_id * step;
        const int32_t first = fan * a.fan;
        const auto tile_values = [&](int32_t i) { return (float)min((int64_t)a.tile_rows, t.sample_rows - ((int64_t)first + i) * a.tile_rows) * (float)a.each; };
        hand_merge<BACKWARD>(a, a.tile_parts + ((int64_t)t.first + first) * step, fan_tiles, tile_values, fan_parts + fan * step);
        if (f.n > 1) {
            if (!count(a.sample_count + t.sample, f.n)) continue;
            const auto fan_values = [&](int32_t i) { return (float)min((int64_t)a.fan * a.tile_rows, t.sample_rows - (int64_t)i * a.fan * a.tile_rows) * (float)a.each; };
            hand_merge<BACKWARD>(a, fan_parts, f.n, fan_values, fan_parts);   // (a lane reads its group's sets before it writes the first)
        }
        __syncwarp();
        const float values = (float)t.sample_rows * (float)a.each;
        for (int32_t g = lane; g < a.groups; g += 32) {
            const float u = __ldcg(fan_parts + g), v = __ldcg(fan_parts + a.groups + g);
            if (BACKWARD) {
                __stcg(a.group_parts + t.sample * step + g, v / values);               // mean of dz w
                __stcg(a.group_parts + t.sample * step + a.groups + g, u / values);    // mean of dz w hat
            } else {
                __stcg(a.mean + (int64_t)t.sample * a.groups + g, u);
                __stcg(a.rstd + (int64_t)t.sample * a.groups + g, rsqrtf(v / values + a.eps));
            }
        }
        __syncwarp();
        if (lane == 0) {
            __threadfence();
            *reinterpret_cast<volatile uint32_t*>(a.ready + t.sample) = 1u;
        }
    }
}

// ---- warps 0 .. 15 ----------------------------------------------------------------------
template <typename T, int VEC> __device__ __forceinline__ void load_shared(Raw<T, VEC>& r, const char* p) {
    constexpr int kBytes = Raw<T, VEC>::kBytes;
    if constexpr (kBytes == 8) { const uint2 v = *reinterpret_cast<const uint2*>(p); r.w[0] = v.x; r.w[1] = v.y; }
    else {
#pragma unroll
        for (int q = 0; q < kBytes / 16; ++q) {
            const uint4 v = *reinterpret_cast<const uint4*>(p + 16 * q);
            r.w[4 * q] = v.x; r.w[4 * q + 1] = v.y; r.w[4 * q + 2] = v.z; r.w[4 * q + 3] = v.w;
        }
    }
}

// The block's threads with the same channels, into `out` ([2][channels] in shared memory).  One array serves means and squares one after the other:
// the mean of all sets first, then every thread's squares about that one.
template <int VEC> __device__ __forceinline__ void put_shared(float* s, const float (&v)[VEC]) {
#pragma unroll
    for (int e = 0; e < VEC; e += 4) *reinterpret_cast<float4*>(s + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
}
template <int VEC, bool BACKWARD>
__device__ __forceinline__ void ring_pairs(const RingArgs& a, Pair<VEC>& p, float* smem, int tx, float* out) {
    const int threads_x = 1 << a.tx, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    lane_pairs<VEC, BACKWARD>(p, threads_x);
    const int across = threads_x < 32 ? kRingWarps : kRingThreads / threads_x, set = threads_x < 32 ? warp : threadIdx.x >> a.tx, width = threads_x * VEC;
    const bool writes = threads_x >= 32 || lane < threads_x;
    float* sn = smem + kRingThreads * VEC;   // [across]
    float* mine = smem + set * width + tx * VEC;
    if (writes) {   // (what was there has been read: the block has met since)
        if (BACKWARD) put_shared<VEC>(mine, p.u);
        else {
            float u[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) u[e] = p.u[e] * p.n;
            put_shared<VEC>(mine, u);
            if (tx == 0) sn[set] = p.n;
        }
    }
    ring_sync();
    float all = 0.f;
    if (!BACKWARD) {
        for (int s = 0; s < across; ++s) all += sn[s];
        all = __fdividef(1.f, all);
    }
    for (int i = threadIdx.x; i < width && i < a.channels; i += kRingThreads) {
        float u = 0.f;
#pragma unroll 8
        for (int s = 0; s < across; ++s) u += smem[s * width + i];
        out[i] = BACKWARD ? u : u * all;
    }
    ring_sync();
    if (writes) {
        if (!BACKWARD) {
            float m[VEC];
            Params<VEC, 8>::read(out + min(tx * VEC, a.channels - VEC), m);
#pragma unroll
            for (int e = 0; e < VEC; ++e) { const float d = p.u[e] - m[e]; p.v[e] = fmaf(d * p.n, d, p.v[e]); }
        }
        put_shared<VEC>(mine, p.v);
    }
    ring_sync();
    for (int i = threadIdx.x; i < width && i < a.channels; i += kRingThreads) {
        float v = 0.f;
#pragma unroll 8
        for (int s = 0; s < across; ++s) v += smem[s * width + i];
        out[a.channels + i] = v;
    }
    ring_sync();
}

template <typename T, int VEC, bool BACKWARD>
__global__ void __launch_bounds__(kRingBlock, 1) k_norm_ring(const __grid_constant__ RingArgs a) {
    extern __shared__ __align__(128) char shared[];
    RingShared* sh = reinterpret_cast<RingShared*>(shared);
    float* scratch = reinterpret_cast<float*>(shared + ring_scratch_at());
    float* sums = reinterpret_cast<float*>(shared + ring_sums_at(VEC));
    char* slots = shared + ring_fixed_bytes(VEC, a.channels);
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kRingSlots; ++i) { tc::mbar_init(&sh->full[i], a.drop.on && a.drop.keys ? 33 : 1); sh->held[i] = -1; }
        for (int i = 0; i < kRingCmds; ++i) { tc::mbar_init(&sh->cmd_full[i], 1); tc::mbar_init(&sh->cmd_done[i], kRingWarps); }
        for (int i = 0; i < kRingHands; ++i) sh->passed[i] = sh->taken[i] = 0;
        sh->failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    if (warp == kRingWarps) { RingLead<T, BACKWARD>(a, sh, slots).work(); return; }
    if (warp > kRingWarps) { ring_hand<BACKWARD>(a, sh, sums, warp - kRingWarps - 1); return; }

    const int tx = threadIdx.x & ((1 << a.tx) - 1), ty = threadIdx.x >> a.tx, n_ty = kRingThreads >> a.tx, lane = threadIdx.x & 31;
    if (!a.equal) {   // samples without rows have no tiles
        for (int32_t s = blockIdx.x; s < a.samples; s += gridDim.x) {
            if (sample_entry(a, s).x != sample_entry(a, s + 1).x) continue;
            for (int32_t g = threadIdx.x; !BACKWARD && g < a.groups; g += kRingThreads) { a.mean[(int64_t)s * a.groups + g] = 0.f; a.rstd[(int64_t)s * a.groups + g] = 0.f; }
        }
    }
    const int32_t c = tx * VEC;
    const bool in = c < a.channels;
    const int32_t row_bytes = a.channels * (int32_t)sizeof(T), step = row_bytes * n_ty;
    const int32_t group = in ? c / a.each : 0;
    float w[VEC], b[VEC];
    load_params<VEC>(in ? a.weight : nullptr, c, 1.f, w);
    load_params<VEC>(in ? a.bias : nullptr, c, 0.f, b);
    Pair<VEC> p;
    // a command's statistics are asked for while the one before it is worked on
    float mean = 0.f, rstd = 0.f, s1 = 0.f, s2 = 0.f;
    const auto statistics = [&](const RingCmd& k) {
        if (k.kind == CMD_EXIT || (!BACKWARD && k.kind == CMD_SUMS)) return;
        const int64_t stat = (int64_t)k.sample * a.groups + group;
        mean = __ldcg(a.mean + stat); rstd = __ldcg(a.rstd + stat);
        if (BACKWARD && k.kind == CMD_RESULT) {
            const int64_t at_group = (int64_t)k.sample * 2 * a.groups + group;
            s1 = __ldcg(a.group_parts + at_group); s2 = __ldcg(a.group_parts + at_group + a.groups);
        }
    };
    bool asked = false;
    int tiles = 0;   // sums that have been finished
    for (int n = 0;; ++n) {
        const int at = n % kRingCmds, parity = n / kRingCmds & 1;
        if (!ring_next(sh, at, parity)) { ring_fail(a, sh); break; }
        const int32_t kind = sh->cmd[at].kind, rows = sh->cmd[at].rows, part = sh->cmd[at].part, wait = sh->cmd[at].wait, slot_at = sh->cmd[at].slot;
        const int64_t row0 = sh->cmd[at].row0;
        if (kind == CMD_EXIT) break;
        if (!asked) statistics(sh->cmd[at]);
        const float mean_n = mean, rstd_n = rstd, s1_n = s1, s2_n = s2;
        const int next = (n + 1) % kRingCmds;
        asked = __all_sync(0xFFFFFFFFu, mbar_test(&sh->cmd_full[next], (n + 1) / kRingCmds & 1));
        if (asked) statistics(sh->cmd[next]);
        if (wait && !tc::mbar_wait(&sh->full[slot_at], (uint32_t)wait - 1)) ring_fail(a, sh);
        const char* slot = slots + (int64_t)slot_at * a.slot_bytes;
        const char* sx = slot + c * (int32_t)sizeof(T);
        const int64_t* keys = reinterpret_cast<const int64_t*>(slot + a.keys_at);
        const auto key_of = [&](int32_t r) { return !a.drop.on ? 0ull : a.drop.keys ? (uint64_t)keys[r] : (uint64_t)(a.drop.first_row + row0 + r); };
        if (kind == CMD_SUMS) {
            if (part & PART_FIRST) {
                p.n = 0.f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) p.u[e] = p.v[e] = 0.f;
            }
            if (in) {
                if constexpr (BACKWARD) {
                    const char* px = sx + ty * row_bytes;
                    for (int32_t r = ty; r < rows; r += n_ty, px += step) {
                        Raw<T, VEC> rx, rd;
                        load_shared(rx, px);
                        load_shared(rd, px + a.d_y_at);
                        float h[VEC], d[VEC];
                        grad_vector<T, VEC>(a, rx, rd, key_of(r), c, mean_n, rstd_n, w, b, h, d);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) { p.u[e] = fmaf(d[e], h[e], p.u[e]); p.v[e] += d[e]; }
                    }
                } else {
                    constexpr int K = sizeof(T) * VEC == 32 ? 2 : 4;
                    const char* px = sx + ty * row_bytes;
                    for (int32_t r = ty; r < rows; r += K * n_ty, px += K * step) {
                        Raw<T, VEC> raw[K];
                        float u[VEC], v[VEC];
                        if (r + (K - 1) * n_ty < rows) {
#pragma unroll
                            for (int k = 0; k < K; ++k) load_shared(raw[k], px + k * step);
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
                            for (int32_t q = r; q < rows; q += n_ty) {
                                load_shared(raw[0], px + (q - r) / n_ty * step);
#pragma unroll
                                for (int e = 0; e < VEC; ++e) { u[e] = raw[0].get(e); v[e] = 0.f; }
                                merge<VEC, false>(p, 1.f, u, v);
                            }
                        }
                    }
                }
            }
            if (part & PART_LAST) ring_pairs<VEC, BACKWARD>(a, p, scratch, tx, sums + tiles++ % kRingSums * 2 * a.channels);
        } else if (in) {
            T* out = static_cast<T*>(a.out) + row0 * a.out_stride + c;
            const char* px = sx + ty * row_bytes;
            float ws[VEC];
            if constexpr (!BACKWARD) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) ws[e] = w[e] * rstd_n;
            }
            for (int32_t r = ty; r < rows; r += n_ty, px += step) {
                Raw<T, VEC> rx;
                load_shared(rx, px);
                float f[VEC];
                if constexpr (BACKWARD) {
                    Raw<T, VEC> rd;
                    load_shared(rd, px + a.d_y_at);
                    float h[VEC];
                    grad_vector<T, VEC>(a, rx, rd, key_of(r), c, mean_n, rstd_n, w, b, h, f);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) f[e] = rstd_n * fmaf(-h[e], s2_n, fmaf(f[e], w[e], -s1_n));
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) f[e] = fmaf(rx.get(e) - mean_n, ws[e], b[e]);
                    act_values<VEC>(a.act, f);
                    if (a.drop.on) {
                        Keep<VEC> keep;
                        keep.draw(a.drop, key_of(r), (uint32_t)c);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) f[e] = keep(a.drop, e) ? f[e] * a.drop.factor : 0.f;
                    }
                }
                rx.put(f);
                rx.store(out + (int64_t)r * a.out_stride);
            }
        }
        __syncwarp();
        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(tc::smem_u32(&sh->cmd_done[at])) : "memory");
    }
}

struct RingLaunch { int vec; bool backward; int grid; };
template <typename T> cudaError_t launch_ring(const RingLaunch& l, const RingArgs& a, cudaStream_t st);

}  // namespace mgnorm
