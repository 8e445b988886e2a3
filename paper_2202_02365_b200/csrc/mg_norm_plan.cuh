// Host side of dropout and of group norm: checks of arguments, and how a call is cut into work.  No CUDA calls.
#pragma once

#include <math.h>

#include <algorithm>

#include "mg_call.cuh"
#include "mg_norm_tiles.cuh"

namespace {

using namespace mgnorm;

int check_dropout(mg_ctx* ctx, const mg_dropout_spec* s, DropArgs* d) {
    *d = DropArgs();
    if (!s) return MG_OK;
    if (!(s->p >= 0.0 && s->p <= 1.0)) return mg_fail(ctx, MG_ERR_ARG, "the share to drop must be in [0, 1]");
    if (s->site > 0xFFFFu) return mg_fail(ctx, MG_ERR_ARG, "a dropout's site must be below 65536");
    if (reinterpret_cast<uintptr_t>(s->row_keys) % 8) return mg_fail(ctx, MG_ERR_ARG, "row keys must be 8-byte aligned");
    const uint32_t limit = (uint32_t)nearbyint(s->p * 65536.0);
    d->on = limit > 0;
    d->below = (uint32_t)((uint64_t)limit * 65536u - 1u);
    d->factor = limit < 65536u ? 65536.f / (float)(65536u - limit) : 0.f;
    for (uint32_t r = 0; r < 10; ++r) { d->k0[r] = (uint32_t)s->seed + r * 0x9E3779B9u; d->k1[r] = (uint32_t)(s->seed >> 32) + r * 0xBB67AE85u; }
    d->tag = kDropTag + s->site;
    d->first_row = s->first_row; d->keys = s->row_keys;
    return MG_OK;
}

int check_rows(mg_ctx* ctx, int dtype, int64_t rows, int32_t channels) {
    if (dtype != MG_DTYPE_F32 && dtype != MG_DTYPE_F16 && dtype != MG_DTYPE_BF16) return mg_fail(ctx, MG_ERR_ARG, "unknown dtype");
    if (rows < 0 || rows >= 1ll << 31) return mg_fail(ctx, MG_ERR_ARG, "the number of rows must be in [0, 2^31)");
    if (channels < 1 || channels > 1 << 24) return mg_fail(ctx, MG_ERR_ARG, "the number of channels must be in [1, 2^24]");
    return MG_OK;
}

int check_norm(mg_ctx* ctx, const mg_norm_spec* s) {
    if (!s) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    if (int rc = check_rows(ctx, s->dtype, s->rows, s->channels)) return rc;
    if (s->groups < 1 || s->channels % s->groups) return mg_fail(ctx, MG_ERR_ARG, "the groups must divide the channels");
    if (s->activation < MG_ACT_NONE || s->activation > MG_ACT_GELU) return mg_fail(ctx, MG_ERR_ARG, "unknown activation");
    if (!(s->eps > 0.f) || isinf(s->eps)) return mg_fail(ctx, MG_ERR_ARG, "eps must be positive and finite");
    if (s->sample_offsets) {
        if (s->n_samples < 1 || s->n_samples > MG_MAX_BATCHES) return mg_fail(ctx, MG_ERR_ARG, "the number of samples must be in [1, %d]", MG_MAX_BATCHES);
        if (s->sample_offsets[0] != 0) return mg_fail(ctx, MG_ERR_ARG, "the first sample starts at row 0");
        for (int32_t i = 0; i < s->n_samples; ++i)
            if (s->sample_offsets[i + 1] < s->sample_offsets[i]) return mg_fail(ctx, MG_ERR_ARG, "the samples' offsets must not decrease");
        if (s->sample_offsets[s->n_samples] > s->rows) return mg_fail(ctx, MG_ERR_ARG, "the samples end behind the last row");
    } else if (s->rows_per_sample < 1 || s->rows % s->rows_per_sample) {
        return mg_fail(ctx, MG_ERR_ARG, "the rows must be a multiple of rows_per_sample, which must be positive");
    }
    return MG_OK;
}

int64_t sample_count(const mg_norm_spec* s) { return s->sample_offsets ? s->n_samples : s->rows / s->rows_per_sample; }

// ---- how a call is cut ------------------------------------------------------------------

enum { NORM_NOTHING = 0, NORM_ROWS = 1, NORM_TILES = 2 };

struct NormPlan {
    int mode = NORM_NOTHING, vec = 1;
    int grid = 0;
    // rows
    int nv = 1;
    int cut = ROW_EVEN;
    RowShape shape{0, 0, 0};
    // workspace: bytes that are cleared first, then where the others start
    size_t cleared = 0, at_fan_count = 0, at_sample_count = 0, at_table = 0, at_tile_parts = 0, at_fan_parts = 0, at_group_parts = 0, at_parts = 0, at_slices = 0, bytes = 0;
    int64_t n_parts = 0;   // backward: what k_norm_params adds up
    int sums_vec = 1;      // tiles: vectors of the sums
    int block_grid = 0, cluster = 0;   // samples that a block or a cluster deals with by itself: how many blocks, and how many to a sample
};

int ceil_log2(int64_t v) { int l = 0; while ((1ll << l) < v) ++l; return l; }
int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

constexpr int64_t kParamSlices = 64;   // of the parts that k_norm_params adds up in two steps
constexpr int kRowsMaxChannels = 32 * kRowValues;
constexpr int kRowBlocks = 8;   // blocks per SM, forward
constexpr int kTileBlocks = 4, kTileBlocksBackward = 3;

// Rows that are samples by themselves, `vec` values to a vector.
void plan_rows(const mg_norm_spec* s, int n_sms, bool backward, int vec, NormPlan* p) {
    p->mode = NORM_ROWS; p->vec = vec;
    const int64_t vecs = s->channels / vec;
    const int64_t each = s->channels / s->groups;
    p->shape.lanes = std::min(5, ceil_log2(vecs));
    p->nv = 1 << ceil_log2((vecs + 31) / 32);
    const int64_t width = each / vec;
    // Groups of other widths than a power of two, us forward / backward.  Narrow ones of whole vectors meet in shared memory: 100,000 fp32 rows of 768 in 32
    // groups 115 / 276 (under masks 1,812 / 2,749), 200,000 of 192 in 16 67 / 124 (591 / 762).  Under masks, one after the other: wide ones, where shared memory
    // takes a lane as many reads as a group has vectors, and all that are not whole vectors, narrow or many as they may be.  That costs what the groups' number
    // and the row's values multiply to: 200,000 fp32 rows of 602 in 2 545 / 2,104 with a ReLU, of 100 in 4 176 / 288, of 300 in 10 1,198 / 2,493, of 320 in 32
    // 2,128 / 3,256 (their bytes 147 / 220, 24 / 37, 73 / 110, 78 / 117); backward also a division and two loads of statistics for every value.
    if (s->groups > 1 && (each % vec || (width & (width - 1)))) p->cut = each % vec == 0 && width < 2 * vec * s->groups ? ROW_NARROW : ROW_MASKS;
    p->shape.width = p->cut == ROW_NARROW ? (int32_t)width : 0;
    p->shape.gshift = s->groups == 1 ? 31 : ceil_log2(std::max<int64_t>(width, 1));
    const int64_t per_block = (int64_t)kNormWarps * (32 >> p->shape.lanes);
    // forward: more blocks where each has sixteen turns all the same (543,000 rows of 256: 201 us in eight to an SM, 196 in sixteen; 60,000 of 128: 15.2 and
    // 16.3); backward: as many as an SM holds
    const int64_t all = (s->rows + per_block - 1) / per_block, per_sm = backward ? (p->nv * vec <= 8 ? 3 : p->nv * vec <= 16 ? 2 : 1) : std::clamp<int64_t>(all / 16 / n_sms, kRowBlocks, 2 * kRowBlocks);
    p->grid = (int)std::min<int64_t>(all, n_sms * per_sm);
    p->n_parts = backward ? p->grid : 0;
    p->at_slices = sizeof(float) * 2 * (size_t)s->channels * (size_t)p->n_parts;
    p->bytes = backward ? p->at_slices + sizeof(float) * 2 * (size_t)s->channels * kParamSlices : 0;
}

// Samples of up to 64 KB go to one block each, larger ones to a cluster of up to 16 with shares as large; one above 32 KB to as many blocks as two to
// an SM leave it (clusters of 16: one to an SM, they are hard to place), with no less than 8 KB each.  In a replayed graph, fp32 rows of 128 channels
// with a SiLU, against the two launches, forward / backward in us: one sample of 16 KB 4.4 / 7.0 against 12.1 / 15.5 (two blocks 6.7 / 9.3), of 64 KB
// in 8 blocks 7.5 / 10.1 against 12.2 / 16.4 (one block 6.9 / 12.7), of 256 KB in 16 8.6 / 11.7 against 12.4 / 16.4, of 1 MB 11.1 / 18.3 against
// 15.4 / 18.5, of 2 MB 14.4 / 25.8 against 16.4 / 19.7; 16 of 256 KB in 8 blocks each 10.1 / 17.0 (in 16: 16.7 / 22.2) against 16.4 / 19.1; 64 of 256 KB
// in 4 12.8 / 23.2 (in 8: 19.4 / 32.6) against 19.9 / 30.5; 600 of 64 KB 24.6 / 49.5 against 30.7 / 59.5; 20,000 of 4 KB 235 / 290 against 300 / 421.
constexpr int64_t kBlockBytes = 64 << 10;
int blocks_of_sample(int64_t n, int64_t bytes, int n_sms) {
    int c = 1;
    while (bytes > 32 << 10 && c < kMaxCluster && bytes > (8 << 10) * c && n * c * 2 <= (c * 2 == kMaxCluster ? n_sms : 2 * n_sms)) c *= 2;
    return bytes <= kBlockBytes * c ? c : 0;
}
// Larger ones are cut into tiles, each summed up by one block, as many as the SMs hold together: one turn.  Where the samples' ends would leave that turn
// uneven, more turns, of tiles of no less than 384 KB.  Results are computed by blocks of a few turns of loads, which make room for the next ones: 128 KB of
// rows each, 512 KB where there is a gradient (its blocks prepare more).  In a replayed graph: 24 samples of 22,625 rows of 256 fp32 channels 292 us with
// tiles of 384 KB for both, 270 so, backward 531 and 512; one sample of 2,000,003 rows of 128, backward, 981 and 844.
constexpr int64_t kTileBytes = 384 << 10, kPartBytes = 128 << 10, kPartBytesBackward = 512 << 10;

TileShape tile_shape(const mg_norm_spec* s, int vec) {
    TileShape t;
    const int64_t vecs = s->channels / vec;
    t.tx = std::min(ceil_log2(kNormThreads), ceil_log2(vecs));
    t.chunks = (int32_t)((vecs + (1 << t.tx) - 1) >> t.tx);
    return t;
}

int64_t longest_sample(const mg_norm_spec* s) {
    if (!s->sample_offsets) return s->rows_per_sample;
    int64_t longest = 0;
    for (int32_t i = 0; i < s->n_samples; ++i) longest = std::max(longest, s->sample_offsets[i + 1] - s->sample_offsets[i]);
    return longest;
}

// How many blocks k_norm_block gives a sample, 0 where it does not take the call.
int sample_blocks(const mg_norm_spec* s, int n_sms, int vec, int64_t longest) {
    if (tile_shape(s, vec).chunks > 1 || s->channels > kBlockChannels || s->groups > kBlockGroups) return 0;
    return blocks_of_sample(sample_count(s), longest * s->channels * elem_size(s->dtype), n_sms);
}

// Samples of several rows, or of a row too wide for a warp.  a: the geometry's part of the arguments.
void plan_tiles(const mg_norm_spec* s, int n_sms, bool backward, int vec, NormPlan* p, TileArgs* a) {
    p->mode = NORM_TILES; p->vec = vec;
    const int64_t n = sample_count(s), elem = elem_size(s->dtype);
    // (16 bytes a thread let more rows be on their way; with a dropout eight channels share a block of the generator)
    p->sums_vec = backward && s->dropout ? vec : (int)std::min<int64_t>(vec, 16 / elem);
    a->sums = tile_shape(s, p->sums_vec); a->results = tile_shape(s, vec);
    a->run = (int32_t)std::min<int64_t>(s->channels, (int64_t)p->sums_vec << a->sums.tx);
    const bool equal = !s->sample_offsets;
    const int64_t used = equal ? s->rows : s->sample_offsets[n], longest = longest_sample(s);
    a->samples = (int32_t)n; a->equal = equal;
    a->rows_per_sample = s->rows_per_sample;
    p->cluster = sample_blocks(s, n_sms, vec, longest);
    if (p->cluster) {
        p->block_grid = (int)std::min<int64_t>(n, (int64_t)n_sms * 4 / p->cluster) * p->cluster;
        size_t at = 0;
        const auto take = [&](size_t bytes) { const size_t was = at; at += (bytes + 15) / 16 * 16; return was; };
        p->cleared = 0;
        p->at_table = take(!equal && n > kInlineSamples ? sizeof(int2) * (size_t)(n + 1) : 0);
        p->n_parts = backward ? p->block_grid : 0;
        p->at_parts = take(8 * (size_t)p->n_parts * s->channels);
        p->at_slices = take(p->n_parts ? 8 * (size_t)kParamSlices * s->channels : 0);
        p->bytes = at;
        a->tiles = 0; a->tile_rows = 1 << 30; a->tiles_per_sample = 1;
        return;
    }
    const int64_t n_ty = kNormThreads >> a->results.tx, row_bytes = (int64_t)s->channels * elem, chunks = a->sums.chunks;
    const int64_t held = (int64_t)n_sms * (backward ? kTileBlocksBackward : kTileBlocks), units = used * chunks;
    const auto count = [&](int64_t rows) {
        if (equal) return n * ((s->rows_per_sample + rows - 1) / rows);
        int64_t tiles = 0;
        for (int64_t i = 0; i < n; ++i) tiles += (s->sample_offsets[i + 1] - s->sample_offsets[i] + rows - 1) / rows;
        return tiles;
    };
    const int64_t least = std::max({round_up((longest + kFan * kFan - 1) / (kFan * kFan), n_ty), (int64_t)16}), most_turns = std::max<int64_t>(1, used * row_bytes / (held * kTileBytes));
    int64_t rows = least, tiles = 0;
    double best = 0.0;
    for (int64_t turns = n > kInlineSamples ? most_turns : 1; used > 0 && turns <= most_turns; turns = turns < 4 || turns == most_turns ? turns + 1 : most_turns) {
        int64_t r = std::max(round_up(std::max<int64_t>(1, (units + held * turns - 1) / (held * turns)), n_ty), least), t = count(r);
        // (a tile more than the blocks' turns costs a turn)
        for (int tries = 0; tries < 4 && t * chunks > held * turns; ++tries) t = count(r += round_up(std::max<int64_t>(r / 32, 1), n_ty));
        const double even = (double)units / ((double)((t * chunks + held - 1) / held * held) * (double)r);
        if (even > best) { best = even; rows = r; tiles = t; }
        if (best >= 0.9) break;
    }
    rows = std::min(rows, std::max(round_up(longest, n_ty), (int64_t)16));
    a->tile_rows = (int32_t)std::min<int64_t>(rows, 1 << 30);
    a->tiles_per_sample = equal ? (int32_t)((s->rows_per_sample + a->tile_rows - 1) / a->tile_rows) : 0;
    a->tiles = (int32_t)tiles;
    // (no more than twice the blocks that have rows)
    const int64_t run_bytes = std::min<int64_t>(s->channels, (int64_t)vec << a->results.tx) * elem, part = backward ? kPartBytesBackward : kPartBytes;
    const int64_t part_of = (rows * run_bytes + part / 2) / part, useful = 2 * used * run_bytes / part / std::max<int64_t>(tiles, 1);
    const int64_t parts = std::max<int64_t>(1, std::min(part_of, useful));
    a->part_rows = (int32_t)round_up((a->tile_rows + parts - 1) / parts, n_ty);
    a->parts_of_tile = (a->tile_rows + a->part_rows - 1) / a->part_rows;
    const int64_t fans = tiles / kFan + n + 1, pair = 2 * (int64_t)sizeof(float);
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t was = at; at += (bytes + 15) / 16 * 16; return was; };
    p->at_fan_count = take(4 * (size_t)fans);
    p->at_sample_count = take(4 * (size_t)n);
    p->cleared = at;
    p->at_table = take(!equal && n > kInlineSamples ? sizeof(int2) * (size_t)(n + 1) : 0);
    p->at_tile_parts = take((size_t)(tiles * chunks * s->groups * pair));
    p->at_fan_parts = take((size_t)(fans * s->groups * pair));
    p->at_group_parts = take(backward ? (size_t)(n * s->groups * pair) : 0);
    p->n_parts = backward ? tiles : 0;
    p->at_parts = take((size_t)(p->n_parts * s->channels * pair));
    p->at_slices = take(p->n_parts ? (size_t)(kParamSlices * s->channels * pair) : 0);
    p->bytes = at;
}

// Many short samples that k_norm_block does not take go to k_norm_wide.  Tiles, of which each sample has one at least, would keep sums by channel for
// every one of them: 200,000 single rows of 2,048 fp32 channels asked for 3.8 GB beside their 1.6, of 4,096 in fp16 for 7.5 GB; here for 7 and 15 MB.  Both
// sides, tiles / k_norm_wide, forward and backward, us: these two, in 32 groups, 4,399 / 1,940 and 9,127 / 4,997, 5,605 / 3,530 and 14,317 / 11,430; 50,000 fp16
// rows of 4,095 in one 8,600 / 5,100 and 15,050 / 7,900; 20,000 samples of 8 fp32 rows of 602 in two 880 / 560 and 1,484 / 1,130; 3,000 of 16 fp16 rows of 2,048
// 148 / 119 and 437 / 320.  Of 30 rows and more tiles are faster (3,000 of 30 of 602: 232 / 295 and 478 / 600), and their sums by channel a quarter of the
// rows or less; 600 rows of 4,096 took 30 / 21 and 60 / 64, 1,200 of them 46 / 31 and 281 / 101.
constexpr int64_t kShortRows = 16, kWideBytes = 128 << 20;
constexpr int kShortSamples = 6, kWideLeastBlocks = 16;   // per SM; in all, whatever kWideBytes says
bool short_samples(const mg_norm_spec* s, int n_sms) { return sample_count(s) > kShortSamples * (int64_t)n_sms && longest_sample(s) <= kShortRows; }

void plan_wide(const mg_norm_spec* s, int n_sms, bool backward, int vec, NormPlan* p, TileArgs* a) {
    p->mode = NORM_TILES; p->vec = p->sums_vec = vec;
    const int64_t n = sample_count(s), pair = 2 * (int64_t)sizeof(float);
    a->sums = a->results = tile_shape(s, vec);
    a->run = (int32_t)std::min<int64_t>(s->channels, (int64_t)vec << a->results.tx);
    a->samples = (int32_t)n; a->equal = !s->sample_offsets;
    a->rows_per_sample = s->rows_per_sample;
    a->tiles = 0; a->tile_rows = 1 << 30; a->tiles_per_sample = 1;
    p->block_grid = (int)std::min<int64_t>(n, (int64_t)n_sms * (!backward ? 8 : vec == 8 ? kWideBlocks<8> : kWideBlocks<1>));
    if (backward) p->block_grid = (int)std::min<int64_t>(p->block_grid, std::max<int64_t>(kWideBytes / (pair * s->channels), kWideLeastBlocks));
    p->cluster = 0;
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t was = at; at += (bytes + 15) / 16 * 16; return was; };
    p->at_table = take(!a->equal && n > kInlineSamples ? sizeof(int2) * (size_t)(n + 1) : 0);
    p->at_group_parts = take(backward ? (size_t)(p->block_grid * s->groups * pair) : 0);
    p->n_parts = backward ? p->block_grid : 0;   // (k_norm_params takes as many in one step)
    p->at_parts = take((size_t)(p->n_parts * s->channels * pair));
    p->bytes = at;
}

// the vector widths that there are kernels for: 32, 16, 8 (16-bit types: 16, 8, 4) and one element
const int* vec_widths(int dtype) {
    static const int wide[] = {8, 4, 1, 0}, narrow[] = {8, 4, 2, 1, 0};
    return dtype == MG_DTYPE_F32 ? wide : narrow;
}

int norm_mode(const mg_norm_spec* s) {
    if (sample_count(s) == 0) return NORM_NOTHING;
    if (!s->sample_offsets && s->rows_per_sample == 1 && s->channels <= kRowsMaxChannels) return NORM_ROWS;
    return NORM_TILES;
}

// what rows, or samples cut as plan_tiles has it, want: the most that the matrices' alignment makes of it
size_t norm_workspace(const mg_norm_spec* s, int n_sms, bool backward) {
    const int mode = norm_mode(s);
    size_t most = 0;
    for (const int* v = vec_widths(s->dtype); *v && mode != NORM_NOTHING; ++v) {
        if (s->channels % *v) continue;
        NormPlan p;
        TileArgs a;
        if (mode == NORM_ROWS) plan_rows(s, n_sms, backward, *v, &p);
        else plan_tiles(s, n_sms, backward, *v, &p, &a);
        most = std::max(most, p.bytes);
    }
    return most;
}

// how a call of samples is cut, given its vectors
void plan_samples(const mg_norm_spec* s, int n_sms, bool backward, int vec, NormPlan* p, TileArgs* a) {
    if (short_samples(s, n_sms) && !sample_blocks(s, n_sms, vec, longest_sample(s))) plan_wide(s, n_sms, backward, vec, p, a);
    else plan_tiles(s, n_sms, backward, vec, p, a);
}

// what a call wants, whatever the matrices' alignment makes of it
size_t call_workspace(const mg_norm_spec* s, int n_sms, bool backward) {
    if (norm_mode(s) != NORM_TILES || !short_samples(s, n_sms)) return norm_workspace(s, n_sms, backward);
    size_t most = 0;
    for (const int* v = vec_widths(s->dtype); *v; ++v) {
        if (s->channels % *v) continue;
        NormPlan p;
        TileArgs a;
        plan_samples(s, n_sms, backward, *v, &p, &a);
        most = std::max(most, p.bytes);
    }
    return most;
}

struct Matrix { const char* what; const void* p; int64_t stride; bool written; };

// the output (the last of the matrices) may be one of the inputs
int check_matrices(mg_ctx* ctx, const Matrix* m, int n, int dtype, int64_t rows, int32_t channels) {
    for (int i = 0; i < n; ++i)
        if (int rc = check_matrix(ctx, m[i].what, m[i].p, m[i].stride, dtype, rows, channels, m[i].written)) return rc;
    for (int i = 0; i + 1 < n; ++i)
        if (int rc = check_apart(ctx, m[i].what, m[i].p, m[i].stride, m[n - 1].p, m[n - 1].stride, dtype, rows, channels)) return rc;
    return MG_OK;
}

// The widest vectors that all the matrices' rows are made of; whole groups of them, or whole rows where the groups do not matter.
int vec_width(const Matrix* m, int n, int dtype, int64_t rows, int32_t of) {
    const int64_t e = elem_size(dtype);
    for (const int* v = vec_widths(dtype); *v; ++v) {
        bool ok = of % *v == 0;
        for (int i = 0; i < n; ++i) ok = ok && reinterpret_cast<uintptr_t>(m[i].p) % (uintptr_t)(*v * e) == 0 && (rows <= 1 || m[i].stride % *v == 0);
        if (ok) return *v;
    }
    return 1;
}

// ... for rows that are samples by themselves: a group's vectors where they are a power of two in number or as wide as fours, else the row's
int rows_vec_width(const Matrix* m, int n, const mg_norm_spec* s) {
    const int32_t each = s->channels / s->groups;
    const int v = vec_width(m, n, s->dtype, s->rows, each), w = each / v;
    return (w & (w - 1)) == 0 || v >= 4 ? v : vec_width(m, n, s->dtype, s->rows, s->channels);
}

// every check of an entry point's arguments but the workspace's; `d`: the dropout as the kernels take it
int check_dropout_call(mg_ctx* ctx, const void* x, int64_t x_stride, const void* y, int64_t y_stride, int dtype, int64_t rows, int32_t channels,
                       const mg_dropout_spec* spec, DropArgs* d) {
    if (!spec) return mg_fail(ctx, MG_ERR_ARG, "null argument");
    if (int rc = check_rows(ctx, dtype, rows, channels)) return rc;
    if (int rc = check_dropout(ctx, spec, d)) return rc;
    const Matrix m[2] = {{"x", x, x_stride, false}, {"y", y, y_stride, true}};
    return check_matrices(ctx, m, 2, dtype, rows, channels);
}

int check_norm_call(mg_ctx* ctx, const mg_norm_spec* s, const void* x, int64_t x_stride, const void* d_y, int64_t d_y_stride, bool backward,
                    const void* out, int64_t out_stride, const float* mean, const float* rstd, const void* workspace, DropArgs* d,
                    const float* d_weight = nullptr, const float* d_bias = nullptr) {
    if (int rc = check_norm(ctx, s)) return rc;
    if (int rc = check_dropout(ctx, s->dropout, d)) return rc;
    const Matrix fwd[2] = {{"x", x, x_stride, false}, {"y", out, out_stride, true}};
    const Matrix bwd[3] = {{"x", x, x_stride, false}, {"d_y", d_y, d_y_stride, false}, {"d_x", out, out_stride, true}};
    if (int rc = check_matrices(ctx, backward ? bwd : fwd, backward ? 3 : 2, s->dtype, s->rows, s->channels)) return rc;
    if (sample_count(s) > 0 && (!mean || !rstd)) return mg_fail(ctx, MG_ERR_ARG, "null statistics");
    for (const void* p : {(const void*)mean, (const void*)rstd, (const void*)s->weight, (const void*)s->bias, (const void*)d_weight, (const void*)d_bias})
        if (reinterpret_cast<uintptr_t>(p) % 4) return mg_fail(ctx, MG_ERR_ARG, "statistics, weight, bias and their gradients must be 4-byte aligned");
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return mg_fail(ctx, MG_ERR_ARG, "the workspace must be 16-byte aligned");
    return MG_OK;
}

}  // namespace
