// Dropout, and group norm of rows that are samples by themselves: a warp, or a part of one, holds a row in registers.
#pragma once

#include "mg_norm.cuh"

namespace mgnorm {

constexpr int kNormThreads = 256, kNormWarps = kNormThreads / 32;
constexpr int kRowValues = 32;   // values of a row that a lane holds at most

struct NormArgs {
    const void* x = nullptr; const void* d_y = nullptr; void* out = nullptr;
    int64_t x_stride = 0, d_y_stride = 0, out_stride = 0;
    const float* weight = nullptr; const float* bias = nullptr;   // null: ones, zeros
    float* mean = nullptr; float* rstd = nullptr;                 // [samples, groups]
    float* parts = nullptr;                                       // backward: sums of dz hat, then of dz, by channel: [parts][2][channels]
    int64_t rows = 0;
    int32_t channels = 0, groups = 0, act = 0;
    int32_t each = 0;                                             // channels of a group
    float eps = 0.f;
    DropArgs drop;
};

// A vector's normalised values, and the gradient in front of weight and bias: dz = dropout(dy) act'
template <typename T, int VEC>
__device__ __forceinline__ void grad_vector(const NormArgs& a, const Raw<T, VEC>& rx, const Raw<T, VEC>& rd, uint64_t key, int32_t c, float mean, float rstd,
                                            const float (&w)[VEC], const float (&b)[VEC], float (&h)[VEC], float (&d)[VEC]) {
    float n[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) { h[e] = (rx.get(e) - mean) * rstd; n[e] = fmaf(h[e], w[e], b[e]); d[e] = rd.get(e); }
    act_slopes<VEC>(a.act, d, n, b, [&](int e) { return ((double)rx.get(e) - (double)mean) * (double)rstd * (double)w[e] + (double)b[e]; });
    drop_vector<VEC>(a.drop, key, c, d);
}

// Dropout of rows of eight-channel vectors: a thread draws a block of the generator for each (ten rounds, some 75 instructions, for 16 or 32 bytes).
// fp32 is bound by the bytes: 543,000 rows of 256 in 162 us, 6.9 TB/s.  fp16 by the instructions, 130 a vector, as much as by the bytes: 150,001 rows of 768
// in 87 us, 5.3 TB/s, 60 % of the issue slots busy.
template <typename T, int VEC>
__global__ void __launch_bounds__(kNormThreads) k_dropout(const T* x, int64_t x_stride, T* y, int64_t y_stride, int32_t rows, int32_t channels, DropArgs d) {
    static_assert(VEC == 8, "a block of the generator");
    const int32_t vecs = channels / VEC;
    const int64_t step = (int64_t)gridDim.x * kNormThreads, i0 = blockIdx.x * (int64_t)kNormThreads + threadIdx.x;
    const int32_t step_rows = (int32_t)(step / vecs), step_v = (int32_t)(step - (int64_t)step_rows * vecs);
    int64_t row = i0 / vecs;   // (beyond the rows by less than a step)
    int32_t v = (int32_t)(i0 - row * vecs);
    constexpr int U = sizeof(T) == 4 ? 2 : 4;   // vectors on their way per thread
    while (row < rows) {
        Raw<T, VEC> p[U];
        int32_t at_row[U], at_v[U];
        uint64_t key[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            at_row[u] = row < rows ? (int32_t)row : -1; at_v[u] = v;
            if (row < rows) {
                p[u].load(x + row * x_stride + v * VEC);
                key[u] = d.on ? drop_key(d, row) : 0;   // (behind it, not behind its arrival: 150,001 keyed fp16 rows of 768 took 100 us so, 91 this way)
            }
            row += step_rows; v += step_v;
            if (v >= vecs) { v -= vecs; ++row; }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (at_row[u] < 0) break;
            if (d.on) {
                float f[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = p[u].get(e);
                drop_vector<VEC>(d, key[u], at_v[u] * VEC, f);
                p[u].put(f);
            }
            p[u].store(y + at_row[u] * y_stride + at_v[u] * VEC);
        }
    }
}

// Dropout of rows of narrower vectors.  A warp takes 8 / VEC pieces of 32 * VEC channels of a row at a time, 32 blocks of the generator in all: every
// lane draws one and leaves it in shared memory for the lanes that have the elements.  Bound by instruction issue (73 % of the slots): 77,777 bf16 rows of
// 101 at any alignment 22.5 us; a block drawn by every lane for itself took 39.
template <typename T, int VEC>
__global__ void __launch_bounds__(kNormThreads, 5) k_dropout_pieces(const T* x, int64_t x_stride, T* y, int64_t y_stride, int32_t rows, int32_t channels, DropArgs d) {
    constexpr int P = 8 / VEC, kBlocks = 32 / P, kWide = 32 * VEC;   // pieces; blocks of the generator in each; channels of one
    __shared__ __align__(16) uint32_t words[kNormWarps][128];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t pieces = (channels + kWide - 1) / kWide;
    const int64_t step = (int64_t)gridDim.x * kNormWarps * P, first = ((int64_t)blockIdx.x * kNormWarps + warp) * P;
    const int32_t step_rows = (int32_t)(step / pieces), step_q = (int32_t)(step - (int64_t)step_rows * pieces);
    int64_t row = first / pieces;   // (beyond the rows by less than a step)
    int32_t q = (int32_t)(first - row * pieces);
    const int64_t x_wrap = x_stride - (int64_t)pieces * kWide, y_wrap = y_stride - (int64_t)pieces * kWide;
    while (row < rows) {
        Raw<T, VEC> p[P];
        uint32_t have = 0;
        int32_t drawn_row = (int32_t)row, drawn_c = 0;
        {
            const T* px = x + row * x_stride + (q * 32 + lane) * VEC;
            int32_t r = (int32_t)row, at = q;
#pragma unroll
            for (int k = 0; k < P; ++k) {
                if (lane / kBlocks == k) { drawn_row = r; drawn_c = at * kWide + lane % kBlocks * 8; }
                if (r < rows && (at * 32 + lane) * VEC < channels) { p[k].load(px); have |= 1u << k; }
                px += kWide;
                if (++at == pieces) { at = 0; ++r; px += x_wrap; }
            }
        }
        if (d.on) {
            uint32_t w[4];
            const uint64_t key = drop_key(d, min(drawn_row, rows - 1));
            drop_block(d, (uint32_t)key, (uint32_t)(key >> 32), (uint32_t)drawn_c >> 3, d.tag, w);
            __syncwarp();
            *reinterpret_cast<uint4*>(words[warp] + 4 * lane) = make_uint4(w[0], w[1], w[2], w[3]);
            __syncwarp();
        }
        T* py = y + row * y_stride + (q * 32 + lane) * VEC;
        int32_t at = q;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            if (have >> k & 1u) {
                if (d.on) {
                    const uint32_t* from = words[warp] + 4 * (k * kBlocks + lane * VEC / 8);
                    Keep<VEC> keep;
                    if constexpr (VEC == 1) keep.w[0] = reinterpret_cast<const uint16_t*>(from)[lane & 7];
                    else if constexpr (VEC == 2) keep.w[0] = from[lane & 3];
                    else {
                        const uint2 v = *reinterpret_cast<const uint2*>(from + (lane & 1) * 2);
                        keep.w[0] = v.x; keep.w[1] = v.y;
                    }
                    float f[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) f[e] = keep(d, e) ? p[k].get(e) * d.factor : 0.f;
                    p[k].put(f);
                }
                p[k].store(py);
            }
            py += kWide;
            if (++at == pieces) { at = 0; py += y_wrap; }
        }
        row += step_rows; q += step_q;
        if (q >= pieces) { q -= pieces; ++row; }
    }
}

// ---- group norm of single rows ----------------------------------------------------------
// The bytes bound it, and half of the issue slots go to the row's sums, the generator and the activation: 768,000 fp32 rows of 256 with a ReLU and a
// dropout 284 us, 5.5 TB/s; the gradient of 543,000 334 us, 5.0 TB/s.
// A row's vectors lie on 2^lanes lanes (all 32 where it has more than 32 vectors, NV of them per lane then); a warp holds 32 >> lanes rows.
// The groups are equal blocks of `1 << gshift` vectors (gshift 31: the whole row), or narrow ones of `width` whole vectors, summed up through shared
// memory, or of any width, taken one after the other under masks.
enum { ROW_EVEN = 0, ROW_NARROW = 1, ROW_MASKS = 2 };

struct RowShape { int32_t lanes, gshift, width; };

template <int NV>
__device__ __forceinline__ void group_sum(float (&s)[NV], const RowShape& r) {
    if (r.gshift >= 31) {
        float t = s[0];
#pragma unroll
        for (int i = 1; i < NV; ++i) t += s[i];
#pragma unroll
        for (int o = 0; o < 5; ++o) if (o < r.lanes) t += __shfl_xor_sync(0xFFFFFFFFu, t, 1 << o);
#pragma unroll
        for (int i = 0; i < NV; ++i) s[i] = t;
        return;
    }
    const int steps = min(r.gshift, r.lanes);
#pragma unroll
    for (int o = 0; o < 5; ++o) {
        if (o < steps) {
#pragma unroll
            for (int i = 0; i < NV; ++i) s[i] += __shfl_xor_sync(0xFFFFFFFFu, s[i], 1 << o);
        }
    }
    if (NV > 1 && r.gshift > 5) {   // (groups wider than a warp are of whole warps)
#pragma unroll
        for (int st = 1; st < NV; st <<= 1) {
            if (32 * st < 1 << r.gshift) {
                float t[NV];
#pragma unroll
                for (int i = 0; i < NV; ++i) t[i] = s[i] + s[i ^ st];
#pragma unroll
                for (int i = 0; i < NV; ++i) s[i] = t[i];
            }
        }
    }
}

// Sums over groups.  Narrow ones: a lane's vectors' sums to shared memory, then its groups' from there, all lanes of a group in the same order.
template <int NV, bool NARROW> struct Groups {
    float* buf = nullptr;   // the row's
    int32_t at[NARROW ? NV : 1], width = 0;   // the groups of a lane's vectors
    __device__ __forceinline__ Groups(float (&all)[kNormWarps][NARROW ? 32 * NV : 1], const RowShape& r, int sub, int32_t vecs) {
        if constexpr (NARROW) {
            width = r.width;   // (above 0)
            buf = all[threadIdx.x >> 5] + ((threadIdx.x & 31) - sub);
#pragma unroll
            for (int i = 0; i < NV; ++i) at[i] = sub + 32 * i < vecs ? (sub + 32 * i) / width : 0;
        }
    }
    __device__ __forceinline__ void sum(float (&s)[NV], const RowShape& r, int sub) const {
        if constexpr (NARROW) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < NV; ++i) buf[sub + 32 * i] = s[i];
            __syncwarp();
#pragma unroll
            for (int i = 0; i < NV; ++i) s[i] = buf[at[i] * width];
            for (int32_t j = 1; j < width; ++j) {
#pragma unroll
                for (int i = 0; i < NV; ++i) s[i] += buf[at[i] * width + j];
            }
        } else group_sum<NV>(s, r);
    }
    // a vector's group, and whether it is the group's first
    __device__ __forceinline__ int32_t of(int i, int32_t v, const RowShape& r) const {
        if constexpr (NARROW) return at[i];
        else return r.gshift >= 31 ? 0 : v >> r.gshift;
    }
    __device__ __forceinline__ bool first(int i, int32_t v, const RowShape& r) const {
        if constexpr (NARROW) return v == at[i] * width;
        else return r.gshift >= 31 ? v == 0 : (v & ((1 << r.gshift) - 1)) == 0;
    }
};

__device__ __forceinline__ float row_sum(float t, int lanes) {
#pragma unroll
    for (int o = 0; o < 5; ++o) if (o < lanes) t += __shfl_xor_sync(0xFFFFFFFFu, t, 1 << o);
    return t;
}

// Weight and bias of a lane's channels: held in registers where they are few, else read from shared memory again for every row.
template <int VEC, int NV, bool BACKWARD> struct Params {
    static constexpr bool kHeld = VEC * NV <= (BACKWARD ? 4 : 8);
    float w[kHeld ? NV : 1][VEC], b[kHeld ? NV : 1][VEC];
    const float* shared;
    int32_t channels;
    __device__ __forceinline__ Params(const NormArgs& a, float* smem, int sub, int32_t vecs) : shared(smem), channels(a.channels) {
        if constexpr (kHeld) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int32_t c = (sub + 32 * i) * VEC + e;
                    const bool in = sub + 32 * i < vecs;
                    w[i][e] = in && a.weight ? a.weight[c] : 1.f;
                    b[i][e] = in && a.bias ? a.bias[c] : 0.f;
                }
        } else {
            for (int32_t c = threadIdx.x; c < a.channels; c += kNormThreads) {
                smem[c] = a.weight ? a.weight[c] : 1.f;
                smem[a.channels + c] = a.bias ? a.bias[c] : 0.f;
            }
            __syncthreads();
        }
    }
    __device__ __forceinline__ static void read(const float* s, float (&o)[VEC]) {
        if constexpr (VEC % 4 == 0) {
#pragma unroll
            for (int q = 0; q < VEC; q += 4) {
                const float4 f = *reinterpret_cast<const float4*>(s + q);
                o[q] = f.x; o[q + 1] = f.y; o[q + 2] = f.z; o[q + 3] = f.w;
            }
        } else {
#pragma unroll
            for (int q = 0; q < VEC; ++q) o[q] = s[q];
        }
    }
    __device__ __forceinline__ void get(int i, int32_t v, float (&wo)[VEC], float (&bo)[VEC]) const {
        if constexpr (kHeld) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) { wo[e] = w[i][e]; bo[e] = b[i][e]; }
        } else {
            read(shared + v * VEC, wo);
            read(shared + channels + v * VEC, bo);
        }
    }
};

template <typename T, int VEC, int NV, int CUT>
__global__ void __launch_bounds__(kNormThreads) k_norm_rows(NormArgs a, RowShape r) {
    extern __shared__ __align__(16) float params[];   // [2][channels], where they are not held
    const int lane = threadIdx.x & 31, sub = lane & ((1 << r.lanes) - 1), per_warp = 32 >> r.lanes;
    const int32_t vecs = a.channels / VEC;
    const float inv = 1.f / (float)a.each;
    const T* x = static_cast<const T*>(a.x);
    T* y = static_cast<T*>(a.out);
    const Params<VEC, NV, false> par(a, params, sub, vecs);
    __shared__ float vector_sums[kNormWarps][CUT == ROW_NARROW ? 32 * NV : 1];
    const Groups<NV, CUT == ROW_NARROW> groups(vector_sums, r, sub, vecs);
    const int64_t step = (int64_t)gridDim.x * kNormWarps * per_warp;
    constexpr bool kAhead = VEC * NV <= 16;   // the next row is on its way while this one is worked on
    Raw<T, VEC> raw[NV], next[kAhead ? NV : 1];
    int64_t row = (blockIdx.x * (int64_t)kNormWarps + (threadIdx.x >> 5)) * per_warp + (lane >> r.lanes);
    const auto fetch = [&](Raw<T, VEC>* to, int64_t from) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            to[i].zero();
            if (from < a.rows && sub + 32 * i < vecs) to[i].load(x + from * a.x_stride + (sub + 32 * i) * VEC);
        }
    };
    if (kAhead) fetch(next, row);
    for (; row - (lane >> r.lanes) < a.rows; row += step) {
        const bool here = row < a.rows;
        float f[NV][VEC];
        if constexpr (kAhead) {
#pragma unroll
            for (int i = 0; i < NV; ++i) raw[i] = next[i];
            fetch(next, row + step);
        } else fetch(raw, row);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[i][e] = raw[i].get(e);
        if constexpr (CUT == ROW_MASKS) {   // f becomes the normalised value
            for (int32_t g = 0, lo = 0; g < a.groups; ++g, lo += a.each) {
                float s = 0.f, q = 0.f;
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) if ((uint32_t)((sub + 32 * i) * VEC + e - lo) < (uint32_t)a.each) s += f[i][e];
                const float mean = row_sum(s, r.lanes) * inv;
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) if ((uint32_t)((sub + 32 * i) * VEC + e - lo) < (uint32_t)a.each) { f[i][e] -= mean; q = fmaf(f[i][e], f[i][e], q); }
                const float rstd = rsqrtf(row_sum(q, r.lanes) * inv + a.eps);
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) if ((uint32_t)((sub + 32 * i) * VEC + e - lo) < (uint32_t)a.each) f[i][e] *= rstd;
                if (here && sub == 0) { a.mean[row * a.groups + g] = mean; a.rstd[row * a.groups + g] = rstd; }
            }
        } else {
            float s[NV], q[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                s[i] = 0.f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) s[i] += f[i][e];
            }
            groups.sum(s, r, sub);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                s[i] *= inv; q[i] = 0.f;
                const bool in = sub + 32 * i < vecs;   // (a lane without a vector would count the mean)
#pragma unroll
                for (int e = 0; e < VEC; ++e) { f[i][e] -= s[i]; q[i] = fmaf(f[i][e], f[i][e], q[i]); }
                if (!in) q[i] = 0.f;
            }
            groups.sum(q, r, sub);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const float rstd = rsqrtf(q[i] * inv + a.eps);
                const int32_t v = sub + 32 * i;
                if (here && v < vecs && groups.first(i, v, r)) {
                    const int64_t at = row * a.groups + groups.of(i, v, r);
                    a.mean[at] = s[i]; a.rstd[at] = rstd;
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[i][e] *= rstd;
            }
        }
        const uint64_t key = here && a.drop.on ? drop_key(a.drop, row) : 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int32_t v = sub + 32 * i;
            if (!here || v >= vecs) continue;
            float w[VEC], b[VEC];
            par.get(i, v, w, b);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[i][e] = fmaf(f[i][e], w[e], b[e]);
            act_values<VEC>(a.act, f[i]);
            drop_vector<VEC>(a.drop, key, v * VEC, f[i]);
            raw[i].put(f[i]);
            raw[i].store(y + row * a.out_stride + v * VEC);
        }
    }
}

// Gradient: dz = dropout(dy) act', then dx = rstd (dz w - mean(dz w) - hat mean(dz w hat)); every lane adds up dz hat and dz of its channels over
// its rows, every block its lanes', and k_norm_params the blocks'.
template <typename T, int VEC, int NV, int CUT>
__global__ void __launch_bounds__(kNormThreads, VEC * NV <= 8 ? 3 : 1) k_norm_rows_backward(NormArgs a, RowShape r) {
    extern __shared__ __align__(16) float params[];   // [2][channels], where they are not held; then the block's sums [2][channels]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane & ((1 << r.lanes) - 1), per_warp = 32 >> r.lanes;
    const int32_t vecs = a.channels / VEC;
    const float inv = 1.f / (float)a.each;
    const T* x = static_cast<const T*>(a.x);
    const T* d_y = static_cast<const T*>(a.d_y);
    T* d_x = static_cast<T*>(a.out);
    const Params<VEC, NV, true> par(a, params, sub, vecs);
    __shared__ float vector_sums[kNormWarps][CUT == ROW_NARROW ? 32 * NV : 1];
    const Groups<NV, CUT == ROW_NARROW> groups(vector_sums, r, sub, vecs);
    float* sums = params + (Params<VEC, NV, true>::kHeld ? 0 : 2 * a.channels);
    float dw[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) dw[i][e] = db[i][e] = 0.f;
    const int64_t step = (int64_t)gridDim.x * kNormWarps * per_warp;
    Raw<T, VEC> rx[NV], rd[NV];
    int64_t row = (blockIdx.x * (int64_t)kNormWarps + warp) * per_warp + (lane >> r.lanes);
    const auto fetch = [&](Raw<T, VEC>* to_x, Raw<T, VEC>* to_d, int64_t from) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            to_x[i].zero(); to_d[i].zero();
            if (from < a.rows && sub + 32 * i < vecs) {
                to_x[i].load(x + from * a.x_stride + (sub + 32 * i) * VEC);
                to_d[i].load(d_y + from * a.d_y_stride + (sub + 32 * i) * VEC);
            }
        }
    };
    for (; row - (lane >> r.lanes) < a.rows; row += step) {
        const bool here = row < a.rows;
        float h[NV][VEC], g[NV][VEC], rstd[NV];
        fetch(rx, rd, row);
        const uint64_t key = here && a.drop.on ? drop_key(a.drop, row) : 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int32_t v = sub + 32 * i;
            const bool in = here && v < vecs;
            float w[VEC], b[VEC];
            par.get(i, in ? v : 0, w, b);
            rstd[i] = 0.f;
            if constexpr (CUT == ROW_MASKS) {   // (every element has statistics of its own)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int64_t at = row * a.groups + (v * VEC + e) / a.each;
                    const float m_e = in ? a.mean[at] : 0.f, r_e = in ? a.rstd[at] : 0.f, x1 = rx[i].get(e), b1[1] = {b[e]};
                    float d1[1] = {rd[i].get(e)};
                    h[i][e] = (x1 - m_e) * r_e;
                    const float n1[1] = {fmaf(h[i][e], w[e], b[e])};
                    act_slopes<1>(a.act, d1, n1, b1, [&](int) { return ((double)x1 - (double)m_e) * (double)r_e * (double)w[e] + (double)b[e]; });
                    g[i][e] = d1[0];
                }
                if (a.drop.on) {
                    Keep<VEC> keep;
                    keep.draw(a.drop, key, (uint32_t)(v * VEC));
#pragma unroll
                    for (int e = 0; e < VEC; ++e) g[i][e] = keep(a.drop, e) ? g[i][e] * a.drop.factor : 0.f;
                }
            } else {
                float mean = 0.f;
                if (in) {
                    const int64_t at = row * a.groups + groups.of(i, v, r);
                    mean = a.mean[at]; rstd[i] = a.rstd[at];
                }
                grad_vector<T, VEC>(a, rx[i], rd[i], key, v * VEC, mean, rstd[i], w, b, h[i], g[i]);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if (!in) g[i][e] = 0.f;
                dw[i][e] = fmaf(g[i][e], h[i][e], dw[i][e]); db[i][e] += g[i][e];
                g[i][e] *= w[e];
            }
        }
        if constexpr (CUT == ROW_MASKS) {
            for (int32_t q = 0, lo = 0; q < a.groups; ++q, lo += a.each) {
                float s1 = 0.f, s2 = 0.f;
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if ((uint32_t)((sub + 32 * i) * VEC + e - lo) < (uint32_t)a.each) { s1 += g[i][e]; s2 = fmaf(g[i][e], h[i][e], s2); }
                s1 = row_sum(s1, r.lanes) * inv; s2 = row_sum(s2, r.lanes) * inv;
                const float r_q = here ? a.rstd[row * a.groups + q] : 0.f;
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if ((uint32_t)((sub + 32 * i) * VEC + e - lo) < (uint32_t)a.each) g[i][e] = r_q * (g[i][e] - s1 - h[i][e] * s2);
            }
        } else {
            float s1[NV], s2[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                s1[i] = s2[i] = 0.f;
#pragma unroll
                for (int e = 0; e < VEC; ++e) { s1[i] += g[i][e]; s2[i] = fmaf(g[i][e], h[i][e], s2[i]); }
            }
            groups.sum(s1, r, sub);
            groups.sum(s2, r, sub);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) g[i][e] = rstd[i] * (g[i][e] - s1[i] * inv - h[i][e] * (s2[i] * inv));
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int32_t v = sub + 32 * i;
            if (!here || v >= vecs) continue;
            rx[i].put(g[i]);
            rx[i].store(d_x + row * a.out_stride + v * VEC);
        }
    }
    if (!a.parts) return;
    // the warp's rows, then the block's warps one after the other
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            for (int o = 1 << r.lanes; o < 32; o <<= 1) {
                dw[i][e] += __shfl_xor_sync(0xFFFFFFFFu, dw[i][e], o);
                db[i][e] += __shfl_xor_sync(0xFFFFFFFFu, db[i][e], o);
            }
    for (int q = 0; q < kNormWarps; ++q) {
        if (q == warp && lane == sub) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int32_t v = sub + 32 * i;
                if (v >= vecs) continue;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    float* at = sums + v * VEC + e;
                    at[0] = q ? at[0] + dw[i][e] : dw[i][e];
                    at[a.channels] = q ? at[a.channels] + db[i][e] : db[i][e];
                }
            }
        }
        __syncthreads();
    }
    float* part = a.parts + (int64_t)blockIdx.x * 2 * a.channels;
    for (int32_t c = threadIdx.x; c < 2 * a.channels; c += kNormThreads) part[c] = sums[c];
}

}  // namespace mgnorm
