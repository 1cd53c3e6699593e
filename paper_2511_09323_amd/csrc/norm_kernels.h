// Layer norm and the gradients of layer norm and RMSNorm.
//
// A row h of d values: n = (h - mean) r, r = 1 / sqrt(mean((h - mean)^2) + eps), out = n gain + bias; RMSNorm has mean = 0 and no
// bias.  With p = dy gain:  dh = r (p - mean(p) - n mean(p n)) (+ dres),  dgain = sum over rows of dy n,  dbias = sum of dy;
// RMSNorm's dh lacks mean(p).  Everything is fp32; the variance is the mean of squared differences from the mean (a sum of squares
// would lose a mean that is large against the spread); dh, out, dgain and dbias are rounded once.
//
// All of it is bound by memory, so every row is read once: TPR lanes hold it in registers, as NV pieces of 16 bytes each, and the
// statistics are computed again in the backward pass instead of being stored.
#pragma once
#include "common.h"
#include "misc_kernels.h"

namespace moc {

// How the pieces of a row lie.  A load stands in no branch: behind one, the compiler cannot count what is still on its way and waits for everything.
//   Whole    rows are whole pieces; pieces past a row's end read as zero (buffer loads check the bound);
//   Odd      any d from a piece's width W on: the last piece is the row's last W elements, and those of them that the piece before it has are
//            zeroed; pieces past the end read that, too, and are zeroed;
//   Narrow   d < W: element by element.
enum class RowForm { Whole, Odd, Narrow };

template <class E, RowForm FORM, int NV, int TPR> struct Row {
    static constexpr int W = Vec16<E>::N;
    int d, lane;
    __device__ __forceinline__ int at(int u) const { return (u * TPR + lane) * W; }                             // the piece's first column
    __device__ __forceinline__ int first(int u) const { return FORM == RowForm::Odd ? min(at(u), d - W) : at(u); }      // the column of its element 0
    // whether some lane's piece u is not W elements of its own (uniform)
    __device__ __forceinline__ bool ragged(int u) const { return FORM != RowForm::Whole && (u + 1) * TPR * W > d; }
    __device__ __forceinline__ bool has(int u, int e) const { return first(u) + e >= at(u) && first(u) + e < d; }
    // Row t of p (t the same in a wavefront), or zeros where `in` is false; p has T rows.
    __device__ __forceinline__ void load(const E* p, int64_t t, int T, bool in, u32x4_t* raw) const {
        if (FORM == RowForm::Whole) {
            const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<E*>(p + (in ? t * d : 0)), 0, in ? (uint32_t)d * sizeof(E) : 0u, 0x00020000);
#pragma unroll
            for (int u = 0; u < NV; ++u) raw[u] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (u * TPR + lane) * 16, 0, 0));
        } else if (FORM == RowForm::Odd) {
            const E* row = p + (in ? t : (int64_t)T - 1) * d;
#pragma unroll
            for (int u = 0; u < NV; ++u) __builtin_memcpy(&raw[u], row + first(u), 16);
        } else {
            float v[W];
#pragma unroll
            for (int e = 0; e < W; ++e) v[e] = in && has(0, e) ? Elem<E>::load(p + t * d + e) : 0.0f;
            raw[0] = Vec16<E>::pack(v);      // (exact: these are E's values)
        }
    }
    // What the loads of an Odd row brought that is not the lane's own becomes zero.  (Apart from the load, which would be waited for.)
    __device__ __forceinline__ void clean(bool in, u32x4_t* raw) const {
        if (FORM != RowForm::Odd) return;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            if (in && !ragged(u)) continue;
            float v[W];
            Vec16<E>::unpack(raw[u], v);
#pragma unroll
            for (int e = 0; e < W; ++e) v[e] = in && has(u, e) ? v[e] : 0.0f;
            raw[u] = Vec16<E>::pack(v);
        }
    }
    __device__ __forceinline__ void store(E* row, int u, const float* v) const {
        if (FORM == RowForm::Whole) {
            const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(row, 0, (uint32_t)d * sizeof(E), 0x00020000);
            __builtin_amdgcn_raw_buffer_store_b128(Vec16<E>::pack(v), rsrc, (u * TPR + lane) * 16, 0, 0);
        } else if (!ragged(u)) {
            const u32x4_t r = Vec16<E>::pack(v);
            __builtin_memcpy(row + at(u), &r, 16);
        } else {
#pragma unroll
            for (int e = 0; e < W; ++e)
                if (has(u, e)) Elem<E>::store(row + first(u) + e, v[e]);
        }
    }
};

// Sum over the TPR lanes of a row, for all of them.  `red` holds the wavefronts' sums; consecutive calls alternate between its two
// halves, so that one barrier a call is enough.
constexpr int kMaxRowWaves = 16;      // wavefronts of a workgroup that walks over rows
struct RowSums {
    float (*red)[kMaxRowWaves];
    int turn = 0;
    template <int TPR> __device__ __forceinline__ float sum(float v) {
        v = wave_sum(v);
        if (TPR == 64) return v;
        const int wave = threadIdx.x >> 6, first = wave & ~(TPR / 64 - 1);
        if ((threadIdx.x & 63) == 0) red[turn][wave] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) v += red[turn][first + w];
        turn ^= 1;
        return v;
    }
};

// mean and 1 / sqrt(variance + eps) of the row whose pieces are in raw.
template <class E, RowForm FORM, int NV, int TPR, bool RMS>
__device__ __forceinline__ void row_stats(const Row<E, FORM, NV, TPR>& row, const u32x4_t* raw, float eps, RowSums& sums, float& mean, float& r) {
    constexpr int W = Vec16<E>::N;
    mean = 0.0f;
    const float scale = 1.0f / (float)row.d;
    if (!RMS) {
        float s = 0.0f;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            float v[W];
            Vec16<E>::unpack(raw[u], v);
#pragma unroll
            for (int e = 0; e < W; ++e) s += v[e];
        }
        mean = sums.sum<TPR>(s) * scale;
    }
    float ss = 0.0f;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        float v[W];
        Vec16<E>::unpack(raw[u], v);
        if (RMS || (FORM == RowForm::Whole ? row.at(u) < row.d : !row.ragged(u))) {
#pragma unroll
            for (int e = 0; e < W; ++e) ss = fmaf(v[e] - mean, v[e] - mean, ss);
        } else if (FORM != RowForm::Whole) {
#pragma unroll
            for (int e = 0; e < W; ++e) ss = row.has(u, e) ? fmaf(v[e] - mean, v[e] - mean, ss) : ss;
        }
    }
    r = 1.0f / sqrtf(sums.sum<TPR>(ss) * scale + eps);
}

// One row per TPR lanes.  out may be h.  bf16, 8192 x 4096, from memory: 134 MB in 29 us, 4.6 TB/s (a large copy: 5.2).
template <class E, RowForm FORM, int NV, int TPR>
__global__ __launch_bounds__(256) void layernorm_kernel(const E* h, const E* __restrict__ gain, const E* __restrict__ bias, float eps, int T, int d, E* out) {
    constexpr int W = Vec16<E>::N;
    __shared__ float red[2][kMaxRowWaves];
    RowSums sums{red};
    const Row<E, FORM, NV, TPR> row{d, (int)threadIdx.x % TPR};
    const int64_t t = (int64_t)blockIdx.x * (256 / TPR) + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);      // (the same in a whole wavefront)
    const bool in = t < T;      // (rows past the last wait with the others)
    u32x4_t raw[NV], rg[NV], rb[NV];
    row.load(h, t, T, in, raw);
    row.load(gain, 0, 1, true, rg);
    row.load(bias ? bias : gain, 0, 1, true, rb);
    row.clean(in, raw);
    float mean, r;
    row_stats<E, FORM, NV, TPR, false>(row, raw, eps, sums, mean, r);
    if (!in) return;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        float v[W], g[W], b[W];
        Vec16<E>::unpack(raw[u], v);
        Vec16<E>::unpack(rg[u], g);
        Vec16<E>::unpack(bias ? rb[u] : u32x4_t{0, 0, 0, 0}, b);
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] = fmaf((v[e] - mean) * r, g[e], b[e]);
        row.store(out + t * d, u, v);
    }
}

// Backward: one workgroup a compute unit; every TPR lanes walk over rows, with the next row on its way while one is worked on, and add dy n and
// dy up in registers.  (Loads come back in order, so nothing that is needed sooner is asked for after the next row: the gain is in LDS.)
// A workgroup's sums are joined in LDS and written as one row of `part` ([workgroup][dgain, dbias][d]), or, where there is a single
// workgroup, to dgain and dbias themselves.  dh may be dy or dres: an element is read by the lane that writes it, and where the lane beside it reads it too, it has
// no use for it.  bf16, from memory: layer norm 8192 x 4096 201 MB in 40.5 us (5.0 TB/s), RMSNorm with dres 8192 x 2048 134 MB in 27 us (5.0 TB/s).
constexpr int kNormThreads = 512;
template <class E, RowForm FORM, int NV, int TPR, bool RMS, bool BIAS>
__global__ __launch_bounds__(kNormThreads) void norm_bwd_kernel(const E* __restrict__ h, const E* __restrict__ gain, float eps, const E* dy, const E* dres, int T, int d, E* dh,
                                                                float* __restrict__ part, E* __restrict__ dgain, E* __restrict__ dbias) {
    constexpr int W = Vec16<E>::N, ROWS = kNormThreads / TPR;
    constexpr bool AHEAD = NV <= 4;      // (more pieces leave no registers for a second row)
    __shared__ float red[2][kMaxRowWaves];
    constexpr int PASS = NV < 16 / W ? NV : 16 / W;      // 32 KB of LDS
    __shared__ __align__(16) float join[ROWS == 1 ? 1 : ROWS][ROWS == 1 ? 1 : PASS * TPR * W];
    __shared__ u32x4_t gains[AHEAD ? NV * TPR : 1];
    RowSums sums{red};
    const Row<E, FORM, NV, TPR> row{d, (int)threadIdx.x % TPR};
    const int lane = row.lane, slot = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);      // (the same in a whole wavefront)
    const float scale = 1.0f / (float)d;
    float ag[NV * W], ab[BIAS ? NV * W : 1];
#pragma unroll
    for (int i = 0; i < NV * W; ++i) ag[i] = 0.0f;
    if (BIAS) {
#pragma unroll
        for (int i = 0; i < NV * W; ++i) ab[i] = 0.0f;
    }
    u32x4_t rh[NV], ry[NV], nh[NV], ny[NV];
    const int64_t step = (int64_t)gridDim.x * ROWS;
    // (every lane goes through the same number of rows: sums over more than a wavefront synchronise the workgroup)
    int64_t t0 = (int64_t)blockIdx.x * ROWS;
    if (AHEAD) {
        u32x4_t g[NV];
        row.load(gain, 0, 1, true, g);
        row.load(h, t0 + slot, T, t0 + slot < T, nh);
        row.load(dy, t0 + slot, T, t0 + slot < T, ny);
        if (slot == 0) {
#pragma unroll
            for (int u = 0; u < NV; ++u) gains[u * TPR + lane] = g[u];
        }
        __syncthreads();
    }
    for (; t0 < T; t0 += step) {
        const int64_t t = t0 + slot, next = t + step;
        const bool in = t < T;
        u32x4_t rr[NV], rg[NV];
        if (dres) row.load(dres, t, T, in, rr);
        if (AHEAD) {
#pragma unroll
            for (int u = 0; u < NV; ++u) rh[u] = nh[u], ry[u] = ny[u];
            row.load(h, next, T, next < T, nh);
            row.load(dy, next, T, next < T, ny);
        } else {
            row.load(h, t, T, in, rh);
            row.load(dy, t, T, in, ry);
            row.load(gain, 0, 1, true, rg);
        }
        row.clean(in, rh);
        row.clean(in, ry);
        float mean, r;
        row_stats<E, FORM, NV, TPR, RMS>(row, rh, eps, sums, mean, r);
        r = in ? r : 0.0f;      // (a slot without a row holds zeros, whose 1 / sqrt(0 + eps) is no number to multiply by where eps is 0; its n is 0 and adds nothing)
        float sp = 0.0f, spn = 0.0f;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            float x[W], y[W], g[W];
            Vec16<E>::unpack(rh[u], x);
            Vec16<E>::unpack(ry[u], y);
            Vec16<E>::unpack(AHEAD ? gains[u * TPR + lane] : rg[u], g);
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const float n = (x[e] - mean) * r, p = y[e] * g[e];      // (past the row's end y and p are zero)
                if (!RMS) sp += p;
                spn = fmaf(p, n, spn);
                ag[u * W + e] = fmaf(y[e], n, ag[u * W + e]);
                if (BIAS) ab[u * W + e] += y[e];
            }
        }
        const float m1 = RMS ? 0.0f : sums.sum<TPR>(sp) * scale, m2 = sums.sum<TPR>(spn) * scale;
        if (!in) continue;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            float x[W], y[W], g[W], o[W];
            Vec16<E>::unpack(rh[u], x);
            Vec16<E>::unpack(ry[u], y);
            Vec16<E>::unpack(AHEAD ? gains[u * TPR + lane] : rg[u], g);
            Vec16<E>::unpack(dres ? rr[u] : u32x4_t{0, 0, 0, 0}, o);
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const float n = (x[e] - mean) * r;
                o[e] = fmaf(r, fmaf(-n, m2, fmaf(y[e], g[e], -m1)), o[e]);
            }
            row.store(dh + t * d, u, o);
        }
    }
    // the workgroup's sums, PASS pieces of a lane at a time
    const bool last = gridDim.x == 1;
    constexpr int SUMS = BIAS ? 2 : 1;
    float* mine = part + (int64_t)blockIdx.x * SUMS * d;
#pragma unroll
    for (int q = 0; q < SUMS; ++q) {
        const float* a = q ? ab : ag;
        E* const out = q ? dbias : dgain;
        const auto result = [&](int i, float s) {
            if (last) Elem<E>::store(out + i, s);
            else mine[q * d + i] = s;
        };
        if (ROWS == 1) {
#pragma unroll
            for (int u = 0; u < NV; ++u)
#pragma unroll
                for (int e = 0; e < W; ++e)
                    if (row.has(u, e)) result(row.first(u) + e, a[u * W + e]);
            continue;
        }
#pragma unroll
        for (int u0 = 0; u0 < NV; u0 += PASS) {
            const int c0 = u0 * TPR * W;
            if (c0 >= d) break;      // (uniform)
            __syncthreads();
#pragma unroll
            for (int u = u0; u < u0 + PASS; ++u) {
                float* at = &join[slot][row.at(u) - c0];
                if (!row.ragged(u)) {      // (16 bytes at a time: single words, 32 bytes apart from lane to lane, take 3 us longer at 1000 x 2048)
#pragma unroll
                    for (int e = 0; e < W; e += 4) *reinterpret_cast<f32x4_t*>(at + e) = f32x4_t{a[u * W + e], a[u * W + e + 1], a[u * W + e + 2], a[u * W + e + 3]};
                } else {
#pragma unroll
                    for (int e = 0; e < W; ++e)
                        if (row.has(u, e)) join[slot][row.first(u) + e - c0] = a[u * W + e];
                }
            }
            __syncthreads();
            for (int c = threadIdx.x; c < min(PASS * TPR * W, d - c0); c += kNormThreads) {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < ROWS; ++w) s += join[w][c];
                result(c0 + c, s);
            }
        }
    }
}

// Sums over the workgroups' rows of `part`, in their order: 64 columns and 16 shares of the rows a workgroup; a share's rows are asked for together.  256 rows of 2 x 4096:
// 4.7 us, of which starting is 1.3.
constexpr int kNormGroups = 256;        // most workgroups of a backward launch, one a compute unit: rows of `part`
template <class E>
__global__ __launch_bounds__(1024) void norm_bwd_join_kernel(const float* __restrict__ part, int rows, int64_t cols, int d, E* __restrict__ dgain, E* __restrict__ dbias) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, share = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float v[kNormGroups / 16];
#pragma unroll
    for (int i = 0; i < kNormGroups / 16; ++i) {
        const int p = share + 16 * i;
        v[i] = p < rows && c < cols ? part[p * cols + c] : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kNormGroups / 16; ++i) s += v[i];
    sums[share][lane] = s;
    __syncthreads();
    if (share != 0 || c >= cols) return;
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += sums[w][lane];
    Elem<E>::store(c < d ? dgain + c : dbias + (c - d), s);
}

}  // namespace moc
