// Layer norm and the gradients of layer norm and RMSNorm.
//
// A row h of d values: n = (h - mean) r, r = 1 / sqrt(mean((h - mean)^2) + eps), out = n gain + bias; RMSNorm has mean = 0 and no
// bias.  With p = dy gain:  dh = r (p - mean(p) - n mean(p n)) (+ dres),  dgain = sum over rows of dy n,  dbias = sum of dy;
// RMSNorm's dh lacks mean(p).  Everything is fp32; the variance is the mean of squared differences from the mean (a sum of squares
// would lose a mean that is large against the spread); dh, out, dgain and dbias are rounded once.
//
// All of it is bound by memory, so every row is read once: TPR lanes hold it in registers, as NV pieces of W elements each (W = 16
// bytes' worth where rows are 16-byte aligned, else 1), and the statistics are computed again in the backward pass instead of being
// stored.  TPR = 64 needs no barrier; more lanes are for long rows, and for few of them.
#pragma once
#include "common.h"
#include "misc_kernels.h"

namespace moc {

template <class E, int W> struct Piece {
    static_assert(W == Vec16<E>::N, "16 bytes, or one element (below)");
    typedef u32x4_t Raw;
    static __device__ __forceinline__ Raw zero() { return u32x4_t{0, 0, 0, 0}; }
    static __device__ __forceinline__ Raw load(const E* p) { return *reinterpret_cast<const u32x4_t*>(p); }
    static __device__ __forceinline__ void unpack(Raw r, float* v) { Vec16<E>::unpack(r, v); }
    static __device__ __forceinline__ void store(E* p, const float* v) { *reinterpret_cast<u32x4_t*>(p) = Vec16<E>::pack(v); }
};
template <class E> struct Piece<E, 1> {
    typedef E Raw;
    static __device__ __forceinline__ Raw zero() { return E(0); }
    static __device__ __forceinline__ Raw load(const E* p) { return *p; }
    static __device__ __forceinline__ void unpack(Raw r, float* v) { v[0] = Elem<E>::load(&r); }
    static __device__ __forceinline__ void store(E* p, const float* v) { Elem<E>::store(p, v[0]); }
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

// mean and 1 / sqrt(variance + eps) of the row whose pieces are in raw (pieces past the row's end are zero).
template <class E, int W, int NV, int TPR, bool RMS>
__device__ __forceinline__ void row_stats(const typename Piece<E, W>::Raw* raw, int lane, int d, float eps, RowSums& sums, float& mean, float& r) {
    mean = 0.0f;
    const float scale = 1.0f / (float)d;
    if (!RMS) {
        float s = 0.0f;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            float v[W];
            Piece<E, W>::unpack(raw[u], v);
#pragma unroll
            for (int e = 0; e < W; ++e) s += v[e];
        }
        mean = sums.sum<TPR>(s) * scale;
    }
    float ss = 0.0f;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        float v[W];
        Piece<E, W>::unpack(raw[u], v);
        if (RMS || (u * TPR + lane) * W < d) {
#pragma unroll
            for (int e = 0; e < W; ++e) ss = fmaf(v[e] - mean, v[e] - mean, ss);
        }
    }
    r = 1.0f / sqrtf(sums.sum<TPR>(ss) * scale + eps);
}

// One row per TPR lanes.  out may be h.
template <class E, int W, int NV, int TPR>
__global__ __launch_bounds__(256) void layernorm_kernel(const E* h, const E* __restrict__ gain, const E* __restrict__ bias, float eps, int T, int d,
                                                        E* out) {
    __shared__ float red[2][kMaxRowWaves];
    RowSums sums{red};
    const int lane = threadIdx.x % TPR;
    const int64_t t = (int64_t)blockIdx.x * (256 / TPR) + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);      // (the same in a whole wavefront)
    const int width = t < T ? d : 0;      // (rows past the last wait with the others)
    const E* x = h + t * d;
    typename Piece<E, W>::Raw raw[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        const int i = (u * TPR + lane) * W;
        raw[u] = i < width ? Piece<E, W>::load(x + i) : Piece<E, W>::zero();
    }
    float mean, r;
    row_stats<E, W, NV, TPR, false>(raw, lane, d, eps, sums, mean, r);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        const int i = (u * TPR + lane) * W;
        if (i >= width) continue;
        float v[W], g[W], b[W];
        Piece<E, W>::unpack(raw[u], v);
        Piece<E, W>::unpack(Piece<E, W>::load(gain + i), g);
        Piece<E, W>::unpack(bias ? Piece<E, W>::load(bias + i) : Piece<E, W>::zero(), b);
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] = fmaf((v[e] - mean) * r, g[e], b[e]);
        Piece<E, W>::store(out + t * d + i, v);
    }
}

// Backward: every TPR lanes walk over rows and add dy n and dy up in registers; a workgroup's sums are joined in LDS and written as
// one row of `part` ([workgroup][dgain, dbias][d]), or, where there is a single workgroup, to dgain and dbias themselves.  dh may
// be dy or dres: an element is read by the lane that writes it.
template <class E, int W, int NV, int TPR, int THREADS, bool RMS, bool BIAS>
__global__ __launch_bounds__(THREADS) void norm_bwd_kernel(const E* __restrict__ h, const E* __restrict__ gain, float eps, const E* dy, const E* dres, int T, int d, E* dh,
                                                           float* __restrict__ part, E* __restrict__ dgain, E* __restrict__ dbias) {
    constexpr int ROWS = THREADS / TPR;
    __shared__ float red[2][kMaxRowWaves];
    __shared__ float join[ROWS == 1 ? 1 : ROWS][ROWS == 1 ? 1 : TPR * W];
    RowSums sums{red};
    const int lane = threadIdx.x % TPR, slot = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);      // (the same in a whole wavefront)
    const float scale = 1.0f / (float)d;
    float ag[NV * W], ab[BIAS ? NV * W : 1];
#pragma unroll
    for (int i = 0; i < NV * W; ++i) ag[i] = 0.0f;
    if (BIAS) {
#pragma unroll
        for (int i = 0; i < NV * W; ++i) ab[i] = 0.0f;
    }
    // (every lane goes through the same number of rows: sums over more than a wavefront synchronise the workgroup)
    for (int64_t t0 = (int64_t)blockIdx.x * ROWS; t0 < T; t0 += (int64_t)gridDim.x * ROWS) {
        const int64_t t = t0 + slot;
        const int width = t < T ? d : 0;
        typename Piece<E, W>::Raw rh[NV], ry[NV];
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int i = (u * TPR + lane) * W;
            rh[u] = i < width ? Piece<E, W>::load(h + t * d + i) : Piece<E, W>::zero();
            ry[u] = i < width ? Piece<E, W>::load(dy + t * d + i) : Piece<E, W>::zero();
        }
        float mean, r;
        row_stats<E, W, NV, TPR, RMS>(rh, lane, d, eps, sums, mean, r);
        float sp = 0.0f, spn = 0.0f;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int i = (u * TPR + lane) * W;
            float x[W], y[W], g[W];
            Piece<E, W>::unpack(rh[u], x);
            Piece<E, W>::unpack(ry[u], y);
            Piece<E, W>::unpack(i < d ? Piece<E, W>::load(gain + i) : Piece<E, W>::zero(), g);
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
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            const int i = (u * TPR + lane) * W;
            if (i >= width) continue;
            float x[W], y[W], g[W], o[W];
            Piece<E, W>::unpack(rh[u], x);
            Piece<E, W>::unpack(ry[u], y);
            Piece<E, W>::unpack(Piece<E, W>::load(gain + i), g);
            Piece<E, W>::unpack(dres ? Piece<E, W>::load(dres + t * d + i) : Piece<E, W>::zero(), o);
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const float n = (x[e] - mean) * r;
                o[e] = fmaf(r, fmaf(-n, m2, fmaf(y[e], g[e], -m1)), o[e]);
            }
            Piece<E, W>::store(dh + t * d + i, o);
        }
    }
    // the workgroup's sums, columns of one piece at a time
    const bool last = gridDim.x == 1;
    constexpr int SUMS = BIAS ? 2 : 1;
    float* mine = part + (int64_t)blockIdx.x * SUMS * d;
#pragma unroll
    for (int q = 0; q < SUMS; ++q) {
        const float* a = q ? ab : ag;
        E* const out = q ? dbias : dgain;
#pragma unroll
        for (int u = 0; u < NV; ++u) {
            if (ROWS == 1) {
                const int i = (u * TPR + lane) * W;
                if (i >= d) continue;
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    if (last) Elem<E>::store(out + i + e, a[u * W + e]);
                    else mine[q * d + i + e] = a[u * W + e];
                }
            } else {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < W; ++e) join[slot][lane * W + e] = a[u * W + e];
                __syncthreads();
                for (int c = threadIdx.x; c < TPR * W; c += THREADS) {
                    const int i = u * TPR * W + c;
                    if (i >= d) continue;
                    float s = 0.0f;
#pragma unroll
                    for (int w = 0; w < ROWS; ++w) s += join[w][c];
                    if (last) Elem<E>::store(out + i, s);
                    else mine[q * d + i] = s;
                }
            }
        }
    }
}

// Sums over the workgroups' rows of `part`, in their order: 64 columns and 16 shares of the rows a workgroup.
template <class E>
__global__ __launch_bounds__(1024) void norm_bwd_join_kernel(const float* __restrict__ part, int rows, int64_t cols, int d, E* __restrict__ dgain, E* __restrict__ dbias) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, share = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (c < cols) {
#pragma unroll 4
        for (int p = share; p < rows; p += 16) s += part[p * cols + c];
    }
    sums[share][lane] = s;
    __syncthreads();
    if (share != 0 || c >= cols) return;
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += sums[w][lane];
    Elem<E>::store(c < d ? dgain + c : dbias + (c - d), s);
}

}  // namespace moc
