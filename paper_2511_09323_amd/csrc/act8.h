// The stored set of a layer in 8 bits, and the backward's pointwise step on it.
//
// 32 consecutive values of a row share one byte e, the exponent field (fp32) of the largest magnitude among them; a value is
// q 2^(e - 133) with q = v 2^(133 - e) rounded to the nearest whole number, halves to even, and held to +-127 (a magnitude just below
// the next power of two rounds to 128).  e < 8 is stored as 0 and stands for zeros, so that no power of two here is subnormal; 255,
// a block with an infinity or a NaN, stands for NaN.  Powers of two keep everything but that one rounding exact: a restored value has
// at most seven significant bits, is the same in fp32 and bf16, and saving it again gives the same bytes.
// The Top-K mask is one bit per channel, channel j in bit j % 32 of word j / 32: F / 8 bytes against 4 K of the indices.
#pragma once
#include "../../include/moc.h"
#include "common.h"
#include "misc_kernels.h"

namespace moc {

constexpr int kAct8Block = 32;
inline __host__ __device__ int act8_blocks(int n) { return (n + kAct8Block - 1) / kAct8Block; }

// The byte e of a block whose largest magnitude has these bits (an infinity or NaN anywhere gives at least 0x7F800000).
__device__ __forceinline__ uint32_t act8_exponent(uint32_t amax_bits) {
    const uint32_t e = amax_bits >> 23;
    return e < 8 ? 0u : e;
}
// What values are multiplied with before rounding: 2^(133 - e), 0 where the block is zeros or NaN.
__device__ __forceinline__ float act8_scale(uint32_t e) { return e == 0 || e == 255 ? 0.0f : __uint_as_float((260u - e) << 23); }
__device__ __forceinline__ int act8_round(float v, float scale, uint32_t e) {
    const int q = cvt_i32(fminf(fmaxf(rintf(v * scale), -127.0f), 127.0f));
    return e == 255 ? 0 : q;
}
// What q is multiplied with: 2^(e - 133), 0, or NaN.  (e >= 8, so the power is 2^-125 at least.)
__device__ __forceinline__ float act8_step(uint32_t e) {
    return e == 255 ? __uint_as_float(0x7FC00000u) : e < 8 ? 0.0f : __uint_as_float((e - 6u) << 23);
}

template <int CTRL> __device__ __forceinline__ uint32_t dpp_max_u32(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xF, 0xF, false);
    return o > v ? o : v;
}
// Largest of 4 neighbouring lanes; of the 32 lanes of a half wavefront.
__device__ __forceinline__ uint32_t quad_max_u32(uint32_t v) { return dpp_max_u32<0x4E>(dpp_max_u32<0xB1>(v)); }      // quad_perm [1,0,3,2], [2,3,0,1]
__device__ __forceinline__ uint32_t half_max_u32(uint32_t v) {
    v = dpp_max_u32<0x121>(dpp_max_u32<0x122>(dpp_max_u32<0x124>(dpp_max_u32<0x128>(v))));      // row_ror 8, 4, 2, 1
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return r[0] > r[1] ? r[0] : r[1];
}

// One row of n values, by the 256 threads of a workgroup.  VEC: n is a multiple of 8, rows start on 16 bytes (q: on 8); a thread
// packs 8 values and 4 threads a block.  Otherwise a thread packs one value and half a wavefront a block.
template <class E, bool VEC> __device__ __forceinline__ void act8_pack_row(const E* __restrict__ v, int n, int8_t* __restrict__ q, uint8_t* __restrict__ e) {
    if (VEC) {
        for (int i = threadIdx.x * 8; i < act8_blocks(n) * kAct8Block; i += 256 * 8) {      // (whole blocks of 4 threads)
            float f[8];
#pragma unroll
            for (int p = 0; p < 8; p += Vec16<E>::N) {
                const u32x4_t raw = i < n ? *reinterpret_cast<const u32x4_t*>(v + i + p) : u32x4_t{0, 0, 0, 0};
                Vec16<E>::unpack(raw, f + p);
            }
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) m = max(m, __float_as_uint(f[k]) & 0x7FFFFFFFu);
            const uint32_t ex = act8_exponent(quad_max_u32(m));
            const float scale = act8_scale(ex);
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k / 4] |= (uint32_t)(act8_round(f[k], scale, ex) & 0xFF) << (k % 4 * 8);
            if (i < n) *reinterpret_cast<u32x2_t*>(q + i) = u32x2_t{w[0], w[1]};
            if ((threadIdx.x & 3) == 0) e[i / kAct8Block] = (uint8_t)ex;
        }
    } else {
        for (int i = threadIdx.x; i < act8_blocks(n) * kAct8Block; i += 256) {
            const float f = i < n ? Elem<E>::load(v + i) : 0.0f;
            const uint32_t ex = act8_exponent(half_max_u32(__float_as_uint(f) & 0x7FFFFFFFu));
            const int r = act8_round(f, act8_scale(ex), ex);
            if (i < n) q[i] = (int8_t)r;
            if ((threadIdx.x & 31) == 0) e[i / kAct8Block] = (uint8_t)ex;
        }
    }
}
template <class E, bool VEC> __device__ __forceinline__ void act8_unpack_row(const int8_t* __restrict__ q, const uint8_t* __restrict__ e, int n, E* __restrict__ v) {
    if (VEC) {
        for (int i = threadIdx.x * 8; i < n; i += 256 * 8) {
            const u32x2_t w = *reinterpret_cast<const u32x2_t*>(q + i);
            const float step = act8_step(e[i / kAct8Block]);
            float f[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = (float)(int8_t)(w[k / 4] >> (k % 4 * 8)) * step;
#pragma unroll
            for (int p = 0; p < 8; p += Vec16<E>::N) *reinterpret_cast<u32x4_t*>(v + i + p) = Vec16<E>::pack(f + p);
        }
    } else {
        for (int i = threadIdx.x; i < n; i += 256) Elem<E>::store(v + i, (float)q[i] * act8_step(e[i / kAct8Block]));
    }
}

// One workgroup per token: x, then the gate and up values, then the mask (words in LDS).  Entries of idx outside [0, F) are ignored.
template <class E, bool VEC>
__global__ __launch_bounds__(256) void act8_save_kernel(const E* __restrict__ x, const int32_t* __restrict__ idx, const E* __restrict__ g, const E* __restrict__ u, int d, int F,
                                                        int K, moc_act8_set set) {
    extern __shared__ uint32_t act8_words[];
    const int64_t t = blockIdx.x;
    const int words = act8_blocks(F), kb = act8_blocks(K);
    for (int i = threadIdx.x; i < words; i += 256) act8_words[i] = 0;
    act8_pack_row<E, VEC>(x + t * d, d, set.xq + t * d, set.xe + t * act8_blocks(d));
    act8_pack_row<E, false>(g + t * K, K, set.gq + t * K, set.ge + t * kb);
    act8_pack_row<E, false>(u + t * K, K, set.uq + t * K, set.ue + t * kb);
    __syncthreads();
    for (int s = threadIdx.x; s < K; s += 256) {
        const int j = idx[t * K + s];
        if (j >= 0 && j < F) atomicOr(&act8_words[j >> 5], 1u << (j & 31));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < words; i += 256) set.sel[t * words + i] = act8_words[i];
}

// The inverse.  Channels are written in the order of the set bits; a row with fewer than K bits (not one that was saved) leaves the rest of its
// indices at -1, bits past the K-th are dropped.
template <class E, bool VEC>
__global__ __launch_bounds__(256) void act8_load_kernel(moc_act8_set set, int d, int F, int K, E* __restrict__ x, int32_t* __restrict__ idx, E* __restrict__ g, E* __restrict__ u) {
    __shared__ int sums[4];
    const int64_t t = blockIdx.x;
    const int words = act8_blocks(F), kb = act8_blocks(K), wave = threadIdx.x >> 6;
    act8_unpack_row<E, VEC>(set.xq + t * d, set.xe + t * act8_blocks(d), d, x + t * d);
    act8_unpack_row<E, false>(set.gq + t * K, set.ge + t * kb, K, g + t * K);
    act8_unpack_row<E, false>(set.uq + t * K, set.ue + t * kb, K, u + t * K);
    int base = 0;
    for (int w0 = 0; w0 < words; w0 += 256) {
        const int w = w0 + threadIdx.x;
        uint32_t bits = w < words ? set.sel[t * words + w] : 0;
        if (w == words - 1 && (F & 31)) bits &= (1u << (F & 31)) - 1;
        const int mine = __popc(bits), upto = wave_inclusive_sum(mine);
        if ((threadIdx.x & 63) == 63) sums[wave] = upto;
        __syncthreads();
        int at = base + upto - mine;
        for (int i = 0; i < wave; ++i) at += sums[i];
        base += sums[0] + sums[1] + sums[2] + sums[3];
        for (; bits != 0 && at < K; bits &= bits - 1) idx[t * K + at++] = w * 32 + __ffs(bits) - 1;
        __syncthreads();
    }
    for (int s = base + threadIdx.x; s < K; s += 256) idx[t * K + s] = -1;
}

// The backward's pointwise step (bwd_expand_kernel) from the 8-bit set, and x restored beside it.  A wavefront takes kAct8Span channels of
// one dense row: the mask bits give it its channels and, by the bits before them, their places in the compact rows; z', dg and du are
// assembled in LDS, zero everywhere else, and streamed out.  No wavefront waits for another.  The first `unpack_groups` workgroups restore x.
constexpr int kAct8Span = 1024;
template <class E>
__global__ __launch_bounds__(256) void bwd_expand_act8_kernel(moc_act8_set set, const E* __restrict__ dzd, RowGroups groups, int rows, int T, int d, int F, int K, int64_t ldf,
                                                              int unpack_groups, E* __restrict__ x, E* __restrict__ zd, E* __restrict__ dgd, E* __restrict__ dud) {
    constexpr int PER16 = 16 / sizeof(E);
    __shared__ __align__(16) E span[4][3][kAct8Span];
    __shared__ uint16_t place[4][kAct8Span];
    if ((int)blockIdx.x < unpack_groups) {
        for (int64_t t = blockIdx.x; t < T; t += unpack_groups) {
            if (d % 8 == 0) act8_unpack_row<E, true>(set.xq + t * d, set.xe + t * act8_blocks(d), d, x + t * d);
            else act8_unpack_row<E, false>(set.xq + t * d, set.xe + t * act8_blocks(d), d, x + t * d);
        }
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int spans = (int)((ldf + kAct8Span - 1) / kAct8Span);
    const int64_t task = (int64_t)(blockIdx.x - unpack_groups) * 4 + wave;
    const int64_t row = task / spans;
    if (row >= rows) return;
    const int c0 = (int)(task - row * spans) * kAct8Span;
    const int width = (int)min((int64_t)kAct8Span, ldf - c0);       // a multiple of 8
    const int64_t t = row_token(groups, (int)row);
    u32x4_t* mine = reinterpret_cast<u32x4_t*>(span[wave][0]);
    for (int i = lane; i < 3 * kAct8Span / PER16; i += 64) mine[i] = u32x4_t{0, 0, 0, 0};
    if (t >= 0) {
        const int words = act8_blocks(F), kb = act8_blocks(K), w0 = c0 / 32;
        const uint32_t* sel = set.sel + t * words;
        int before = 0;
        for (int w = lane; w < w0; w += 64) before += __popc(sel[w]);
        // half a word a lane
        const int w = w0 + lane / 2;
        uint32_t bits = w < words ? sel[w] : 0;
        if (w == words - 1 && (F & 31)) bits &= (1u << (F & 31)) - 1;
        bits = lane & 1 ? bits >> 16 : bits & 0xFFFFu;
        const int own = __popc(bits), upto = wave_inclusive_sum(own);
        before = __builtin_amdgcn_readlane(wave_inclusive_sum(before), 63);
        const int n = min(__builtin_amdgcn_readlane(upto, 63), K - before);      // (negative: the row has more bits than slots)
        for (int at = upto - own; bits != 0; bits &= bits - 1) place[wave][at++] = (uint16_t)(lane * 16 + __ffs(bits) - 1);
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");      // (LDS keeps a wavefront's order; this keeps the compiler's)
        __builtin_amdgcn_wave_barrier();
        for (int s = lane; s < n; s += 64) {
            const int j = place[wave][s], k = before + s;
            const float gv = (float)set.gq[t * K + k] * act8_step(set.ge[t * kb + k / kAct8Block]);
            const float uv = (float)set.uq[t * K + k] * act8_step(set.ue[t * kb + k / kAct8Block]);
            const float dz = Elem<E>::load(dzd + t * ldf + c0 + j);
            float z, dg, du;
            moc_bwd_pointwise(gv, uv, dz, z, dg, du);
            Elem<E>::store(&span[wave][0][j], z);
            Elem<E>::store(&span[wave][1][j], dg);
            Elem<E>::store(&span[wave][2][j], du);
        }
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    const int64_t at = row * ldf + c0;
    for (int i = lane; i < width / PER16; i += 64) {
        reinterpret_cast<u32x4_t*>(zd + at)[i] = mine[i];
        reinterpret_cast<u32x4_t*>(dgd + at)[i] = mine[kAct8Span / PER16 + i];
        reinterpret_cast<u32x4_t*>(dud + at)[i] = mine[2 * (kAct8Span / PER16) + i];
    }
}

}  // namespace moc
