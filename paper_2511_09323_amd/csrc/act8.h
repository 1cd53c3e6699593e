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

// A row is packed and unpacked by the 256 threads of a workgroup, in two ways.  Pieces: 8 values a thread, 4 threads a block; rows are
// whole pieces and start on 16 bytes (their q on 8).  Single values: a value a thread, half a wavefront a block.
template <class E> struct Act8Piece {
    static constexpr int R = 8 / Vec16<E>::N;
    u32x4_t raw[R];
    __device__ __forceinline__ void load(const E* v, bool in) {
#pragma unroll
        for (int p = 0; p < R; ++p) raw[p] = in ? reinterpret_cast<const u32x4_t*>(v)[p] : u32x4_t{0, 0, 0, 0};
    }
    __device__ __forceinline__ u32x2_t pack(uint32_t& e) const {
        float f[8];
#pragma unroll
        for (int p = 0; p < R; ++p) Vec16<E>::unpack(raw[p], f + p * Vec16<E>::N);
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = max(m, __float_as_uint(f[k]) & 0x7FFFFFFFu);
        e = act8_exponent(quad_max_u32(m));
        const float scale = act8_scale(e);
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k / 4] |= (uint32_t)(act8_round(f[k], scale, e) & 0xFF) << (k % 4 * 8);
        return u32x2_t{w[0], w[1]};
    }
};
template <class E> __device__ __forceinline__ void act8_unpack_piece(u32x2_t w, uint32_t e, E* v) {
    const float step = act8_step(e);
    float f[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = (float)(int8_t)(w[k / 4] >> (k % 4 * 8)) * step;
#pragma unroll
    for (int p = 0; p < 8; p += Vec16<E>::N) *reinterpret_cast<u32x4_t*>(v + p) = Vec16<E>::pack(f + p);
}
__device__ __forceinline__ int act8_pack_one(float f, uint32_t& e) {
    e = act8_exponent(half_max_u32(__float_as_uint(f) & 0x7FFFFFFFu));
    return act8_round(f, act8_scale(e), e);
}

// One workgroup per token.  A step takes 2048 values of x (256, where rows are not whole pieces) and 1024 slots: everything it reads is
// asked for before anything is worked on, so that a row of the usual sizes costs one trip to memory.  The mask is put together in LDS.
// Entries of idx outside [0, F) are ignored.
constexpr int kAct8Slots = 4;      // of a thread in a step
template <class E, bool VEC>
__global__ __launch_bounds__(256) void act8_save_kernel(const E* __restrict__ x, const int32_t* __restrict__ idx, const E* __restrict__ g, const E* __restrict__ u, int d, int F,
                                                        int K, moc_act8_set set) {
    extern __shared__ uint32_t act8_words[];
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, words = act8_blocks(F), db = act8_blocks(d), kb = act8_blocks(K);
    constexpr int XSTEP = VEC ? 2048 : 256, KSTEP = 256 * kAct8Slots;
    const int xend = db * kAct8Block, kend = kb * kAct8Block;      // whole blocks: their lanes stay together
    for (int i = tid; i < words; i += 256) act8_words[i] = 0;
    for (int x0 = 0, k0 = 0; x0 < d || k0 < K; x0 += XSTEP, k0 += KSTEP) {
        const int xi = x0 + tid * (VEC ? 8 : 1);
        Act8Piece<E> piece;
        float one = 0.0f, gv[kAct8Slots], uv[kAct8Slots];
        int ch[kAct8Slots];
        if (VEC) piece.load(x + t * d + xi, xi < d);
        else if (xi < d) one = Elem<E>::load(x + t * d + xi);
#pragma unroll
        for (int q = 0; q < kAct8Slots; ++q) {
            const int s = k0 + q * 256 + tid;
            ch[q] = s < K ? idx[t * K + s] : -1;
            gv[q] = s < K ? Elem<E>::load(g + t * K + s) : 0.0f;
            uv[q] = s < K ? Elem<E>::load(u + t * K + s) : 0.0f;
        }
        if (x0 == 0) __syncthreads();      // (the words are zero)
        if (xi < xend) {
            uint32_t e;
            if (VEC) {
                const u32x2_t w = piece.pack(e);
                if (xi < d) *reinterpret_cast<u32x2_t*>(set.xq + t * d + xi) = w;
            } else {
                const int w = act8_pack_one(one, e);
                if (xi < d) set.xq[t * d + xi] = (int8_t)w;
            }
            if (xi % kAct8Block == 0) set.xe[t * db + xi / kAct8Block] = (uint8_t)e;
        }
#pragma unroll
        for (int q = 0; q < kAct8Slots; ++q) {
            const int s = k0 + q * 256 + tid;
            if (s >= kend) continue;
            if (ch[q] >= 0 && ch[q] < F) atomicOr(&act8_words[ch[q] >> 5], 1u << (ch[q] & 31));
            uint32_t eg, eu;
            const int wg = act8_pack_one(gv[q], eg), wu = act8_pack_one(uv[q], eu);
            if (s < K) {
                set.gq[t * K + s] = (int8_t)wg;
                set.uq[t * K + s] = (int8_t)wu;
            }
            if (s % kAct8Block == 0) {
                set.ge[t * kb + s / kAct8Block] = (uint8_t)eg;
                set.ue[t * kb + s / kAct8Block] = (uint8_t)eu;
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < words; i += 256) set.sel[t * words + i] = act8_words[i];
}

// x of a row from its 8 bits
template <class E, bool VEC> __device__ __forceinline__ void act8_unpack_row(const int8_t* __restrict__ q, const uint8_t* __restrict__ e, int n, E* __restrict__ v) {
    if (VEC) {
        for (int i = threadIdx.x * 8; i < n; i += 256 * 8) act8_unpack_piece<E>(*reinterpret_cast<const u32x2_t*>(q + i), e[i / kAct8Block], v + i);
    } else {
        for (int i = threadIdx.x; i < n; i += 256) Elem<E>::store(v + i, (float)q[i] * act8_step(e[i / kAct8Block]));
    }
}

// The inverse, with the same steps.  Channels are written in the order of the set bits; a row with fewer than K bits (not one that was saved) leaves the
// rest of its indices at -1, bits past the K-th are dropped.
template <class E, bool VEC>
__global__ __launch_bounds__(256) void act8_load_kernel(moc_act8_set set, int d, int F, int K, E* __restrict__ x, int32_t* __restrict__ idx, E* __restrict__ g, E* __restrict__ u) {
    __shared__ int sums[2][4];
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, words = act8_blocks(F), db = act8_blocks(d), kb = act8_blocks(K), wave = tid >> 6;
    constexpr int XSTEP = VEC ? 2048 : 256, KSTEP = 256 * kAct8Slots;
    int base = 0, turn = 0;
    for (int x0 = 0, k0 = 0, w0 = 0; x0 < d || k0 < K || w0 < words; x0 += XSTEP, k0 += KSTEP, w0 += 256, turn ^= 1) {
        const int xi = x0 + tid * (VEC ? 8 : 1), w = w0 + tid;
        uint32_t bits = w < words ? set.sel[t * words + w] : 0;
        u32x2_t xw{0, 0};
        uint32_t xe = 0;
        float one = 0.0f, gv[kAct8Slots], uv[kAct8Slots];
        uint32_t ge[kAct8Slots], ue[kAct8Slots];
        if (xi < d) {
            if (VEC) xw = *reinterpret_cast<const u32x2_t*>(set.xq + t * d + xi);
            else one = (float)set.xq[t * d + xi];
            xe = set.xe[t * db + xi / kAct8Block];
        }
#pragma unroll
        for (int q = 0; q < kAct8Slots; ++q) {
            const int s = k0 + q * 256 + tid;
            gv[q] = s < K ? (float)set.gq[t * K + s] : 0.0f;
            uv[q] = s < K ? (float)set.uq[t * K + s] : 0.0f;
            ge[q] = s < K ? set.ge[t * kb + s / kAct8Block] : 0u;
            ue[q] = s < K ? set.ue[t * kb + s / kAct8Block] : 0u;
        }
        if (w0 < words) {
            if (w == words - 1 && (F & 31)) bits &= (1u << (F & 31)) - 1;
            const int mine = __popc(bits), upto = wave_inclusive_sum(mine);
            if ((tid & 63) == 63) sums[turn][wave] = upto;
            __syncthreads();
            int at = base + upto - mine;
            for (int i = 0; i < wave; ++i) at += sums[turn][i];
            base += sums[turn][0] + sums[turn][1] + sums[turn][2] + sums[turn][3];
            for (; bits != 0 && at < K; bits &= bits - 1) idx[t * K + at++] = w * 32 + __ffs(bits) - 1;
        }
        if (xi < d) {
            if (VEC) act8_unpack_piece<E>(xw, xe, x + t * d + xi);
            else Elem<E>::store(x + t * d + xi, one * act8_step(xe));
        }
#pragma unroll
        for (int q = 0; q < kAct8Slots; ++q) {
            const int s = k0 + q * 256 + tid;
            if (s >= K) continue;
            Elem<E>::store(g + t * K + s, gv[q] * act8_step(ge[q]));
            Elem<E>::store(u + t * K + s, uv[q] * act8_step(ue[q]));
        }
    }
    for (int s = base + tid; s < K; s += 256) idx[t * K + s] = -1;
}

// The backward's pointwise step (bwd_expand_kernel) from the 8-bit set, and x restored beside it.  A wavefront takes kAct8Span channels of
// one dense row: the mask bits give it its channels and, by the bits before them, their places in the compact rows; z', dg and du are
// assembled in LDS, zero everywhere else, and streamed out.  No wavefront waits for another.  The first `unpack_groups` workgroups restore x.
constexpr int kAct8Span = 1024;
template <class E>
__global__ __launch_bounds__(256) void bwd_expand_act8_kernel(moc_act8_set set, const E* __restrict__ dzd, RowGroups groups, int rows, int T, int d, int F, int K, int64_t ldf,
                                                              int unpack_groups, E* __restrict__ x, E* __restrict__ zd, E* __restrict__ dgd, E* __restrict__ dud) {
    constexpr int PER16 = 16 / sizeof(E), SLOTS = kAct8Span / 64, BATCH = 4;
    __shared__ __align__(16) E span[4][3][kAct8Span];
    if ((int)blockIdx.x < unpack_groups) {
        for (int64_t t = blockIdx.x; t < T; t += unpack_groups) {
            if (d % 8 == 0) act8_unpack_row<E, true>(set.xq + t * d, set.xe + t * act8_blocks(d), d, x + t * d);
            else act8_unpack_row<E, false>(set.xq + t * d, set.xe + t * act8_blocks(d), d, x + t * d);
        }
        return;
    }
    // (the wavefront's number is the same in all its lanes: what follows from it stays out of the vector registers)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned spans = (unsigned)(ldf + kAct8Span - 1) / kAct8Span, task = (blockIdx.x - unpack_groups) * 4u + wave;      // (ldf < 2^16, tasks < 2^32)
    const unsigned row = task / spans;
    if (row >= (unsigned)rows) return;
    const int c0 = (int)(task - row * spans) * kAct8Span;
    const int width = (int)min((int64_t)kAct8Span, ldf - c0);       // a multiple of 8
    const int64_t t = row_token(groups, (int)row);
    u32x4_t* mine = reinterpret_cast<u32x4_t*>(span[wave][0]);
    const auto ordered = [] {      // (LDS keeps a wavefront's order; this keeps the compiler's)
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    int channel[SLOTS], before = 0, n = 0;
    if (t >= 0) {
        const int words = act8_blocks(F), w0 = c0 / 32;
        const uint32_t* sel = set.sel + t * words;
        // half a word a lane
        const int w = w0 + lane / 2;
        uint32_t bits = w < words ? sel[w] : 0;
        for (int v = lane; v < w0; v += 64) before += __popc(sel[v]);
        if (w == words - 1 && (F & 31)) bits &= (1u << (F & 31)) - 1;
        bits = lane & 1 ? bits >> 16 : bits & 0xFFFFu;
        const int own = __popc(bits), upto = wave_inclusive_sum(own);
        before = __builtin_amdgcn_readlane(wave_inclusive_sum(before), 63);
        n = min(__builtin_amdgcn_readlane(upto, 63), K - before);      // (negative: the row has more bits than slots)
        // channels by place, through the LDS that the rows take next
        uint16_t* place = reinterpret_cast<uint16_t*>(mine);
        for (int at = upto - own; bits != 0; bits &= bits - 1) place[at++] = (uint16_t)(lane * 16 + __ffs(bits) - 1);
        ordered();
#pragma unroll
        for (int q = 0; q < SLOTS; ++q) {
            if (q * 64 >= n) break;
            channel[q] = place[q * 64 + lane];
        }
        ordered();
    }
    for (int i = lane; i < 3 * kAct8Span / PER16; i += 64) mine[i] = u32x4_t{0, 0, 0, 0};
    ordered();
    const int8_t *gq = set.gq + t * K + before, *uq = set.uq + t * K + before;
    const uint8_t *ge = set.ge + t * act8_blocks(K), *ue = set.ue + t * act8_blocks(K);
    const E* dzrow = dzd + t * ldf + c0;
#pragma unroll
    for (int q0 = 0; q0 < SLOTS; q0 += BATCH) {      // (what BATCH slots read is asked for before any is worked on)
        if (q0 * 64 >= n) break;
        float gv[BATCH], uv[BATCH], dz[BATCH];
        uint32_t gx[BATCH], ux[BATCH];
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            const int s = (q0 + q) * 64 + lane, block = (before + s) / kAct8Block;
            if (s < n) {
                gv[q] = (float)gq[s];
                uv[q] = (float)uq[s];
                gx[q] = ge[block];
                ux[q] = ue[block];
                dz[q] = Elem<E>::load(dzrow + channel[q0 + q]);
            }
        }
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            if ((q0 + q) * 64 + lane >= n) continue;
            const int j = channel[q0 + q];
            float z, dg, du;
            moc_bwd_pointwise(gv[q] * act8_step(gx[q]), uv[q] * act8_step(ux[q]), dz[q], z, dg, du);
            Elem<E>::store(&span[wave][0][j], z);
            Elem<E>::store(&span[wave][1][j], dg);
            Elem<E>::store(&span[wave][2][j], du);
        }
    }
    ordered();
    const int64_t at = (int64_t)row * ldf + c0;
    for (int i = lane; i < width / PER16; i += 64) {
        reinterpret_cast<u32x4_t*>(zd + at)[i] = mine[i];
        reinterpret_cast<u32x4_t*>(dgd + at)[i] = mine[kAct8Span / PER16 + i];
        reinterpret_cast<u32x4_t*>(dud + at)[i] = mine[2 * (kAct8Span / PER16) + i];
    }
}

}  // namespace moc
