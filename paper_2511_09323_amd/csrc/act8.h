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

// The set from token t on.
inline moc_act8_set act8_from(const moc_act8_set& s, int64_t t, int d, int F, int K) {
    return moc_act8_set{s.xq + t * d, s.xe + t * act8_blocks(d), s.sel + t * act8_blocks(F), s.gq + t * K, s.ge + t * act8_blocks(K), s.uq + t * K, s.ue + t * act8_blocks(K)};
}

// The byte e of a block whose largest magnitude has these bits (an infinity or NaN anywhere gives at least 0x7F800000).
__device__ __forceinline__ uint32_t act8_exponent(uint32_t amax_bits) {
    const uint32_t e = amax_bits >> 23;
    return e < 8 ? 0u : e;
}
// What values are multiplied with before rounding: 2^(133 - e), 0 where the block is zeros or NaN.
__device__ __forceinline__ float act8_scale(uint32_t e) { return e == 0 || e == 255 ? 0.0f : __uint_as_float((260u - e) << 23); }
// What q is multiplied with: 2^(e - 133), 0, or NaN.  (e >= 8, so the power is 2^-125 at least.)
__device__ __forceinline__ float act8_step(uint32_t e) {
    return e == 255 ? __uint_as_float(0x7FC00000u) : e < 8 ? 0.0f : __uint_as_float((e - 6u) << 23);
}

// Largest of 4 neighbouring lanes
template <int CTRL> __device__ __forceinline__ uint32_t dpp_max_u32(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xF, 0xF, false);
    return o > v ? o : v;
}
__device__ __forceinline__ uint32_t quad_max_u32(uint32_t v) { return dpp_max_u32<0x4E>(dpp_max_u32<0xB1>(v)); }      // quad_perm [1,0,3,2], [2,3,0,1]

// Rows are worked on in pieces of 8 values, 4 lanes a block.  Rows of K values start anywhere: pieces are loaded and stored at the element's alignment, which the
// memory pipeline takes at no measurable cost.  The last piece of a row, where it is not whole, is loaded as the row's last 8 values and shifted: loaded
// value by value, the last pieces of the 1B layer's gate and up values took 4 us of the 29 that saving it took.
template <class E> struct Act8Piece;
template <> struct Act8Piece<float> {
    uint32_t raw[8];
    __device__ __forceinline__ uint32_t top() const {      // bits of the largest magnitude
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = max(m, raw[k] & 0x7FFFFFFFu);
        return m;
    }
    __device__ __forceinline__ float value(int k) const { return __uint_as_float(raw[k]); }
    __device__ __forceinline__ void set(int k, float v) { raw[k] = __float_as_uint(v); }
    __device__ __forceinline__ void shift(int by) {      // values `by` .. 7 to the front, zeros behind them (all zeros from 8 on)
#pragma unroll
        for (int o = 1; o < 8; o <<= 1)
#pragma unroll
            for (int k = 0; k < 8; ++k) raw[k] = by & o ? (k + o < 8 ? raw[k + o & 7] : 0u) : raw[k];
#pragma unroll
        for (int k = 0; k < 8; ++k) raw[k] = by >= 8 ? 0u : raw[k];
    }
};
template <> struct Act8Piece<bf16_t> {
    uint32_t raw[4];
    typedef uint16_t Pair __attribute__((ext_vector_type(2)));
    __device__ __forceinline__ uint32_t top() const {
        Pair m = {0, 0};
#pragma unroll
        for (int k = 0; k < 4; ++k) m = __builtin_elementwise_max(m, __builtin_bit_cast(Pair, raw[k] & 0x7FFF7FFFu));
        const uint32_t lo = m.x, hi = m.y;
        return (lo > hi ? lo : hi) << 16;
    }
    __device__ __forceinline__ float value(int k) const { return __uint_as_float(k & 1 ? raw[k / 2] & 0xFFFF0000u : raw[k / 2] << 16); }
    __device__ __forceinline__ void set(int k, float v) {      // (in pairs; v has bf16's bits)
        const uint32_t b = __float_as_uint(v);
        raw[k / 2] = k & 1 ? (raw[k / 2] & 0xFFFFu) | (b & 0xFFFF0000u) : b >> 16;
    }
    __device__ __forceinline__ void shift(int by) {
#pragma unroll
        for (int k = 0; k < 4; ++k) raw[k] = by & 1 ? __builtin_amdgcn_alignbit(k < 3 ? raw[k + 1 & 3] : 0u, raw[k], 16) : raw[k];
#pragma unroll
        for (int o = 1; o < 4; o <<= 1)
#pragma unroll
            for (int k = 0; k < 4; ++k) raw[k] = by & 2 * o ? (k + o < 4 ? raw[k + o & 3] : 0u) : raw[k];
#pragma unroll
        for (int k = 0; k < 4; ++k) raw[k] = by >= 8 ? 0u : raw[k];
    }
};
// The 8 values at value i of a row of n (n and the row the same in a wavefront): the load, and, apart from it, what makes the last ones of a row the lane's own.
template <class E> __device__ __forceinline__ void act8_read(Act8Piece<E>& p, const E* row, int n, int i) {
    if (n >= 8) {
        __builtin_memcpy(p.raw, row + min(i, n - 8), sizeof(p.raw));
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) p.set(k, i + k < n ? Elem<E>::load(row + i + k) : 0.0f);
    }
}
template <class E> __device__ __forceinline__ void act8_settle(Act8Piece<E>& p, int n, int i) {
    if (n >= 8 && n - (i & ~511) < 512) p.shift(max(0, i - (n - 8)));      // (the wavefront's 512 values are not all there)
}
__device__ __forceinline__ uint64_t act8_read_bytes(const int8_t* row, int n, int i) {
    uint64_t w = 0;
    if (n >= 8) {
        __builtin_memcpy(&w, row + min(i, n - 8), 8);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) w |= i + k < n ? (uint64_t)(uint8_t)row[i + k] << (8 * k) : 0u;
    }
    return w;
}
__device__ __forceinline__ u32x2_t act8_settle_bytes(uint64_t w, int n, int i) {
    if (n >= 8 && n - (i & ~511) < 512) w >>= 8 * min(7, max(0, i - (n - 8)));      // (nobody looks at values past the row's end)
    return u32x2_t{(uint32_t)w, (uint32_t)(w >> 32)};
}
// The first `left` of 8 values, or all of them.
template <class E> __device__ __forceinline__ void act8_write(const Act8Piece<E>& p, E* v, int left) {
    if (left >= 8) {
        __builtin_memcpy(v, p.raw, sizeof(p.raw));
    } else {
#pragma unroll
        for (int k = 0; k < 7; ++k)
            if (k < left) Elem<E>::store(v + k, p.value(k));
    }
}
__device__ __forceinline__ void act8_write_bytes(u32x2_t w, int8_t* q, int left) {
    if (left >= 8) {
        __builtin_memcpy(q, &w, 8);
    } else if (left > 0) {
        const uint32_t rest = left & 4 ? w[1] : w[0], last = left & 2 ? rest >> 16 : rest;
        if (left & 4) __builtin_memcpy(q, &w, 4);
        q += left & 4;
        if (left & 2) __builtin_memcpy(q, &rest, 2);
        if (left & 1) q[left & 2] = (int8_t)last;
    }
}
// Rounding: held to +-127 (which rounds to itself, so that it may come first), 1.5 2^23 added: the sum's last byte is the nearest whole number, halves to even,
// in two's complement, and its one rounding is that of v 2^(133 - e).  Restoring: a byte plus 128 is converted without a sign
// (one instruction a byte) and 128 taken off again (before the product: 128 steps may be past the largest number).
template <class E> __device__ __forceinline__ u32x2_t act8_pack(const Act8Piece<E>& p, uint32_t& e) {
    e = act8_exponent(quad_max_u32(p.top()));
    const float scale = act8_scale(e);
    uint32_t b[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) b[k] = __float_as_uint(__builtin_amdgcn_fmed3f(p.value(k) * scale, -127.0f, 127.0f) + 12582912.0f);
    const uint32_t keep = e == 255 ? 0u : 0xFFFFFFFFu;
    u32x2_t w;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __builtin_amdgcn_perm(b[4 * h + 1], b[4 * h], 0x0C0C0400u), hi = __builtin_amdgcn_perm(b[4 * h + 3], b[4 * h + 2], 0x0C0C0400u);
        w[h] = __builtin_amdgcn_perm(hi, lo, 0x05040100u) & keep;
    }
    return w;
}
template <class E> __device__ __forceinline__ void act8_unpack(u32x2_t w, uint32_t e, Act8Piece<E>& p) {
    const float step = act8_step(e);
    w ^= 0x80808080u;
#pragma unroll
    for (int k = 0; k < 8; ++k) p.set(k, ((float)((w[k / 4] >> (k % 4 * 8)) & 0xFFu) - 128.0f) * step);
}
// A token's x, gate and up values in steps of 64 pieces, a piece a lane; a step lies in one of the three, so that all but a lane's offset stays in scalar registers.
template <class V> struct Act8Step {
    V* v;
    int8_t* q;
    uint8_t* e;
    int n, first;      // values of the row, first piece of the step
    __device__ __forceinline__ Act8Step(int s, const moc_act8_set& set, int64_t t, int d, int K, V* x, V* g, V* u) {
        const int xs = act8_steps(d), ks = act8_steps(K);
        n = d;
        v = x, q = set.xq, e = set.xe;
        if (s >= xs) {
            s -= xs;
            n = K;
            v = g, q = set.gq, e = set.ge;
            if (s >= ks) s -= ks, v = u, q = set.uq, e = set.ue;
        }
        v += t * n, q += t * n, e += t * act8_blocks(n);
        first = s * 64;
    }
    __device__ __forceinline__ int piece(int lane) const { return first + lane; }
    __device__ __forceinline__ int left(int lane) const { return n - piece(lane) * 8; }      // values from here to the row's end
    __device__ __forceinline__ bool in(int lane) const { return piece(lane) < 4 * act8_blocks(n); }      // (blocks of 4 lanes stay together)
    static __host__ __device__ __forceinline__ int act8_steps(int n) { return (act8_blocks(n) + 15) / 16; }
    static __device__ __forceinline__ int total(int d, int K) { return act8_steps(d) + 2 * act8_steps(K); }
};

// Four or one wavefronts (WAVES) take a token.  Their number: a workgroup's four take four tokens, or one.  The eight chiplets, which take workgroups in turn, get an
// eighth of the workgroups each, one behind the other: rows of K values and of block bytes end inside cache lines, and neighbours on one chiplet share its
// cache, where on two they each move the line (the 1B layer's set, just written, restored in 26.4 us without, 23.6 with, in the form that the kernel had then).
template <int WAVES> __device__ __forceinline__ int64_t act8_token(int wave) {
    const unsigned chip = blockIdx.x & 7, each = gridDim.x >> 3, over = gridDim.x & 7;
    const int64_t group = (int64_t)chip * each + min(chip, over) + (blockIdx.x >> 3);
    return WAVES == 4 ? group : group * 4 + wave;
}
// What a token's wavefronts wait for each other with: a barrier, or for one only that the compiler keeps the order that LDS keeps.
template <int WAVES> __device__ __forceinline__ void act8_sync() {
    if (WAVES > 1) {
        __syncthreads();
    } else {
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// Saving, four wavefronts a token.  The steps are shared out over them and asked for together (8 steps, 1024 values of idx), so that a token of the usual sizes is one
// trip to memory; then the mask, which is put together in LDS, and the pieces.  Entries of idx outside [0, F) are ignored.
// 8192 tokens, d 2048, F 5461, K 683, bf16: 113 MB from memory in 24.4 us, one such launch after the other (4.6 TB/s of the 5.2 that a large copy reaches); 27.5 in turn
// with the restoring launch (4.1).
constexpr int kAct8Steps = 8, kAct8Idx = 4;
template <class E>
__global__ __launch_bounds__(256) void act8_save_kernel(const E* __restrict__ x, const int32_t* __restrict__ idx, const E* __restrict__ g, const E* __restrict__ u, int d, int F,
                                                        int K, moc_act8_set set) {
    extern __shared__ uint32_t act8_words[];
    typedef Act8Step<const E> Step;
    constexpr int AHEAD = kAct8Steps / 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t t = act8_token<4>(wave);
    const int words = act8_blocks(F), steps = Step::total(d, K);
    const int32_t* row = idx + t * K;
    int ch[kAct8Idx];
#pragma unroll
    for (int i = 0; i < kAct8Idx; ++i) ch[i] = tid + 256 * i < K ? row[tid + 256 * i] : -1;
    Act8Piece<E> piece[AHEAD];
    const auto read = [&](int s0) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int s = s0 + i * 4 + wave;
            if (s >= steps) break;
            const Step at(s, set, t, d, K, x, g, u);
            act8_read<E>(piece[i], at.v, at.n, at.piece(lane) * 8);
        }
    };
    read(0);
    for (int i = tid; i < words; i += 256) act8_words[i] = 0;
    __syncthreads();
    const auto mark = [&](int j) {
        if (j >= 0 && j < F) atomicOr(&act8_words[j >> 5], 1u << (j & 31));
    };
#pragma unroll
    for (int i = 0; i < kAct8Idx; ++i) mark(ch[i]);
    for (int s = tid + 256 * kAct8Idx; s < K; s += 256) mark(row[s]);
    __syncthreads();
    for (int i = tid; i < words; i += 256) set.sel[t * words + i] = act8_words[i];
    for (int s0 = 0; s0 < steps; s0 += kAct8Steps) {
        if (s0 > 0) read(s0);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int s = s0 + i * 4 + wave;
            if (s >= steps) break;
            const Step at(s, set, t, d, K, x, g, u);
            uint32_t e;
            act8_settle<E>(piece[i], at.n, at.piece(lane) * 8);
            const u32x2_t w = act8_pack<E>(piece[i], e);
            act8_write_bytes(w, at.q + at.piece(lane) * 8, at.left(lane));
            if (at.in(lane) && (lane & 3) == 0) at.e[at.piece(lane) / 4] = (uint8_t)e;
        }
    }
}

// Restoring, shared out in the same way over one or four wavefronts a token, the channels first.  They go to LDS in the order of the set bits, 32 for each of the token's lanes at a time, and from there to
// memory; a row with fewer than K bits (not one that was saved) leaves the rest of its indices at -1, bits past the K-th are dropped.
// 8192 tokens, d 2048, F 5461, K 683, bf16: 113 MB in 28 us from memory (4.0 TB/s), as in a backward pass long after its forward; in 21 where the set was just written
// and is read from the last-level cache.
template <class E, int WAVES>
__global__ __launch_bounds__(256) void act8_load_kernel(moc_act8_set set, int T, int d, int F, int K, E* __restrict__ x, int32_t* __restrict__ idx, E* __restrict__ g,
                                                        E* __restrict__ u) {
    __shared__ int sums[2][4];
    __shared__ uint16_t places[256 * 32];
    typedef Act8Step<E> Step;
    constexpr int AHEAD = kAct8Steps / WAVES, LANES = 64 * WAVES, WORDS = 4 / WAVES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = WAVES == 4 ? wave : 0, tid = threadIdx.x & (LANES - 1);
    const int64_t t = act8_token<WAVES>(wave);
    if (t >= T) return;
    const int words = act8_blocks(F), steps = Step::total(d, K);
    uint16_t* place = places + (WAVES == 4 ? 0 : wave * 64 * 32);
    const uint32_t* sel = set.sel + t * words;
    int32_t* row = idx + t * K;
    uint32_t head[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) head[i] = i * LANES + tid < words ? sel[i * LANES + tid] : 0;
    uint64_t w[AHEAD];
    uint32_t e[AHEAD];
    const auto read = [&](int s0) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int s = s0 + i * WAVES + mine;
            if (s >= steps) break;
            const Step at(s, set, t, d, K, x, g, u);
            w[i] = act8_read_bytes(at.q, at.n, at.piece(lane) * 8);
            e[i] = at.e[min(at.piece(lane) / 4, act8_blocks(at.n) - 1)];
        }
    };
    read(0);
    int base = 0;
    const auto channels = [&](int w0, uint32_t bits, int turn) {
        if (w0 + tid == words - 1 && (F & 31)) bits &= (1u << (F & 31)) - 1;
        const int own = __popc(bits), upto = wave_inclusive_sum(own);
        int at = upto - own, n = __builtin_amdgcn_readlane(upto, 63);
        if (WAVES > 1) {
            if (lane == 63) sums[turn][wave] = upto;
            __syncthreads();      // (and the channels before these are out of LDS)
            for (int i = 0; i < wave; ++i) at += sums[turn][i];
            n = sums[turn][0] + sums[turn][1] + sums[turn][2] + sums[turn][3];
        }
        for (; bits != 0; bits &= bits - 1) place[at++] = (uint16_t)(tid * 32 + __ffs(bits) - 1);
        act8_sync<WAVES>();
        for (int s = tid; s < min(n, K - base); s += LANES) row[base + s] = w0 * 32 + place[s];
        if (WAVES == 1) act8_sync<WAVES>();
        base += n;
    };
#pragma unroll
    for (int i = 0; i < WORDS; ++i)
        if (i * LANES < words) channels(i * LANES, head[i], i & 1);
    for (int w0 = WORDS * LANES, turn = WORDS & 1; w0 < words; w0 += LANES, turn ^= 1) channels(w0, w0 + tid < words ? sel[w0 + tid] : 0, turn);
    for (int s = base + tid; s < K; s += LANES) row[s] = -1;
    for (int s0 = 0; s0 < steps; s0 += kAct8Steps) {
        if (s0 > 0) read(s0);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int s = s0 + i * WAVES + mine;
            if (s >= steps) break;
            const Step at(s, set, t, d, K, x, g, u);
            Act8Piece<E> piece;
            act8_unpack<E>(act8_settle_bytes(w[i], at.n, at.piece(lane) * 8), e[i], piece);
            act8_write<E>(piece, at.v + at.piece(lane) * 8, at.left(lane));
        }
    }
}

// The backward's pointwise step (bwd_expand_kernel) from the 8-bit set, and x restored beside it.  A wavefront takes kAct8Span channels of
// one dense row: the mask bits give it its channels and, by the bits before them, their places in the compact rows; z', dg and du are
// assembled in LDS, zero everywhere else, and streamed out.  No wavefront waits for another.  The first `unpack_groups` workgroups restore x.
// Rounded to E: dz', by the product that made it, and z', dg, du, which the matrix cores take in E; so the gradients are bit for bit those of
// moc_ffn_bwd from the restored set where it, too, takes this step in a launch of its own; where it does not, so does the backward from 8 bits (dz' in fp32 would add 90 MB to what that product and this launch each move at the first of the sizes below).
// Bound by memory: 8192 x 5461, K 683, x 8192 x 2048: 439 MB in 82 us, 5.3 TB/s, the rate of a large copy; 16384 x 2048, K 384, x 16384 x 768: 328 MB in 70 us.
constexpr int kAct8Span = 1024;
template <class E>
__global__ __launch_bounds__(256) void bwd_expand_act8_kernel(moc_act8_set set, const E* __restrict__ dzd, RowGroups groups, int rows, int T, int d, int F, int K, int64_t ldf,
                                                              int unpack_groups, E* __restrict__ x, E* __restrict__ zd, E* __restrict__ dgd, E* __restrict__ dud) {
    constexpr int PER16 = 16 / sizeof(E), SLOTS = kAct8Span / 64, BATCH = 4;
    __shared__ __align__(16) E span[4][3][kAct8Span];
    if ((int)blockIdx.x < unpack_groups) {
        // (a row a wavefront)
        for (int64_t t = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); t < T; t += unpack_groups * 4)
#pragma unroll 4
            for (int i = (threadIdx.x & 63) * 8; i < d; i += 64 * 8) {
                Act8Piece<E> piece;
                act8_unpack<E>(act8_settle_bytes(act8_read_bytes(set.xq + t * d, d, i), d, i), set.xe[t * act8_blocks(d) + i / kAct8Block], piece);
                act8_write<E>(piece, x + t * d + i, d - i);
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
    for (int q0 = 0; q0 < SLOTS; q0 += BATCH) {
        if (q0 * 64 >= n) break;
        // What BATCH slots read is asked for before any is worked on; lanes past the last slot read that one's, and nothing is converted yet: in a branch that
        // would be waited for.
        int gv[BATCH], uv[BATCH], ch[BATCH];
        uint32_t gx[BATCH], ux[BATCH];
        E dz[BATCH];
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            if ((q0 + q) * 64 >= n) break;
            const int s = min((q0 + q) * 64 + lane, n - 1), block = (before + s) / kAct8Block;
            ch[q] = (q0 + q) * 64 + lane < n ? channel[q0 + q] : 0;
            gv[q] = gq[s];
            uv[q] = uq[s];
            gx[q] = ge[block];
            ux[q] = ue[block];
            dz[q] = dzrow[ch[q]];
        }
#pragma unroll
        for (int q = 0; q < BATCH; ++q) {
            if ((q0 + q) * 64 + lane >= n) continue;
            float z, dg, du;
            moc_bwd_pointwise((float)gv[q] * act8_step(gx[q]), (float)uv[q] * act8_step(ux[q]), Elem<E>::load(&dz[q]), z, dg, du);
            Elem<E>::store(&span[wave][0][ch[q]], z);
            Elem<E>::store(&span[wave][1][ch[q]], dg);
            Elem<E>::store(&span[wave][2][ch[q]], du);
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
