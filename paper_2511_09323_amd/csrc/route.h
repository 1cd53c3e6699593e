// The softmax router before the expert entry points: the k experts of every token with their weights, the copies of the tokens in
// expert order, and the balance loss with its gradient.
//
// For a token's logits l: its slots hold the k largest, ties to the lower expert; p = softmax(l); a slot's weight is p, or p over
// the sum of the chosen.  With c_e the copies that go to expert e, A = sum c and N the tokens that have any:
//     loss = E sum_e (c_e / A) (1 / N) sum_t p_te,      coef_e = dloss/dp_te = E c_e / (A N), the same for every token,
//     dl_e = s_e (w_e dw_e) - b_e sum_j w_j dw_j + dloss p_e (coef_e - sum_f p_f coef_f),
// where s_e says whether e was chosen, and b is p, or the weights where they are renormalised.  Everything is fp32; the sums over
// tokens are fp32 inside a workgroup and fp64 across them, in a fixed order, and the counts are whole numbers, so that a call
// gives the same bits every time.
//
// L lanes hold a token's logits, 8 each.  Routing is two launches (one, if a single workgroup does): slots and a histogram by
// workgroup, then, with the histograms of the workgroups before it, every copy's place.  Both are bound by launch and latency up to
// some ten thousand tokens.
#pragma once
#include "common.h"
#include "misc_kernels.h"

namespace moc {

constexpr int kRoutePer = 8;              // logits of a lane
constexpr int kMaxRouteExperts = 256;     // 32 lanes
constexpr int kMaxRouteSlots = 16;
constexpr int kRouteGroups = 256;         // most workgroups of a routing launch (the places' histograms are read by all of them)

// Reductions over the L lanes of a token (L = 1 .. 32, aligned), for all of them; every step's partner holds another part of them.
template <int L, class T, class Op> __device__ __forceinline__ T token_reduce(T v, const Op& op) {
    static_assert(sizeof(T) == 4, "a register");
    auto move = [](T x, auto ctrl) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, false));
    };
    if (L >= 2) v = op(v, move(v, std::integral_constant<int, 0xB1>{}));       // quad_perm [1,0,3,2]
    if (L >= 4) v = op(v, move(v, std::integral_constant<int, 0x4E>{}));       // quad_perm [2,3,0,1]
    if (L >= 8) v = op(v, move(v, std::integral_constant<int, 0x141>{}));      // row_half_mirror
    if (L >= 16) v = op(v, move(v, std::integral_constant<int, 0x140>{}));     // row_mirror
    if (L >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
        const uint32_t a = r[0], b = r[1];      // (a bit cast of a vector's element takes its first one)
        v = op(__builtin_bit_cast(T, a), __builtin_bit_cast(T, b));
    }
    return v;
}
struct OpSum { template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a + b; } };
struct OpMax { template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a > b ? a : b; } };
struct OpMin { template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a < b ? a : b; } };

// The 8 logits from expert e0 on; experts past the last are -inf.  VEC: rows are whole 16-byte pieces.
template <class E, bool VEC> __device__ __forceinline__ void route_logits(const E* row, int e0, int experts, float* l) {
    if (VEC) {
#pragma unroll
        for (int p = 0; p < kRoutePer; p += Vec16<E>::N) {
            if (e0 + p < experts) Vec16<E>::unpack(*reinterpret_cast<const u32x4_t*>(row + e0 + p), l + p);
            else
#pragma unroll
                for (int i = 0; i < Vec16<E>::N; ++i) l[p + i] = -INFINITY;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) l[i] = e0 + i < experts ? Elem<E>::load(row + e0 + i) : -INFINITY;
    }
}

// Slots of a token are spread over its lanes: slot j is in lane j % L, register j / L.
template <int L> constexpr int route_regs() { return L == 1 ? kRoutePer : (kMaxRouteSlots + L - 1) / L; }
// f(register, lane of the token, slot) for the k slots in order; the register is a constant.
template <int L, class F> __device__ __forceinline__ void route_slots(int k, const F& f) {
#pragma unroll
    for (int r = 0; r < route_regs<L>(); ++r) {
        if (r * L >= k) break;
        for (int l = 0; l < L && r * L + l < k; ++l) f(r, l, r * L + l);
    }
}

struct RouteArgs {
    int T, E, k, chunk, groups;      // tokens of a workgroup, workgroups
    bool renorm;
    const uint8_t* valid;
    int32_t* ids;
    float* weights;
    int32_t *counts, *order;
    float *loss, *coef;
    // by workgroup: copies of every expert, then tokens with a slot; and the sum of p over the tokens
    int32_t* hist;                   // [groups, E + 1]
    float* psum;                     // [groups, E]
};

// Threads share out `groups` rows of values for E experts: thread tid takes expert tid % width of the rows part, part + parts, ...
struct RouteShare {
    int e, part, parts, width;
    __device__ __forceinline__ RouteShare(int E) {
        const int bits = 32 - __clz((E - 1) | 1);           // 2^bits >= E
        width = 1 << bits;
        e = threadIdx.x & (width - 1);
        part = threadIdx.x >> bits;
        parts = blockDim.x >> bits;
    }
};

// The loss, its derivative and the counts, by the first wavefront, from every expert's copies, the tokens with a slot (count[E]) and the
// sums of p: `parts` rows of `width` sums.
template <class F> __device__ __forceinline__ void route_loss(const RouteArgs& a, const int* count, const F* psum, int parts, int width) {
    const int tid = threadIdx.x;
    if (tid >= 64) return;
    int A = 0;
    for (int e = tid; e < a.E; e += 64) A += count[e];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) A += __shfl_xor(A, o, 64);
    const double scale = A > 0 ? (double)a.E / ((double)A * (double)count[a.E]) : 0.0;
    double loss = 0.0;
    for (int e = tid; e < a.E; e += 64) {
        double p = 0.0;
        for (int q = 0; q < parts; ++q) p += (double)psum[q * width + e];
        if (A > 0) loss += scale * count[e] * p;
        a.counts[e] = count[e];
        a.coef[e] = (float)(scale * count[e]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) loss += __shfl_xor(loss, o, 64);
    if (tid == 0) a.loss[0] = (float)loss;
}

// The places of the copies of tokens t0 .. t0 + n - 1 (n <= 256), whose experts are in `ids` (of copy tid + THREADS * i): a bit per token and expert gives
// every copy the number of those before it.  base[e] (LDS): the place of expert e's first one, moved on behind its last.  `mask`, `place`: LDS, 8 E words each;
// mask is zero, and again after the call.
constexpr int route_copies(int threads) { return 256 * kMaxRouteSlots / threads; }
template <int THREADS> __device__ __forceinline__ void route_places(const RouteArgs& a, int t0, int n, const int* ids, int* base, uint32_t* mask, int* place) {
    const int tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < route_copies(THREADS); ++i) {
        const int c = tid + THREADS * i, t = c / a.k;
        if (c < n * a.k && ids[i] >= 0) atomicOr(&mask[ids[i] * 8 + (t >> 5)], 1u << (t & 31));
    }
    __syncthreads();
    for (int i = tid; i < 8 * a.E; i += THREADS) {
        int at = base[i >> 3];
        for (int w = i & ~7; w < i; ++w) at += __popc(mask[w]);
        place[i] = at;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < route_copies(THREADS); ++i) {
        const int c = tid + THREADS * i, t = c / a.k;
        if (c >= n * a.k || ids[i] < 0) continue;
        const int at = ids[i] * 8 + (t >> 5);
        a.order[place[at] + __popc(mask[at] & ((1u << (t & 31)) - 1))] = t0 * a.k + c;
    }
    for (int e = tid; e < a.E; e += THREADS) base[e] = place[e * 8 + 7] + __popc(mask[e * 8 + 7]);
    __syncthreads();
    for (int i = tid; i < 8 * a.E; i += THREADS) mask[i] = 0;
    __syncthreads();
}
template <int THREADS> __device__ __forceinline__ void route_ids(const RouteArgs& a, int t0, int n, int* ids) {
#pragma unroll
    for (int i = 0; i < route_copies(THREADS); ++i) {
        const int c = threadIdx.x + THREADS * i;
        ids[i] = c < n * a.k ? a.ids[(int64_t)t0 * a.k + c] : -1;
    }
}
// base[e] += the copies of the experts before e, for up to 256 experts whose copies are in all[]; the result is their sum over all experts.  `waves`: LDS, 4 words.
__device__ __forceinline__ int route_bases(int experts, const int* all, int* base, int* waves) {
    const int tid = threadIdx.x;
    int upto = 0, n = 0;
    if (tid < 256) {
        n = tid < experts ? all[tid] : 0;
        upto = wave_inclusive_sum(n);
        if ((tid & 63) == 63) waves[tid >> 6] = upto;
    }
    __syncthreads();
    if (tid < experts) {
        for (int w = 0; w < (tid >> 6); ++w) upto += waves[w];
        base[tid] += upto - n;
    }
    __syncthreads();
    return waves[0] + waves[1] + waves[2] + waves[3];
}

// Second launch.  A workgroup places its own copies; the last workgroup does the loss.
constexpr int kRouteOrderThreads = 1024;
static __global__ __launch_bounds__(kRouteOrderThreads) void route_order_kernel(RouteArgs a) {
    constexpr int THREADS = kRouteOrderThreads;
    __shared__ int all[kMaxRouteExperts + 1], base[kMaxRouteExperts], waves[4];
    __shared__ __align__(16) uint32_t mem[2 * THREADS > 16 * kMaxRouteExperts ? 2 * THREADS : 16 * kMaxRouteExperts];
    const int tid = threadIdx.x, group = blockIdx.x;
    const RouteShare sh(a.E);
    if (group == a.groups) {
        double* psum = reinterpret_cast<double*>(mem);
        for (int i = tid; i <= a.E; i += THREADS) all[i] = 0;
        __syncthreads();
        double p = 0.0;
        if (sh.e < a.E) {
            int n = 0;
#pragma unroll 4
            for (int g = sh.part; g < a.groups; g += sh.parts) {
                n += a.hist[g * (a.E + 1) + sh.e];
                p += (double)a.psum[g * a.E + sh.e];
            }
            atomicAdd(&all[sh.e], n);
        }
        psum[tid] = p;
        for (int g = tid; g < a.groups; g += THREADS) atomicAdd(&all[a.E], a.hist[g * (a.E + 1) + a.E]);
        __syncthreads();
        route_loss(a, all, psum, sh.parts, sh.width);
        return;
    }
    const int t0 = group * a.chunk, t1 = (int)min((int64_t)a.T, (int64_t)t0 + a.chunk);
    int ids[route_copies(THREADS)];
    route_ids<THREADS>(a, t0, min(256, t1 - t0), ids);
    // copies of every expert in all workgroups, and in those before this one
    int n = 0, before = 0;
    if (sh.e < a.E) {
#pragma unroll 8
        for (int g = sh.part; g < a.groups; g += sh.parts) {
            const int h = a.hist[g * (a.E + 1) + sh.e];
            n += h;
            before += g < group ? h : 0;
        }
    }
    for (int i = tid; i < a.E; i += THREADS) base[i] = all[i] = 0;
    for (int i = tid; i < 8 * a.E; i += THREADS) mem[i] = 0;
    __syncthreads();
    if (sh.e < a.E) {
        atomicAdd(&all[sh.e], n);
        atomicAdd(&base[sh.e], before);
    }
    __syncthreads();
    const int A = route_bases(a.E, all, base, waves);
    for (int t = t0; t < t1; t += 256) {
        if (t > t0) route_ids<THREADS>(a, t, min(256, t1 - t), ids);
        route_places<THREADS>(a, t, min(256, t1 - t), ids, base, mem, reinterpret_cast<int*>(mem) + 8 * a.E);
    }
    for (int64_t i = (int64_t)A + group * THREADS + tid; i < (int64_t)a.T * a.k; i += (int64_t)a.groups * THREADS) a.order[i] = -1;
}

// First launch, and the only one where a workgroup holds all tokens (a.groups = 1).  LDS: the wavefronts' sums of p, the histogram (E + 1 words), and for a single
// workgroup the places.
constexpr int route_threads(int L) { return L >= 4 ? 1024 : 256 * L; }
constexpr int route_rows_words(int E, int threads, bool one) { return (threads / 64) * E + E + 1 + (one ? 17 * E + 4 : 0); }
template <class E, int L, bool VEC> __global__ __launch_bounds__(route_threads(L)) void route_rows_kernel(const E* __restrict__ logits, RouteArgs a) {
    extern __shared__ __align__(16) uint32_t route_smem[];
    constexpr int THREADS = route_threads(L), WAVES = THREADS / 64, TOKENS = THREADS / L, REGS = route_regs<L>();
    float* sums = reinterpret_cast<float*>(route_smem);                  // [WAVES, E]
    int* hist = reinterpret_cast<int*>(route_smem) + WAVES * a.E;        // [E + 1]
    const int lane = threadIdx.x % L, slot = threadIdx.x / L, e0 = lane * kRoutePer, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i <= a.E; i += THREADS) hist[i] = 0;
    __syncthreads();
    float acc[kRoutePer];
#pragma unroll
    for (int i = 0; i < kRoutePer; ++i) acc[i] = 0.0f;
    const int group = blockIdx.x, t1 = (int)min((int64_t)a.T, (int64_t)(group + 1) * a.chunk);
    for (int t0 = group * a.chunk; t0 < t1; t0 += TOKENS) {
        const int t = t0 + slot;
        if (t >= t1) continue;      // (a token's lanes leave together)
        float l[kRoutePer], ex[kRoutePer];
        route_logits<E, VEC>(logits + (int64_t)t * a.E, e0, a.E, l);
        bool used = !a.valid || a.valid[t] != 0;
        // keys: larger logits are larger, a NaN is below everything
        uint32_t key[kRoutePer];
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) key[i] = l[i] == l[i] ? float_key(l[i]) : 0u;
        const uint32_t floor_key = float_key(-INFINITY);
        float top = 0.0f, chosen = 0.0f, all = 1.0f, mine_x[REGS];
        int mine_e[REGS];
        route_slots<L>(a.k, [&](int r, int holder, int j) {
            uint32_t best = 0;
            int at = 0;
#pragma unroll
            for (int i = 0; i < kRoutePer; ++i)
                if (key[i] > best) best = key[i], at = i;
            const uint32_t row = token_reduce<L>(best, OpMax());
            const int e = token_reduce<L>(best == row ? e0 + at : INT32_MAX, OpMin());
            const bool live = used && row > floor_key;
            if (j == 0) {
                used = live;
                top = key_float(row);
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < kRoutePer; ++i) ex[i] = live && e0 + i < a.E ? expf(l[i] - top) : 0.0f, s += ex[i];
                all = token_reduce<L>(s, OpSum());
            }
            const float x = live ? expf(key_float(row) - top) : 0.0f;
            chosen += x;
            if (lane == holder) mine_e[r] = live ? e : -1, mine_x[r] = x;
#pragma unroll
            for (int i = 0; i < kRoutePer; ++i)
                if (e0 + i == e) key[i] = 0;
        });
        const float by = used ? (a.renorm ? chosen : all) : 1.0f, den = used ? 1.0f / all : 0.0f;
#pragma unroll
        for (int r = 0; r < REGS; ++r) {
            const int j = r * L + lane;
            if (j >= a.k) continue;
            a.ids[(int64_t)t * a.k + j] = mine_e[r];
            a.weights[(int64_t)t * a.k + j] = mine_x[r] / by;
            if (mine_e[r] >= 0) atomicAdd(&hist[mine_e[r]], 1);
        }
        if (used && lane == 0) atomicAdd(&hist[a.E], 1);
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) acc[i] += ex[i] * den;
    }
    // the wavefront's tokens, then the wavefronts in LDS
#pragma unroll
    for (int i = 0; i < kRoutePer; ++i) {
        float v = acc[i];
#pragma unroll
        for (int o = L; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
        if ((threadIdx.x & 63) < L && e0 + i < a.E) sums[wave * a.E + e0 + i] = v;
    }
    if (a.groups == 1) {
        uint32_t* mask = route_smem + WAVES * a.E + a.E + 1;
        int *place = reinterpret_cast<int*>(mask) + 8 * a.E, *base = place + 8 * a.E, *waves = base + a.E;
        for (int i = threadIdx.x; i < 8 * a.E; i += THREADS) mask[i] = 0;
        for (int i = threadIdx.x; i < a.E; i += THREADS) base[i] = 0;
        __syncthreads();      // (the workgroup's own ids are in memory, too)
        route_loss(a, hist, sums, WAVES, a.E);
        int ids[route_copies(THREADS)];
        route_ids<THREADS>(a, 0, a.T, ids);
        const int A = route_bases(a.E, hist, base, waves);
        route_places<THREADS>(a, 0, a.T, ids, base, mask, place);
        for (int i = A + threadIdx.x; i < a.T * a.k; i += THREADS) a.order[i] = -1;
        return;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += THREADS) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += sums[w * a.E + e];
        a.psum[group * a.E + e] = v;
    }
    for (int e = threadIdx.x; e <= a.E; e += THREADS) a.hist[group * (a.E + 1) + e] = hist[e];
}

// Gradient of the logits.  A token without a slot gets zeros, whatever its logits are.  dlogits may be logits: a lane writes what it alone read.
template <class E, int L, bool VEC>
__global__ __launch_bounds__(256) void route_bwd_kernel(int T, int experts, int k, bool renorm, const E* logits, const int32_t* __restrict__ ids,
                                                        const float* __restrict__ coef, const float* __restrict__ dweights, const float* __restrict__ dloss,
                                                        E* dlogits) {
    const int64_t t = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    const int lane = threadIdx.x % L, e0 = lane * kRoutePer;
    if (t >= T) return;
    float out[kRoutePer];
#pragma unroll
    for (int i = 0; i < kRoutePer; ++i) out[i] = 0.0f;
    if (ids[t * k] >= 0) {
        float l[kRoutePer], ex[kRoutePer], dw[kRoutePer], mine_w[route_regs<L>()];
        int mine_e[route_regs<L>()];
        bool chosen[kRoutePer];
#pragma unroll
        for (int r = 0; r < route_regs<L>(); ++r) {
            const int j = r * L + lane;
            mine_e[r] = j < k ? ids[t * k + j] : -1;
            mine_w[r] = j < k && dweights ? dweights[t * k + j] : 0.0f;
        }
        route_logits<E, VEC>(logits + t * experts, e0, experts, l);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) top = fmaxf(top, l[i]), dw[i] = 0.0f, chosen[i] = false;
        top = token_reduce<L>(top, OpMax());
        route_slots<L>(k, [&](int r, int holder, int) {
            const int from = (threadIdx.x & 63) - lane + holder;
            const int e = L == 1 ? mine_e[r] : __shfl(mine_e[r], from, 64);
            const float w = L == 1 ? mine_w[r] : __shfl(mine_w[r], from, 64);
#pragma unroll
            for (int i = 0; i < kRoutePer; ++i)
                if (e == e0 + i) dw[i] = w, chosen[i] = true;
        });
        const float scale = dloss ? dloss[0] : 0.0f;
        float c[kRoutePer];
        float all = 0.0f, part = 0.0f, wdw = 0.0f, pc = 0.0f;
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) {
            const bool real = e0 + i < experts;
            ex[i] = real ? expf(l[i] - top) : 0.0f;
            c[i] = real ? coef[e0 + i] : 0.0f;
            all += ex[i];
            part += chosen[i] ? ex[i] : 0.0f;
            wdw += chosen[i] ? ex[i] * dw[i] : 0.0f;
            pc += ex[i] * c[i];
        }
        all = token_reduce<L>(all, OpSum());
        part = token_reduce<L>(part, OpSum());
        wdw = token_reduce<L>(wdw, OpSum());
        pc = token_reduce<L>(pc, OpSum());
        const float by = 1.0f / (renorm ? part : all), pn = 1.0f / all;
        wdw *= by;
        pc *= pn;
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) {
            const float p = ex[i] * pn, w = chosen[i] ? ex[i] * by : 0.0f;
            out[i] = (renorm ? w * (dw[i] - wdw) : w * dw[i] - p * wdw) + scale * (p * (c[i] - pc));
        }
    }
    E* row = dlogits + t * experts;
    if (VEC) {
#pragma unroll
        for (int p = 0; p < kRoutePer; p += Vec16<E>::N)
            if (e0 + p < experts) *reinterpret_cast<u32x4_t*>(row + e0 + p) = Vec16<E>::pack(out + p);
    } else {
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i)
            if (e0 + i < experts) Elem<E>::store(row + e0 + i, out[i]);
    }
}

}  // namespace moc
