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
constexpr int kRouteGroups = 256;         // most workgroups of a routing launch

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

struct RouteArgs {
    int T, E, k, chunk, groups;      // tokens of a workgroup, workgroups
    bool renorm;
    const uint8_t* valid;
    int32_t* ids;
    float* weights;
    int32_t *counts, *order;
    float *loss, *coef;
    // by workgroup: copies of every expert, tokens with a slot, and the sum of p over the tokens
    int32_t* hist;                   // [groups, E + 1]
    float* psum;                     // [groups, E]
};

// Places of a workgroup's copies, and the loss (workgroup 0).  `base` (LDS, E words) and `mask` (8 E words).
__device__ __forceinline__ void route_order(const RouteArgs& a, int group, int* base, uint32_t* mask, int* total) {
    const int tid = threadIdx.x;
    // copies of every expert in all workgroups, and in those before this one
    for (int e = tid; e < a.E; e += 256) {
        int all = 0, before = 0;
        for (int g = 0; g < a.groups; ++g) {
            const int n = a.hist[g * (a.E + 1) + e];
            all += n;
            before += g < group ? n : 0;
        }
        total[e] = all;
        base[e] = before;
    }
    __syncthreads();
    int A = 0;
    for (int e = 0; e < a.E; ++e) A += total[e];
    for (int e = tid; e < a.E; e += 256) {
        int first = 0;
        for (int f = 0; f < e; ++f) first += total[f];
        base[e] += first;
    }
    if (group == 0) {
        int N = 0;
        for (int g = 0; g < a.groups; ++g) N += a.hist[g * (a.E + 1) + a.E];
        const double scale = A > 0 ? (double)a.E / ((double)A * (double)N) : 0.0;
        double* part = reinterpret_cast<double*>(mask);      // 8 E words hold E doubles
        for (int e = tid; e < a.E; e += 256) {
            double p = 0.0;
            for (int g = 0; g < a.groups; ++g) p += (double)a.psum[g * a.E + e];
            a.counts[e] = total[e];
            a.coef[e] = (float)(scale * total[e]);
            part[e] = A > 0 ? scale * total[e] * p : 0.0;
        }
        __syncthreads();
        if (tid == 0) {
            double s = 0.0;
            for (int e = 0; e < a.E; ++e) s += part[e];
            a.loss[0] = (float)s;
        }
        __syncthreads();
    }
    // 256 tokens at a time: a bit per token and expert gives every copy the number of those before it
    const int t1 = (int)min((int64_t)a.T, (int64_t)(group + 1) * a.chunk);
    for (int t0 = group * a.chunk; t0 < t1; t0 += 256) {
        for (int i = tid; i < 8 * a.E; i += 256) mask[i] = 0;
        __syncthreads();
        const int t = t0 + tid;
        if (t < t1)
            for (int j = 0; j < a.k; ++j) {
                const int e = a.ids[(int64_t)t * a.k + j];
                if (e >= 0) atomicOr(&mask[e * 8 + (tid >> 5)], 1u << (tid & 31));
            }
        __syncthreads();
        if (t < t1)
            for (int j = 0; j < a.k; ++j) {
                const int e = a.ids[(int64_t)t * a.k + j];
                if (e < 0) continue;
                int at = base[e] + __popc(mask[e * 8 + (tid >> 5)] & ((1u << (tid & 31)) - 1));
                for (int w = 0; w < (tid >> 5); ++w) at += __popc(mask[e * 8 + w]);
                a.order[at] = t * a.k + j;
            }
        __syncthreads();
        for (int e = tid; e < a.E; e += 256) {
            int n = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) n += __popc(mask[e * 8 + w]);
            base[e] += n;
        }
        __syncthreads();
    }
    for (int64_t i = (int64_t)A + group * 256 + tid; i < (int64_t)a.T * a.k; i += (int64_t)a.groups * 256) a.order[i] = -1;
}

constexpr int route_order_lds(int E) { return (1 + 8 + 1) * E * 4; }

static __global__ __launch_bounds__(256) void route_order_kernel(RouteArgs a) {
    extern __shared__ __align__(16) uint32_t route_smem[];
    uint32_t* mask = route_smem;
    int* base = reinterpret_cast<int*>(mask + 8 * a.E);
    route_order(a, blockIdx.x, base, mask, base + a.E);
}

// LDS: route_order's, and before that the sums of four wavefronts and the histogram (E + 1 words).
constexpr int route_rows_lds(int E) {
    const int rows = (4 * E + E + 1) * 4, order = route_order_lds(E);
    return rows > order ? rows : order;
}
template <class E, int L, bool VEC> __global__ __launch_bounds__(256) void route_rows_kernel(const E* __restrict__ logits, RouteArgs a) {
    extern __shared__ __align__(16) uint32_t route_smem[];
    float* sums = reinterpret_cast<float*>(route_smem);              // [4, E]
    int* hist = reinterpret_cast<int*>(route_smem) + 4 * a.E;        // [E + 1]
    constexpr int TOKENS = 256 / L;
    const int lane = threadIdx.x % L, slot = threadIdx.x / L, e0 = lane * kRoutePer, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i <= a.E; i += 256) hist[i] = 0;
    __syncthreads();
    float acc[kRoutePer];
#pragma unroll
    for (int i = 0; i < kRoutePer; ++i) acc[i] = 0.0f;
    const int group = blockIdx.x, t1 = (int)min((int64_t)a.T, (int64_t)(group + 1) * a.chunk);
    for (int t0 = group * a.chunk; t0 < t1; t0 += TOKENS) {
        const int t = t0 + slot;
        if (t >= t1) continue;      // (a token's lanes leave together)
        float l[kRoutePer];
        route_logits<E, VEC>(logits + (int64_t)t * a.E, e0, a.E, l);
        const bool in = !a.valid || a.valid[t] != 0;
        // keys: larger logits are larger, a NaN is below everything
        uint32_t key[kRoutePer];
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) key[i] = l[i] == l[i] ? float_key(l[i]) : 0u;
        const uint32_t floor_key = float_key(-INFINITY);
        float top = 0.0f, chosen = 0.0f;
        int32_t* ids = a.ids + (int64_t)t * a.k;
        float* weights = a.weights + (int64_t)t * a.k;
        float ex[kRoutePer];
        float all = 0.0f;
        bool used = in;
        for (int j = 0; j < a.k; ++j) {
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
                for (int i = 0; i < kRoutePer; ++i) ex[i] = live ? (e0 + i < a.E ? expf(l[i] - top) : 0.0f) : 0.0f, s += ex[i];
                all = token_reduce<L>(s, OpSum());
                if (live && lane == 0) atomicAdd(&hist[a.E], 1);
            }
            const float x = live ? expf(key_float(row) - top) : 0.0f;
            chosen += x;
            if (lane == 0) {
                ids[j] = live ? e : -1;
                weights[j] = x;
                if (live) atomicAdd(&hist[e], 1);
            }
#pragma unroll
            for (int i = 0; i < kRoutePer; ++i)
                if (e0 + i == e) key[i] = 0;
        }
        const float den = used ? 1.0f / all : 0.0f;
        if (lane == 0) {
            const float by = a.renorm ? chosen : all;
            for (int j = 0; j < a.k; ++j) weights[j] = used ? weights[j] / by : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) acc[i] += ex[i] * den;
    }
    // the wavefront's tokens, then its lanes in LDS
#pragma unroll
    for (int i = 0; i < kRoutePer; ++i) {
        float v = acc[i];
#pragma unroll
        for (int o = L; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
        if ((threadIdx.x & 63) < L && e0 + i < a.E) sums[wave * a.E + e0 + i] = v;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += 256) a.psum[group * a.E + e] = (sums[e] + sums[a.E + e]) + (sums[2 * a.E + e] + sums[3 * a.E + e]);
    for (int e = threadIdx.x; e <= a.E; e += 256) a.hist[group * (a.E + 1) + e] = hist[e];
    if (a.groups > 1) return;
    __syncthreads();      // the workgroup's own ids, sums and histogram are in memory; its LDS is free
    uint32_t* mask = route_smem;
    int* base = reinterpret_cast<int*>(mask + 8 * a.E);
    route_order(a, 0, base, mask, base + a.E);
}

// Gradient of the logits.  A token without a slot gets zeros, whatever its logits are.  dlogits may be logits: a lane writes what it alone read.
template <class E, int L, bool VEC>
__global__ __launch_bounds__(256) void route_bwd_kernel(int T, int experts, int k, bool renorm, const E* logits, const int32_t* __restrict__ ids,
                                                        const float* __restrict__ coef, const float* __restrict__ dweights, const float* __restrict__ dloss,
                                                        E* dlogits) {
    const int64_t t = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    const int e0 = threadIdx.x % L * kRoutePer;
    if (t >= T) return;
    float out[kRoutePer];
#pragma unroll
    for (int i = 0; i < kRoutePer; ++i) out[i] = 0.0f;
    if (ids[t * k] >= 0) {
        float l[kRoutePer], ex[kRoutePer], dw[kRoutePer];
        bool chosen[kRoutePer];
        route_logits<E, VEC>(logits + t * experts, e0, experts, l);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) top = fmaxf(top, l[i]), dw[i] = 0.0f, chosen[i] = false;
        top = token_reduce<L>(top, OpMax());
        for (int j = 0; j < k; ++j) {
            const int e = ids[t * k + j];
            const float w = dweights ? dweights[t * k + j] : 0.0f;
#pragma unroll
            for (int i = 0; i < kRoutePer; ++i)
                if (e == e0 + i) dw[i] = w, chosen[i] = true;
        }
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
