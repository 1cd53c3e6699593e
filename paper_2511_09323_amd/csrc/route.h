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
// workgroup, then, with the histograms of the workgroups before it, every copy's place.  All are bound by launch and latency (a launch
// that does nothing takes 1.3 us, one round trip to memory 1 to 2): us for slots, places, gradient: 37 tokens, 8 experts 4.5 in one, 2.9; 16384, 8 experts 4.4, 5.3,
// 4.1; 32768, 64 experts, six slots 8.6, 6.4, 6.9 (8.4 MB of logits in and out).
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
// Sum over a wavefront's tokens, lane by lane of a token: every lane gets that of the lanes congruent to it modulo L.  (Register moves as in wave_reduce, stopped
// at L.)
template <int L> __device__ __forceinline__ float column_sum(float v) {
    {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (L <= 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (L <= 8) v += dpp_move<0x128>(v);      // row_ror 8, 4, 2, 1
    if (L <= 4) v += dpp_move<0x124>(v);
    if (L <= 2) v += dpp_move<0x122>(v);
    if (L <= 1) v += dpp_move<0x121>(v);
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
        // (every lane loads eight, the last one again and again past the end: a load in a branch of its own would be waited for before the next)
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) l[i] = Elem<E>::load(row + min(e0 + i, experts - 1));
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) l[i] = e0 + i < experts ? l[i] : -INFINITY;
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

// Choosing one expert after the other.  fp32: the largest key (common.h), then the lowest expert that has it.  bf16 leaves half of a key's bits free for the
// expert's number, inverted, so that one reduction finds both (about 25 instructions a slot instead of 60).  A NaN is below everything, an expert that
// was chosen, too.
template <class E> struct RouteKeys;
template <> struct RouteKeys<float> {
    uint32_t key[kRoutePer];
    __device__ __forceinline__ void set(int i, int, float l) { key[i] = l == l ? float_key(l) : 0u; }
    template <int L> __device__ __forceinline__ int take(int e0, float& value, bool& above) {      // the expert, its logit, whether that is above -inf
        uint32_t best = 0;
        int at = 0;
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i)
            if (key[i] > best) best = key[i], at = i;
        const uint32_t top = token_reduce<L>(best, OpMax());
        const int e = token_reduce<L>(best == top ? e0 + at : INT32_MAX, OpMin());
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) key[i] = e0 + i == e ? 0u : key[i];
        value = key_float(top);
        above = top > float_key(-INFINITY);
        return e;
    }
};
template <> struct RouteKeys<bf16_t> {
    uint32_t key[kRoutePer];
    __device__ __forceinline__ void set(int i, int e, float l) { key[i] = l == l ? (float_key(l) & 0xFFFF0000u) | (0xFFFFu - e) : 0u; }
    template <int L> __device__ __forceinline__ int take(int, float& value, bool& above) {
        uint32_t best = 0;
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) best = max(best, key[i]);
        const uint32_t top = token_reduce<L>(best, OpMax());
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) key[i] = key[i] == top ? 0u : key[i];
        const uint32_t h = top >> 16;
        value = __uint_as_float(h & 0x8000u ? (h & 0x7FFFu) << 16 : ~top & 0xFFFF0000u);
        above = h > (float_key(-INFINITY) >> 16);
        return (int)(0xFFFFu - (top & 0xFFFFu));
    }
};

struct RouteArgs {
    int T, E, k, chunk, groups;      // tokens of a workgroup, workgroups
    bool renorm;
    const uint8_t* valid;
    int32_t* ids;
    float* weights;
    int32_t *counts, *order;
    float *loss, *coef;
    // by workgroup (rows of route_pad(groups)): copies of every expert, then tokens with a slot; and the sum of p over the tokens
    int32_t* hist;                   // [E + 1][groups]
    float* psum;                     // [E][groups]
};

__device__ __forceinline__ int round_up_64(int n) { return (n + 63) & ~63; }

// Sums over the workgroups: an expert's numbers lie side by side ([expert][workgroup]), `lanes` neighbouring threads (2 .. 64) share them out in fours.
constexpr int kRouteOrderLog = 9, kRouteOrderThreads = 1 << kRouteOrderLog;
struct RouteShare {
    int lanes, e, at;
    __device__ __forceinline__ RouteShare(int E) {
        const int bits = 32 - __clz((E - 1) | 1), log = min(6, kRouteOrderLog - bits);      // 2^bits >= E
        lanes = 1 << log;
        e = threadIdx.x >> log;
        at = (threadIdx.x & (lanes - 1)) * 4;
    }
    template <class T> __device__ __forceinline__ T sum(T v) const {
        for (int o = 1; o < lanes; o <<= 1) v += __shfl_xor(v, o, 64);
        return v;
    }
};
inline __host__ __device__ int route_pad(int groups) { return (groups + 3) & ~3; }

// Running sums of up to 256 experts' copies (LDS), by every wavefront for itself: no barrier.
struct RouteScan {
    static constexpr int N = kMaxRouteExperts / 64;
    int before[N], total = 0;      // lane l: the copies of the experts before 64 c + l
    __device__ __forceinline__ RouteScan(const int* count, int experts) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int c = 0; c < N; ++c) {
            before[c] = 0;
            if (c * 64 >= experts) continue;
            const int n = c * 64 + lane < experts ? count[c * 64 + lane] : 0, upto = wave_inclusive_sum(n);
            before[c] = total + upto - n;
            total += __builtin_amdgcn_readlane(upto, 63);
        }
    }
    // Of expert e, all of a wavefront's in the same 64.
    __device__ __forceinline__ int operator()(int e) const {
        int v = 0;
#pragma unroll
        for (int c = 0; c < N; ++c)
            if (__builtin_amdgcn_readfirstlane(e >> 6) == c) v = __shfl(before[c], e & 63, 64);
        return v;
    }
};

// The loss, its derivative and the counts, by one wavefront, from every expert's copies, the tokens with a slot (count[E]) and the
// sums of p: `rows` rows of E.
template <class F> __device__ __forceinline__ void route_loss(const RouteArgs& a, const int* count, const F* psum, int rows) {
    const int tid = threadIdx.x & 63;
    const int A = RouteScan(count, a.E).total;
    const double scale = A > 0 ? (double)a.E / ((double)A * (double)count[a.E]) : 0.0;
    double loss = 0.0;
    for (int e = tid; e < a.E; e += 64) {
        double p = 0.0;
        for (int q = 0; q < rows; ++q) p += (double)psum[q * a.E + e];
        if (A > 0) loss += scale * count[e] * p;
        a.counts[e] = count[e];
        a.coef[e] = (float)(scale * count[e]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) loss += __shfl_xor(loss, o, 64);
    if (tid == 0) a.loss[0] = (float)loss;
}

// Places of copies: a bit per token (of 256) and expert gives every copy the number of those before it.  A thread holds the experts of copies tid + THREADS * i.
constexpr int route_copies(int threads) { return 256 * kMaxRouteSlots / threads; }
template <int THREADS> __device__ __forceinline__ void route_ids(const RouteArgs& a, int t0, int n, int* ids) {
#pragma unroll
    for (int i = 0; i < route_copies(THREADS); ++i) {
        const int c = threadIdx.x + THREADS * i;
        ids[i] = c < n * a.k ? a.ids[(int64_t)t0 * a.k + c] : -1;
    }
}
template <int THREADS> __device__ __forceinline__ void route_mark(const RouteArgs& a, const int* ids, uint32_t* mask) {
#pragma unroll
    for (int i = 0; i < route_copies(THREADS); ++i) {
        const int t = (threadIdx.x + THREADS * i) / a.k;
        if (ids[i] >= 0) atomicOr(&mask[ids[i] * 8 + (t >> 5)], 1u << (t & 31));
    }
}
// the copies of mask word i's expert in the words before it
__device__ __forceinline__ int route_before(const uint32_t* mask, int i) {
    int n = 0;
    for (int w = i & ~7; w < i; ++w) n += __popc(mask[w]);
    return n;
}

// Second launch.  A workgroup places its own copies, behind those of the workgroups before it.  The loss is the first one's: the last of
// many starts a few us after it, and the loss takes as long as the places (32768 tokens, 64 experts: 10.3 us with it last, 8.2 with it first; 6.5 with 512 threads a workgroup
// instead of 1024, of which 256 take longer to start, and 9.5 with 256).
static __global__ __launch_bounds__(kRouteOrderThreads) void route_order_kernel(RouteArgs a) {
    constexpr int THREADS = kRouteOrderThreads;
    __shared__ int all[kMaxRouteExperts + 1], base[kMaxRouteExperts];
    __shared__ __align__(16) uint32_t mem[16 * kMaxRouteExperts];
    const int tid = threadIdx.x, group = (int)blockIdx.x - 1, ld = route_pad(a.groups);
    const RouteShare sh(a.E);
    typedef int32_t Four __attribute__((ext_vector_type(4)));
    if (group < 0) {
        double* psum = reinterpret_cast<double*>(mem);
        int n = 0, tokens = 0;
        double p = 0.0;
        if (sh.e < a.E) {
#pragma unroll 4
            for (int g = sh.at; g < a.groups; g += 4 * sh.lanes) {
                const Four h = *reinterpret_cast<const Four*>(a.hist + sh.e * ld + g);
                const f32x4_t q = *reinterpret_cast<const f32x4_t*>(a.psum + sh.e * ld + g);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    n += g + i < a.groups ? h[i] : 0;
                    p += g + i < a.groups ? (double)q[i] : 0.0;
                }
            }
        }
        if (tid < a.groups) tokens = a.hist[a.E * ld + tid];      // (kRouteGroups <= THREADS)
        if (tid == 0) all[a.E] = 0;
        n = sh.sum(n);
        p = sh.sum(p);
        if (sh.e < a.E && sh.at == 0) all[sh.e] = n, psum[sh.e] = p;
        __syncthreads();
        if (tid < a.groups) atomicAdd(&all[a.E], tokens);
        __syncthreads();
        if (tid < 64) route_loss(a, all, psum, 1);
        return;
    }
    uint32_t* mask = mem;
    int* place = reinterpret_cast<int*>(mem) + 8 * a.E;
    const int t0 = group * a.chunk, t1 = (int)min((int64_t)a.T, (int64_t)t0 + a.chunk);
    int ids[route_copies(THREADS)];
    route_ids<THREADS>(a, t0, min(256, t1 - t0), ids);
    // copies of every expert in all workgroups, and in those before this one
    int n = 0, before = 0;
    if (sh.e < a.E) {
#pragma unroll 4
        for (int g = sh.at; g < a.groups; g += 4 * sh.lanes) {
            const Four h = *reinterpret_cast<const Four*>(a.hist + sh.e * ld + g);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                n += g + i < a.groups ? h[i] : 0;
                before += g + i < group ? h[i] : 0;
            }
        }
    }
    for (int i = tid; i < 8 * a.E; i += THREADS) mask[i] = 0;
    n = sh.sum(n);
    before = sh.sum(before);
    if (sh.e < a.E && sh.at == 0) all[sh.e] = n, base[sh.e] = before;
    __syncthreads();
    route_mark<THREADS>(a, ids, mask);
    __syncthreads();
    const RouteScan scan(all, a.E);
    for (int t = t0; t < t1; t += 256) {
        if (t > t0) {
            route_ids<THREADS>(a, t, min(256, t1 - t), ids);
            for (int i = tid; i < 8 * a.E; i += THREADS) mask[i] = 0;
            __syncthreads();
            route_mark<THREADS>(a, ids, mask);
            __syncthreads();
        }
        for (int i = tid; i < round_up_64(8 * a.E); i += THREADS) {      // (whole wavefronts)
            const int first = t == t0 ? scan(i >> 3) : 0;
            if (i < 8 * a.E) place[i] = base[i >> 3] + first + route_before(mask, i);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < route_copies(THREADS); ++i) {
            const int c = tid + THREADS * i, u = c / a.k;
            if (ids[i] < 0) continue;
            const int at = ids[i] * 8 + (u >> 5);
            a.order[place[at] + __popc(mask[at] & ((1u << (u & 31)) - 1))] = t * a.k + c;
        }
        if (t + 256 >= t1) break;
        for (int e = tid; e < a.E; e += THREADS) base[e] = place[e * 8 + 7] + __popc(mask[e * 8 + 7]);
        __syncthreads();
    }
    for (int64_t i = (int64_t)scan.total + group * THREADS + tid; i < (int64_t)a.T * a.k; i += (int64_t)a.groups * THREADS) a.order[i] = -1;
}

// First launch, and (ONE) the only one where one pass of one workgroup does: its copies' places come from the same bits, out of the registers that hold their
// experts.  LDS: the wavefronts' sums of p, the histogram (E + 1 words), and for a single workgroup the bits and the places.
constexpr int route_threads(int L) { return L >= 4 ? 1024 : 256 * L; }
constexpr int route_rows_words(int E, int threads, bool one) { return (threads / 64) * E + E + 1 + (one ? 16 * E : 0); }
template <class E, int L, bool VEC, bool ONE> __global__ __launch_bounds__(route_threads(L)) void route_rows_kernel(const E* __restrict__ logits, RouteArgs a) {
    extern __shared__ __align__(16) uint32_t route_smem[];
    constexpr int THREADS = route_threads(L), WAVES = THREADS / 64, TOKENS = THREADS / L, REGS = route_regs<L>();
    float* sums = reinterpret_cast<float*>(route_smem);                  // [WAVES, E]
    int* hist = reinterpret_cast<int*>(route_smem) + WAVES * a.E;        // [E + 1]
    const int lane = threadIdx.x % L, slot = threadIdx.x / L, e0 = lane * kRoutePer, wave = threadIdx.x >> 6;
    uint32_t* mask = route_smem + WAVES * a.E + a.E + 1;                  // [E, 8], ONE
    int* place = reinterpret_cast<int*>(mask) + 8 * a.E;
    for (int i = threadIdx.x; i < (ONE ? 9 * a.E + 1 : a.E + 1); i += THREADS) hist[i] = 0;      // (the mask follows)
    __syncthreads();
    int mine_e[REGS];
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
        RouteKeys<E> keys;
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) keys.set(i, e0 + i, l[i]);
        float top = 0.0f, chosen = 0.0f, all = 1.0f, mine_x[REGS];
        route_slots<L>(a.k, [&](int r, int holder, int j) {
            float logit;
            bool above;
            const int e = keys.template take<L>(e0, logit, above);
            const bool live = used && above;
            if (j == 0) {
                used = live;
                top = logit;
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < kRoutePer; ++i) ex[i] = live && e0 + i < a.E ? expf(l[i] - top) : 0.0f, s += ex[i];
                all = token_reduce<L>(s, OpSum());
            }
            const float x = live ? expf(logit - top) : 0.0f;
            chosen += x;
            if (lane == holder) mine_e[r] = live ? e : -1, mine_x[r] = x;
        });
        const float by = used ? (a.renorm ? chosen : all) : 1.0f, den = used ? 1.0f / all : 0.0f;
#pragma unroll
        for (int r = 0; r < REGS; ++r) {
            const int j = r * L + lane;
            if (j >= a.k) continue;
            a.ids[(int64_t)t * a.k + j] = mine_e[r];
            a.weights[(int64_t)t * a.k + j] = mine_e[r] < 0 ? 0.0f : mine_x[r] / by;      // (by may be NaN)
            if (mine_e[r] < 0) continue;
            atomicAdd(&hist[mine_e[r]], 1);
            if (ONE) atomicOr(&mask[mine_e[r] * 8 + (t >> 5)], 1u << (t & 31));
        }
        if (used && lane == 0) atomicAdd(&hist[a.E], 1);
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) acc[i] += ex[i] * den;
    }
    // the wavefront's tokens, then the wavefronts in LDS
#pragma unroll
    for (int i = 0; i < kRoutePer; ++i) {
        const float v = column_sum<L>(acc[i]);
        if ((threadIdx.x & 63) < L && e0 + i < a.E) sums[wave * a.E + e0 + i] = v;
    }
    __syncthreads();
    if (ONE) {
        const RouteScan scan(hist, a.E);
        for (int i = threadIdx.x; i < round_up_64(8 * a.E); i += THREADS) {      // (whole wavefronts)
            const int first = scan(i >> 3);
            if (i < 8 * a.E) place[i] = first + route_before(mask, i);
        }
        __syncthreads();
        const int t = slot;
#pragma unroll
        for (int r = 0; r < REGS; ++r) {
            const int j = r * L + lane;
            if (t >= a.T || j >= a.k || mine_e[r] < 0) continue;
            const int at = mine_e[r] * 8 + (t >> 5);
            a.order[place[at] + __popc(mask[at] & ((1u << (t & 31)) - 1))] = t * a.k + j;
        }
        for (int i = scan.total + threadIdx.x; i < a.T * a.k; i += THREADS) a.order[i] = -1;
        if (wave == WAVES - 1) route_loss(a, hist, sums, WAVES);
        return;
    }
    for (int e = threadIdx.x; e < a.E; e += THREADS) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += sums[w * a.E + e];
        a.psum[e * route_pad(a.groups) + group] = v;
    }
    for (int e = threadIdx.x; e <= a.E; e += THREADS) a.hist[e * route_pad(a.groups) + group] = hist[e];
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
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) c[i] = coef[min(e0 + i, experts - 1)];
        float all = 0.0f, part = 0.0f, wdw = 0.0f, pc = 0.0f;
#pragma unroll
        for (int i = 0; i < kRoutePer; ++i) {
            const bool real = e0 + i < experts;
            ex[i] = real ? expf(l[i] - top) : 0.0f;
            c[i] = real ? c[i] : 0.0f;
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
