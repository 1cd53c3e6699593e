// The router and its gradient: argument checks, choice of a kernel and the C entry points.
#include "api_common.h"
#include "route.h"

using namespace moc;
using namespace mocapi;

namespace {

moc_status check_route(int32_t T, int32_t E, int32_t k, int32_t dtype) {
    if (T < 1 || E < 1) return fail(MOC_ERR_BAD_ARG, "T and E must be >= 1 (got %d, %d)", T, E);
    if (k < 1 || k > E) return fail(MOC_ERR_BAD_ARG, "k must satisfy 1 <= k <= E (got k=%d, E=%d)", k, E);
    if (dtype != MOC_F32 && dtype != MOC_BF16) return fail(MOC_ERR_BAD_ARG, "unknown dtype %d", dtype);
    if (E > kMaxRouteExperts) return fail(MOC_ERR_UNSUPPORTED, "E = %d exceeds %d", E, kMaxRouteExperts);
    if (k > kMaxRouteSlots) return fail(MOC_ERR_UNSUPPORTED, "k = %d exceeds %d", k, kMaxRouteSlots);
    if ((int64_t)T * k > INT32_MAX - 65536) return fail(MOC_ERR_UNSUPPORTED, "T*k = %lld copies are too many", (long long)T * k);
    return MOC_OK;
}

struct RouteWs {
    int groups, chunk;
    int32_t* hist;
    float* psum;
    size_t bytes;
    RouteWs(void* ws, int T, int E) {
        // one pass of route_rows_kernel, 256 tokens at most, unless that makes too many workgroups
        int lanes = 1;
        while (lanes * kRoutePer < E) lanes *= 2;
        chunk = std::max(route_threads(lanes) / lanes, (T + kRouteGroups - 1) / kRouteGroups);
        groups = (T + chunk - 1) / chunk;
        Carver c(ws);
        hist = c.take<int32_t>((size_t)route_pad(groups) * (E + 1));
        psum = c.take<float>((size_t)route_pad(groups) * E);
        bytes = c.off;
    }
};

// f(lanes of a token, whether its logits are whole 16-byte pieces)
template <class E, int L = 1, class F> void for_token(int experts, const F& f) {
    if constexpr (L < 32) {
        if (experts > L * kRoutePer) return for_token<E, 2 * L>(experts, f);
    }
    if (experts % Vec16<E>::N == 0) f(std::integral_constant<int, L>{}, std::true_type{});
    else f(std::integral_constant<int, L>{}, std::false_type{});
}

template <class E> moc_status route(const E* logits, const RouteArgs& a, hipStream_t st) {
    {
        Span span("route_rows", st);
        for_token<E>(a.E, [&](auto L, auto vec) {
            constexpr int threads = route_threads(L);
            if (a.groups == 1)
                hipLaunchKernelGGL((route_rows_kernel<E, L, vec, true>), dim3(1), dim3(threads), route_rows_words(a.E, threads, true) * 4, st, logits, a);
            else
                hipLaunchKernelGGL((route_rows_kernel<E, L, vec, false>), dim3(a.groups), dim3(threads), route_rows_words(a.E, threads, false) * 4, st, logits, a);
        });
    }
    HIP_TRY(hipGetLastError());
    if (a.groups == 1) return MOC_OK;
    Span span("route_order", st);
    hipLaunchKernelGGL(route_order_kernel, dim3(a.groups + 1), dim3(kRouteOrderThreads), 0, st, a);
    HIP_TRY(hipGetLastError());
    return MOC_OK;
}

template <class E>
moc_status route_bwd(int T, int experts, int k, bool renorm, const E* logits, const int32_t* ids, const float* coef, const float* dweights, const float* dloss, E* dlogits,
                     hipStream_t st) {
    Span span("route_bwd", st);
    for_token<E>(experts, [&](auto L, auto vec) {
        constexpr int tokens = 256 / L;
        in_launches(T, tokens, [&](int64_t t0, int n) {
            hipLaunchKernelGGL((route_bwd_kernel<E, L, vec>), dim3((n + tokens - 1) / tokens), dim3(256), 0, st, n, experts, k, renorm, logits + t0 * experts, ids + t0 * k, coef,
                               dweights ? dweights + t0 * k : nullptr, dloss, dlogits + t0 * experts);
        });
    });
    HIP_TRY(hipGetLastError());
    return MOC_OK;
}

}  // namespace

extern "C" {

size_t moc_route_workspace_bytes(int32_t T, int32_t E, int32_t k) {
    if (check_route(T, E, k, MOC_F32) != MOC_OK) return 0;
    return RouteWs(nullptr, T, E).bytes;
}

moc_status moc_route(int32_t T, int32_t E, int32_t k, int32_t dtype, int32_t renorm, const void* logits, const uint8_t* valid_or_null, int32_t* ids, float* weights,
                     int32_t* counts, int32_t* order, float* loss, float* coef, void* ws, size_t ws_bytes, void* hip_stream) {
    moc_status s = check_route(T, E, k, dtype);
    if (s != MOC_OK) return s;
    CHECK_PTR(logits); CHECK_PTR(ids); CHECK_PTR(weights); CHECK_PTR(counts); CHECK_PTR(order); CHECK_PTR(loss); CHECK_PTR(coef);
    if (valid_or_null) CHECK_PTR(valid_or_null);
    CHECK_WS_BYTES(moc_route_workspace_bytes(T, E, k));
    MOC_SETUP();
    const RouteWs W(ws, T, E);
    const RouteArgs a{T, E, k, W.chunk, W.groups, renorm != 0, valid_or_null, ids, weights, counts, order, loss, coef, W.hist, W.psum};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return dtype == MOC_BF16 ? route<bf16_t>((const bf16_t*)logits, a, st) : route<float>((const float*)logits, a, st);
}

moc_status moc_route_bwd(int32_t T, int32_t E, int32_t k, int32_t dtype, int32_t renorm, const void* logits, const int32_t* ids, const float* coef,
                         const float* dweights_or_null, const float* dloss_or_null, void* dlogits, void* hip_stream) {
    moc_status s = check_route(T, E, k, dtype);
    if (s != MOC_OK) return s;
    CHECK_PTR(logits); CHECK_PTR(ids); CHECK_PTR(coef); CHECK_PTR(dlogits);
    if (dweights_or_null) CHECK_PTR(dweights_or_null);
    if (dloss_or_null) CHECK_PTR(dloss_or_null);
    MOC_SETUP();
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (dtype == MOC_BF16)
        return route_bwd<bf16_t>(T, E, k, renorm != 0, (const bf16_t*)logits, ids, coef, dweights_or_null, dloss_or_null, (bf16_t*)dlogits, st);
    return route_bwd<float>(T, E, k, renorm != 0, (const float*)logits, ids, coef, dweights_or_null, dloss_or_null, (float*)dlogits, st);
}

}  // extern "C"
