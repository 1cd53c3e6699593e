// Layer norm, its backward and RMSNorm's: argument checks, choice of a kernel and the C entry points.
#include "api_common.h"
#include "norm_kernels.h"

using namespace moc;
using namespace mocapi;

namespace {

constexpr int kMaxNormDim = 16384;      // 64 elements in each of 256 lanes, 32 in each of 512
constexpr int kNormGroups = 256;        // most workgroups of a backward launch, one a compute unit: rows of `part`

moc_status check_norm(int32_t T, int32_t d, int32_t dtype) {
    if (T < 1 || d < 1) return fail(MOC_ERR_BAD_ARG, "T and d must be >= 1 (got %d, %d)", T, d);
    if (dtype != MOC_F32 && dtype != MOC_BF16) return fail(MOC_ERR_BAD_ARG, "unknown dtype %d", dtype);
    if (d > kMaxNormDim) return fail(MOC_ERR_UNSUPPORTED, "d = %d exceeds %d", d, kMaxNormDim);
    return MOC_OK;
}

// Whether rows of d elements all start on 16 bytes.
template <class E> bool rows_aligned(int d) { return d % Vec16<E>::N == 0; }

// f(pieces of W elements, their number NV, lanes of a row): the fewest lanes that hold d elements with at most EL, or twice as many
// in rows past that, in each.
template <class E, int EL, int MIN, int MAX, class F> void for_row(int d, int least, const F& f) {
    constexpr int V = Vec16<E>::N;
    if constexpr (MIN < MAX) {
        if (MIN < least || d > MIN * EL) return for_row<E, EL, 2 * MIN, MAX>(d, least, f);
    }
    typedef std::integral_constant<int, MIN> Lanes;
    const bool aligned = rows_aligned<E>(d), once = d <= MIN * EL;
    if (aligned && once) f(std::integral_constant<int, V>{}, std::integral_constant<int, EL / V>{}, Lanes{});
    else if (once) f(std::integral_constant<int, 1>{}, std::integral_constant<int, EL>{}, Lanes{});
    if constexpr (MIN == MAX) {
        if (aligned && !once) f(std::integral_constant<int, V>{}, std::integral_constant<int, 2 * EL / V>{}, Lanes{});
        else if (!once) f(std::integral_constant<int, 1>{}, std::integral_constant<int, 2 * EL>{}, Lanes{});
    }
}

template <class E> moc_status layernorm(int T, int d, const E* h, const E* gain, const E* bias, float eps, E* out, hipStream_t st) {
    Span span("layernorm", st);
    for_row<E, 32, 64, 256>(d, T < 1024 ? 256 : 64, [&](auto W, auto NV, auto TPR) {
        constexpr int rows = 256 / TPR;
        hipLaunchKernelGGL((layernorm_kernel<E, W, NV, TPR>), dim3((T + rows - 1) / rows), dim3(256), 0, st, h, gain, bias, eps, T, d, out);
    });
    HIP_TRY(hipGetLastError());
    return MOC_OK;
}

template <class E, bool RMS, bool BIAS>
moc_status norm_bwd(int T, int d, const E* h, const E* gain, float eps, const E* dy, const E* dres, E* dh, E* dgain, E* dbias, float* part, hipStream_t st) {
    int groups = 0;
    {
        Span span(RMS ? "rmsnorm_bwd" : "layernorm_bwd", st);
        for_row<E, 16, 64, 512>(d, 64, [&](auto W, auto NV, auto TPR) {
            constexpr int threads = 512, rows = threads / TPR;
            groups = std::min(kNormGroups, (T + rows - 1) / rows);
            hipLaunchKernelGGL((norm_bwd_kernel<E, W, NV, TPR, threads, RMS, BIAS>), dim3(groups), dim3(threads), 0, st, h, gain, eps, dy, dres, T, d, dh, part, dgain,
                               dbias);
        });
    }
    HIP_TRY(hipGetLastError());
    if (groups == 1) return MOC_OK;
    Span span("norm_bwd_join", st);
    const int64_t cols = (int64_t)d * (BIAS ? 2 : 1);
    hipLaunchKernelGGL((norm_bwd_join_kernel<E>), dim3((unsigned)((cols + 63) / 64)), dim3(1024), 0, st, part, groups, cols, d, dgain, dbias);
    HIP_TRY(hipGetLastError());
    return MOC_OK;
}

}  // namespace

extern "C" {

moc_status moc_layernorm(int32_t T, int32_t d, int32_t dtype, const void* h, const void* gain, const void* bias_or_null, float eps, void* out, void* hip_stream) {
    moc_status s = check_norm(T, d, dtype);
    if (s != MOC_OK) return s;
    CHECK_PTR(h); CHECK_PTR(gain); CHECK_PTR(out);
    if (bias_or_null) CHECK_PTR(bias_or_null);
    MOC_SETUP();
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (dtype == MOC_BF16) return layernorm<bf16_t>(T, d, (const bf16_t*)h, (const bf16_t*)gain, (const bf16_t*)bias_or_null, eps, (bf16_t*)out, st);
    return layernorm<float>(T, d, (const float*)h, (const float*)gain, (const float*)bias_or_null, eps, (float*)out, st);
}

size_t moc_norm_bwd_workspace_bytes(int32_t T, int32_t d, int32_t dtype) {
    if (check_norm(T, d, dtype) != MOC_OK) return 0;
    return round_up_sz((size_t)std::min(T, kNormGroups) * 2 * d * sizeof(float), 256);
}

moc_status moc_layernorm_bwd(int32_t T, int32_t d, int32_t dtype, const void* h, const void* gain, float eps, const void* dy, const void* dres_or_null, void* dh,
                             void* dgain, void* dbias_or_null, void* ws, size_t ws_bytes, void* hip_stream) {
    moc_status s = check_norm(T, d, dtype);
    if (s != MOC_OK) return s;
    CHECK_PTR(h); CHECK_PTR(gain); CHECK_PTR(dy); CHECK_PTR(dh); CHECK_PTR(dgain);
    if (dres_or_null) CHECK_PTR(dres_or_null);
    if (dbias_or_null) CHECK_PTR(dbias_or_null);
    CHECK_WS_BYTES(moc_norm_bwd_workspace_bytes(T, d, dtype));
    MOC_SETUP();
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto e) {
        typedef decltype(e) E;
        return dbias_or_null ? norm_bwd<E, false, true>(T, d, (const E*)h, (const E*)gain, eps, (const E*)dy, (const E*)dres_or_null, (E*)dh, (E*)dgain, (E*)dbias_or_null,
                                                       (float*)ws, st)
                             : norm_bwd<E, false, false>(T, d, (const E*)h, (const E*)gain, eps, (const E*)dy, (const E*)dres_or_null, (E*)dh, (E*)dgain, nullptr,
                                                        (float*)ws, st);
    };
    return dtype == MOC_BF16 ? run(bf16_t()) : run(float());
}

moc_status moc_rmsnorm_bwd(int32_t T, int32_t d, int32_t dtype, const void* h, const void* gain, float eps, const void* dy, const void* dres_or_null, void* dh,
                           void* dgain, void* ws, size_t ws_bytes, void* hip_stream) {
    moc_status s = check_norm(T, d, dtype);
    if (s != MOC_OK) return s;
    CHECK_PTR(h); CHECK_PTR(gain); CHECK_PTR(dy); CHECK_PTR(dh); CHECK_PTR(dgain);
    if (dres_or_null) CHECK_PTR(dres_or_null);
    CHECK_WS_BYTES(moc_norm_bwd_workspace_bytes(T, d, dtype));
    MOC_SETUP();
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    auto run = [&](auto e) {
        typedef decltype(e) E;
        return norm_bwd<E, true, false>(T, d, (const E*)h, (const E*)gain, eps, (const E*)dy, (const E*)dres_or_null, (E*)dh, (E*)dgain, nullptr, (float*)ws, st);
    };
    return dtype == MOC_BF16 ? run(bf16_t()) : run(float());
}

}  // extern "C"
