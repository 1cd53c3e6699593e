// Layer norm, its backward and RMSNorm's: argument checks, choice of a kernel and the C entry points.
#include "api_common.h"
#include "norm_kernels.h"

using namespace moc;
using namespace mocapi;

namespace {

constexpr int kFewRows = 128;
constexpr int kMaxNormDim = 16384;      // 64 elements in each of 256 lanes, 32 in each of 512

moc_status check_norm(int32_t T, int32_t d, int32_t dtype) {
    if (T < 1 || d < 1) return fail(MOC_ERR_BAD_ARG, "T and d must be >= 1 (got %d, %d)", T, d);
    if (dtype != MOC_F32 && dtype != MOC_BF16) return fail(MOC_ERR_BAD_ARG, "unknown dtype %d", dtype);
    if (d > kMaxNormDim) return fail(MOC_ERR_UNSUPPORTED, "d = %d exceeds %d", d, kMaxNormDim);
    return MOC_OK;
}

template <RowForm F> struct Form { static constexpr RowForm value = F; };

// f(form of the rows, pieces of a lane, lanes of a row) for the fewest lanes, MIN .. MAX and at least `least` (MORE: may be more than d needs), that hold d
// elements in NV pieces each (fewer than FULL lanes: NV / 2); rows that fill a half or a quarter of that take NV / 2 or NV / 4, rows past MAX lanes 2 or 4
// times as many.
template <class E, int NV, int FULL, int MIN, int MAX, bool MORE, class F> void for_row(int d, int least, const F& f) {
    constexpr int W = Vec16<E>::N, EL = NV * W;
    constexpr bool PARTS = NV >= 4 && (MORE || MIN == 64);
    const auto with = [&](auto nv) {
        const std::integral_constant<int, MIN> lanes{};
        if (d % W == 0) f(Form<RowForm::Whole>{}, nv, lanes);
        else f(Form<RowForm::Odd>{}, nv, lanes);
    };
    if constexpr (MIN == 64) {
        if (d < W) return f(Form<RowForm::Narrow>{}, std::integral_constant<int, 1>{}, std::integral_constant<int, 64>{});
    }
    if constexpr (MIN < MAX) {
        if (MIN < least || d > MIN * (MIN < FULL ? EL / 2 : EL)) return for_row<E, NV, FULL, 2 * MIN, MAX, MORE>(d, least, f);
        if constexpr (PARTS) {
            if (d <= MIN * EL / 4) return with(std::integral_constant<int, NV / 4>{});
            if (d <= MIN * EL / 2) return with(std::integral_constant<int, NV / 2>{});
        }
        if constexpr (MIN >= FULL) with(std::integral_constant<int, NV>{});
    } else {
        if constexpr (PARTS) {
            if (d <= MIN * EL / 4) return with(std::integral_constant<int, NV / 4>{});
            if (d <= MIN * EL / 2) return with(std::integral_constant<int, NV / 2>{});
        }
        if (d <= MIN * EL) return with(std::integral_constant<int, NV>{});
        if constexpr (MIN * EL < kMaxNormDim) {
            if (d <= 2 * MIN * EL) return with(std::integral_constant<int, 2 * NV>{});
        }
        if constexpr (2 * MIN * EL < kMaxNormDim) with(std::integral_constant<int, 4 * NV>{});
    }
}

template <class E> moc_status layernorm(int T, int d, const E* h, const E* gain, const E* bias, float eps, E* out, hipStream_t st) {
    Span span("layernorm", st);
    // The fewest lanes that hold a row, however many rows there are: a row's bits do not depend on the others, and 256 lanes for few rows gain little or lose.  us with the fewest
    // and with 256: bf16 1 x 512 1.70 and 1.93, 512 x 1024 2.05 and 2.77, 128 x 2048 2.24 and 2.26; fp32 512 x 768 2.57 and 2.72, 128 x 2048 2.40 and 2.24.
    for_row<E, 16 / Vec16<E>::N, 64, 64, 256, false>(d, 64, [&](auto form, auto NV, auto TPR) {
        constexpr int rows = 256 / TPR;
        in_launches(T, rows, [&](int64_t t0, int n) {
            hipLaunchKernelGGL((layernorm_kernel<E, decltype(form)::value, NV, TPR>), dim3((unsigned)(((int64_t)n + rows - 1) / rows)), dim3(256), 0, st, h + t0 * d, gain, bias, eps,
                               n, d, out + t0 * d);
        });
    });
    HIP_TRY(hipGetLastError());
    return MOC_OK;
}

template <class E, bool RMS, bool BIAS>
moc_status norm_bwd(int T, int d, const E* h, const E* gain, float eps, const E* dy, const E* dres, E* dh, E* dgain, E* dbias, float* part, hipStream_t st) {
    int groups = 0;
    {
        Span span(RMS ? "rmsnorm_bwd" : "layernorm_bwd", st);
        // A wavefront's registers do not hold 4 pieces of a bf16 layer norm's row, of the next one and of both sums; in fp32 they do, and it gains nothing.  us, with the join, 4
        // pieces from 64 lanes on and from 128: bf16 2047 x 2048 16.8 and 14.4, 8192 x 2048 30.2 and 26.3; fp32 300 x 1001 8.7 and 8.4, 2047 x 1001 13.8 and 13.8, 16384 x 1001
        // 46.2 and 42.8.
        constexpr int NV = 4, FULL = RMS ? 64 : 128, MAX = kNormThreads;
        // A few rows for more than one workgroup leave most of the chip idle, and what counts is how long a row takes: then a piece a lane.  bf16, us: 16 x 4096
        // 13.2 against 9.9, 128 x 2048 9.5 against 8.3; 512 x 4096 15.7 against 16.6; 4 x 2048, one workgroup otherwise, 6.3 against 7.6.
        int least = 64, rows_at_once = 0;
        for_row<E, NV, FULL, 64, MAX, true>(d, least, [&](auto, auto, auto TPR) { rows_at_once = kNormThreads / TPR; });
        while (T > rows_at_once && T <= kFewRows && least < MAX && least * Vec16<E>::N < d) least *= 2;
        for_row<E, NV, FULL, 64, MAX, true>(d, least, [&](auto form, auto NV, auto TPR) {
            constexpr int rows = kNormThreads / TPR;
            groups = (int)std::min<int64_t>(kNormGroups, ((int64_t)T + rows - 1) / rows);
            hipLaunchKernelGGL((norm_bwd_kernel<E, decltype(form)::value, NV, TPR, RMS, BIAS>), dim3(groups), dim3(kNormThreads), 0, st, h, gain, eps, dy, dres, T, d, dh, part, dgain, dbias);
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
