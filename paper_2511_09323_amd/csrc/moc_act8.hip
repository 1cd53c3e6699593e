// Saving a layer's stored set in 8 bits and restoring it: argument checks and the C entry points (the backward pass from such a set is in
// moc_bwd.hip).
#include "act8.h"
#include "api_common.h"

using namespace moc;
using namespace mocapi;

namespace {

template <class E> void save(const Dims& D, const E* x, const int32_t* idx, const E* g, const E* u, const moc_act8_set& set, hipStream_t st) {
    Span span("act8_save", st);
    in_launches(D.T, 1, [&](int64_t t, int n) {
        hipLaunchKernelGGL((act8_save_kernel<E>), dim3(n), dim3(256), (size_t)act8_blocks(D.F) * 4, st, x + t * D.d, idx + t * D.K, g + t * D.K, u + t * D.K, D.d, D.F, D.K,
                           act8_from(set, t, D.d, D.F, D.K));
    });
}

// A wavefront a token has fewer to start and more to wait for in each, but takes longer for its token.  The line goes by the tokens alone: narrow layers would have it at
// 2000, and of the largest sets, which memory bounds, four wavefronts take up to a tenth less.  bf16, sets from memory, us with one and with four: 512 x 1376, K 172,
// 1024 tokens 4.4 and 4.0, 3000 5.9 and 7.1, 4096 7.2 and 9.2, 16384 17.7 and 28.6; 2048 x 5461, K 683, 2048 11.3 and 9.2, 4096 15.6 and 16.0, 6144 19.3 and 22.6, 16384 55.3
// and 50.8; 4096 x 11008, K 1376, 2048 19.2 and 16.0, 4096 28.9 and 28.5, 6144 39.9 and 40.9, 16384 104 and 99.
constexpr int kAct8ManyTokens = 4096;
template <class E> void load(const Dims& D, const moc_act8_set& set, E* x, int32_t* idx, E* g, E* u, hipStream_t st) {
    Span span("act8_load", st);
    if (D.T < kAct8ManyTokens)
        hipLaunchKernelGGL((act8_load_kernel<E, 4>), dim3(D.T), dim3(256), 0, st, set, D.T, D.d, D.F, D.K, x, idx, g, u);
    else
        in_launches(D.T, 4, [&](int64_t t, int n) {
            hipLaunchKernelGGL((act8_load_kernel<E, 1>), dim3((unsigned)(((int64_t)n + 3) / 4)), dim3(256), 0, st, act8_from(set, t, D.d, D.F, D.K), n, D.d, D.F, D.K, x + t * D.d,
                               idx + t * D.K, g + t * D.K, u + t * D.K);
        });
}

}  // namespace

extern "C" {

moc_status moc_act8_save(const moc_shape* shape, const void* x, const int32_t* idx, const void* gvals, const void* uvals, const moc_act8_set* set, void* hip_stream) {
    moc_status s = check_shape(shape, false);
    if (s != MOC_OK) return s;
    if ((s = check_act8_set(shape, set)) != MOC_OK) return s;
    CHECK_PTR(x); CHECK_PTR(idx); CHECK_PTR(gvals); CHECK_PTR(uvals);
    Dims D(*shape);
    MOC_SETUP();
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (shape->dtype == MOC_BF16) save<bf16_t>(D, (const bf16_t*)x, idx, (const bf16_t*)gvals, (const bf16_t*)uvals, *set, st);
    else save<float>(D, (const float*)x, idx, (const float*)gvals, (const float*)uvals, *set, st);
    HIP_TRY(hipGetLastError());
    return MOC_OK;
}

moc_status moc_act8_load(const moc_shape* shape, const moc_act8_set* set, void* x, int32_t* idx, void* gvals, void* uvals, void* hip_stream) {
    moc_status s = check_shape(shape, false);
    if (s != MOC_OK) return s;
    if ((s = check_act8_set(shape, set)) != MOC_OK) return s;
    CHECK_PTR(x); CHECK_PTR(idx); CHECK_PTR(gvals); CHECK_PTR(uvals);
    Dims D(*shape);
    MOC_SETUP();
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (shape->dtype == MOC_BF16) load<bf16_t>(D, *set, (bf16_t*)x, idx, (bf16_t*)gvals, (bf16_t*)uvals, st);
    else load<float>(D, *set, (float*)x, idx, (float*)gvals, (float*)uvals, st);
    HIP_TRY(hipGetLastError());
    return MOC_OK;
}

}  // extern "C"
