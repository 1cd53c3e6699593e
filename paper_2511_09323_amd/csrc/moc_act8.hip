// Saving a layer's stored set in 8 bits and restoring it: argument checks and the C entry points (the backward pass from such a set is in
// moc_bwd.hip).
#include "act8.h"
#include "api_common.h"

using namespace moc;
using namespace mocapi;

namespace {

// (a step's offsets in a row stay in 32 bits)
moc_status check_width(const moc_shape* shape) {
    if (shape->d > 1 << 24) return fail(MOC_ERR_UNSUPPORTED, "d = %d exceeds 2^24", shape->d);
    return MOC_OK;
}

template <class E> void save(const Dims& D, const E* x, const int32_t* idx, const E* g, const E* u, const moc_act8_set& set, hipStream_t st) {
    Span span("act8_save", st);
    const size_t lds = (size_t)act8_blocks(D.F) * 4;
    hipLaunchKernelGGL((act8_save_kernel<E>), dim3(D.T), dim3(256), lds, st, x, idx, g, u, D.d, D.F, D.K, set);
}

template <class E> void load(const Dims& D, const moc_act8_set& set, E* x, int32_t* idx, E* g, E* u, hipStream_t st) {
    Span span("act8_load", st);
    hipLaunchKernelGGL((act8_load_kernel<E>), dim3(D.T), dim3(256), 0, st, set, D.d, D.F, D.K, x, idx, g, u);
}

}  // namespace

extern "C" {

moc_status moc_act8_save(const moc_shape* shape, const void* x, const int32_t* idx, const void* gvals, const void* uvals, const moc_act8_set* set, void* hip_stream) {
    moc_status s = check_shape(shape, false);
    if (s != MOC_OK) return s;
    if ((s = check_width(shape)) != MOC_OK || (s = check_act8_set(set)) != MOC_OK) return s;
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
    if ((s = check_width(shape)) != MOC_OK || (s = check_act8_set(set)) != MOC_OK) return s;
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
