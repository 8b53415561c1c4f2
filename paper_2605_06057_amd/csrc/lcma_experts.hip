// Instances of the experts' products (csrc/lcma_experts.hpp).
#include "lcma_experts_pingpong.hpp"
#include "lcma_experts_any.hpp"
#include "lcma_experts_narrow.hpp"

using namespace lcma;

namespace {

template <class T, bool ACOL, bool BCOL, bool GRAD, int TM, int TN, int WGM, int WGN> __global__ __launch_bounds__(64 * WGM * WGN, 2) void exp_staged(const ExpertsGemmParams p) {
    using G = ExpStaged<T, ACOL, BCOL, GRAD, TM, TN, WGM, WGN>;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    G::run(p, (LCMA_LDS char *)smem);
}

template <class T, bool ACOL, bool BCOL, bool GRAD, int TM, int TN, int WGM, int WGN> __global__ __launch_bounds__(64 * WGM * WGN, 2) void exp_ring(const ExpertsGemmParams p) {
    using G = ExpRing<T, ACOL, BCOL, GRAD, TM, TN, WGM, WGN>;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    G::run(p, (LCMA_LDS char *)smem);
}
template <class T, bool BCOL, int R, int WK> __global__ __launch_bounds__(64 * WK) void exp_few(const ExpertsGemmParams p) {
    using G = ExpFewRows<T, BCOL, R, WK>;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    G::run(p, (LCMA_LDS char *)smem);
}
template <class T, bool BCOL, int WK> __global__ __launch_bounds__(64 * WK) void exp_any_few(const ExpertsGemmParams p) {
    using G = ExpAnyFewRows<T, BCOL, WK>;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    G::run(p, (LCMA_LDS char *)smem);
}
template <class T, bool BCOL> __global__ __launch_bounds__(512, 2) void exp_narrow(const ExpertsGemmParams) {
    using G = ExpNarrow<T, BCOL>;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    G::run((LCMA_LDS char *)smem);
}
template <class T, bool ACOL, bool BCOL, bool GRAD, bool LINES = false> __global__ __launch_bounds__(512, 2) void exp_256(const ExpertsGemmParams) {
    using G = ExpPingPong<T, ACOL, BCOL, GRAD, LINES>;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    G::run((LCMA_LDS char *)smem);
}

} // namespace

// form: 0 the right operand N x K, 1 K x N, 2 the gradient
extern "C" int lcma_launch_experts_gemm(const lcma::ExpertsGemmParams *p, int form, int kernel, int dtype, int grid, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
#define LCMA_EXP_LAUNCH(THREADS, ...) __VA_ARGS__<<<dim3(grid), dim3(THREADS), 0, s>>>(*p)
#define LCMA_EXP_FORM(NAME, THREADS, T, ...)                                                          \
    if (form == 0) LCMA_EXP_LAUNCH(THREADS, NAME<T, false, false, false __VA_ARGS__>);                \
    else if (form == 1) LCMA_EXP_LAUNCH(THREADS, NAME<T, false, true, false __VA_ARGS__>);            \
    else LCMA_EXP_LAUNCH(THREADS, NAME<T, true, true, true __VA_ARGS__>);
#define LCMA_EXP(NAME, THREADS, ...)                                           \
    if (dtype == 1) { LCMA_EXP_FORM(NAME, THREADS, BF16, __VA_ARGS__) }        \
    else { LCMA_EXP_FORM(NAME, THREADS, F16, __VA_ARGS__) }                    \
    break;
#define LCMA_EXP_ANY(NAME, THREADS, ...)                                       \
    if (dtype == 0) { LCMA_EXP_FORM(NAME, THREADS, F32, __VA_ARGS__) }         \
    else LCMA_EXP(NAME, THREADS, __VA_ARGS__)                                  \
    break;
#define LCMA_COMMA ,
    switch (kernel) {
    case kExpStaged64: LCMA_EXP_ANY(exp_staged, 256, LCMA_COMMA 64, 64, 2, 2)
    case kExpStaged128: LCMA_EXP_ANY(exp_staged, 256, LCMA_COMMA 128, 128, 2, 2)
    case kExpAnyFew32:
        if (dtype == 1 && form == 0) LCMA_EXP_LAUNCH(256, exp_any_few<BF16, false, 4>);
        else if (dtype == 1) LCMA_EXP_LAUNCH(256, exp_any_few<BF16, true, 4>);
        else if (form == 0) LCMA_EXP_LAUNCH(256, exp_any_few<F16, false, 4>);
        else LCMA_EXP_LAUNCH(256, exp_any_few<F16, true, 4>);
        break;
    case kExpFew16:
        if (dtype == 1) LCMA_EXP_LAUNCH(256, exp_few<BF16, false, 16, 4>);
        else LCMA_EXP_LAUNCH(256, exp_few<F16, false, 16, 4>);
        break;
    case kExpFew32:
        if (dtype == 0 && form == 0) LCMA_EXP_LAUNCH(256, exp_few<F32, false, 32, 4>);
        else if (dtype == 0) LCMA_EXP_LAUNCH(256, exp_few<F32, true, 32, 4>);
        else if (dtype == 1 && form == 0) LCMA_EXP_LAUNCH(256, exp_few<BF16, false, 32, 4>);
        else if (dtype == 1) LCMA_EXP_LAUNCH(256, exp_few<BF16, true, 32, 4>);
        else if (form == 0) LCMA_EXP_LAUNCH(256, exp_few<F16, false, 32, 4>);
        else LCMA_EXP_LAUNCH(256, exp_few<F16, true, 32, 4>);
        break;
    case kExpRing64: LCMA_EXP_ANY(exp_ring, 256, LCMA_COMMA 64, 64, 2, 2)
    case kExpRing64x128: LCMA_EXP(exp_ring, 256, LCMA_COMMA 64, 128, 2, 2)
    case kExpNarrow:
        if (dtype == 1 && form == 0) LCMA_EXP_LAUNCH(512, exp_narrow<BF16, false>);
        else if (dtype == 1) LCMA_EXP_LAUNCH(512, exp_narrow<BF16, true>);
        else if (form == 0) LCMA_EXP_LAUNCH(512, exp_narrow<F16, false>);
        else LCMA_EXP_LAUNCH(512, exp_narrow<F16, true>);
        break;
    default:
        if (form == 2 && p->lines) {
            if (dtype == 1) LCMA_EXP_LAUNCH(512, exp_256<BF16, true, true, true, true>);
            else LCMA_EXP_LAUNCH(512, exp_256<F16, true, true, true, true>);
            break;
        }
        LCMA_EXP(exp_256, 512, )
    }
#undef LCMA_EXP_LAUNCH
#undef LCMA_EXP_FORM
#undef LCMA_EXP
#undef LCMA_EXP_ANY
#undef LCMA_COMMA
    return (int)hipGetLastError();
}
