// Instances of the experts' products (csrc/lcma_experts.hpp).
#include "lcma_experts_pingpong.hpp"

using namespace lcma;

namespace {

template <class T, bool ACOL, bool BCOL, bool GRAD, int TM, int TN, int WGM, int WGN> __global__ __launch_bounds__(64 * WGM * WGN, 2) void exp_staged(const ExpertsGemmParams p) {
    using G = ExpStaged<T, ACOL, BCOL, GRAD, TM, TN, WGM, WGN>;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    G::run(p, (LCMA_LDS char *)smem);
}

template <class T, bool ACOL, bool BCOL, bool GRAD> __global__ __launch_bounds__(512, 2) void exp_256(const ExpertsGemmParams) {
    using G = ExpPingPong<T, ACOL, BCOL, GRAD>;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    G::run((LCMA_LDS char *)smem);
}

} // namespace

// form: 0 the right operand N x K, 1 K x N, 2 the gradient
extern "C" int lcma_launch_experts_gemm(const lcma::ExpertsGemmParams *p, int form, int kernel, int dtype, int grid, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
#define LCMA_EXP_T(NAME, THREADS, ...)                                                                   \
    if (dtype == 0) NAME<F32, __VA_ARGS__><<<dim3(grid), dim3(THREADS), 0, s>>>(*p);                     \
    else if (dtype == 1) NAME<BF16, __VA_ARGS__><<<dim3(grid), dim3(THREADS), 0, s>>>(*p);               \
    else NAME<F16, __VA_ARGS__><<<dim3(grid), dim3(THREADS), 0, s>>>(*p);
#define LCMA_EXP(NAME, THREADS, ...)                                          \
    if (form == 0) { LCMA_EXP_T(NAME, THREADS, false, false, false, __VA_ARGS__) } \
    else if (form == 1) { LCMA_EXP_T(NAME, THREADS, false, true, false, __VA_ARGS__) } \
    else { LCMA_EXP_T(NAME, THREADS, true, true, true, __VA_ARGS__) }         \
    break;
    switch (kernel) {
    case kExpStaged64: LCMA_EXP(exp_staged, 256, 64, 64, 2, 2)
    case kExpStaged128: LCMA_EXP(exp_staged, 256, 128, 128, 2, 2)
    default:
#define LCMA_EXP_256(T)                                                                               \
    if (form == 0) exp_256<T, false, false, false><<<dim3(grid), dim3(512), 0, s>>>(*p);              \
    else if (form == 1) exp_256<T, false, true, false><<<dim3(grid), dim3(512), 0, s>>>(*p);          \
    else exp_256<T, true, true, true><<<dim3(grid), dim3(512), 0, s>>>(*p);
        if (dtype == 1) { LCMA_EXP_256(BF16) }
        else { LCMA_EXP_256(F16) }
#undef LCMA_EXP_256
    }
#undef LCMA_EXP
#undef LCMA_EXP_T
    return (int)hipGetLastError();
}
