// Weights laid out in 4 bits, and the instances of their product (csrc/lcma_i4.hpp).
#include "lcma_gated.hpp"
#include "lcma_i4.hpp"

using namespace lcma;

namespace {

// A work-group: the blocks of 16 rows; a wave: a block in turn.  Lane: row lane % 16 and, of every 32 columns, the eight from 8 (lane / 16) on.  Codes from their values: rint(x / S),
// S = max |x| / 7 of the group, in fp32, held to -7 .. 7; a group whose S is zero, infinite or NaN has codes of zero.  Runs once for a matrix of weights, and is plain: values come 16 bytes a load,
// codes one by one.  Groups of 128, 14336 x 4096: 53 us from bf16 values (2.8 TB/s), 118 from codes (0.8); eight experts of 28672 x 4096: 625 (3.8 TB/s) and 1754 (0.84), as long as 20 single tokens' products with them.
template <class T, bool CODES> __global__ __launch_bounds__(256) void i4_prepare(const I4PrepareParams p) {
#pragma clang fp contract(off)
    const int lane = threadIdx.x & 63, groups = 128 / p.group, blocks = (p.K + 127) / 128, per_row = (p.K + p.group - 1) / p.group;
    const int64_t row_blocks = ((int64_t)p.N + 15) / 16, all = row_blocks * p.experts;
    const int block_bytes = 1024 + groups * 64;
    for (int64_t nb = blockIdx.x; nb < all; nb += gridDim.x) {
        const int64_t e = nb / row_blocks, n = (nb - e * row_blocks) * 16 + (lane & 15);
        const bool in = n < p.N;
        char *q = p.Q + e * p.expert_q + (nb - e * row_blocks) * blocks * block_bytes;
        const char *row = (const char *)p.W + e * p.expert_b + n * p.ldw_b;
        for (int y = threadIdx.x >> 6; y < blocks; y += 4) {
            u32x4 out;
            float scale[4]; // of the 32 columns' groups
            float v[4][8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = y * 128 + j * 32 + (lane >> 4) * 8;
                if constexpr (CODES) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int c = in && k + i < p.K ? ((const int8_t *)row)[k + i] : 0;
                        v[j][i] = (float)(c < -8 ? -8 : c > 7 ? 7 : c);
                    }
                } else {
                    if (in) eight<T>(row, k, p.K, v[j]);
                    else
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[j][i] = 0.f;
                }
            }
            if constexpr (!CODES) {
                uint32_t most[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) { // magnitudes as bits: NaN is above infinity there
                    most[j] = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) most[j] = max(most[j], __builtin_bit_cast(uint32_t, v[j][i]) & 0x7fffffffu);
                    most[j] = max(most[j], (uint32_t)__shfl_xor((int)most[j], 16));
                    most[j] = max(most[j], (uint32_t)__shfl_xor((int)most[j], 32));
                }
                if (groups <= 2) {
                    most[0] = most[1] = max(most[0], most[1]);
                    most[2] = most[3] = max(most[2], most[3]);
                }
                if (groups == 1) most[0] = most[1] = most[2] = most[3] = max(most[0], most[2]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    scale[j] = __builtin_bit_cast(float, most[j]) / 7.f;
                    const bool none = scale[j] == 0.f || most[j] >= 0x7f800000u;
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[j][i] = none ? 0.f : __builtin_fminf(7.f, __builtin_fmaxf(-7.f, __builtin_rintf(v[j][i] / scale[j])));
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                out[j] = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) out[j] |= (uint32_t)((int)v[j][i] + 8) << (4 * (i / 2 + 4 * (i & 1)));
            }
            char *to = q + (int64_t)y * block_bytes;
            *(u32x4 *)(to + lane * 16) = out;
            const int g = lane >> 4; // (a group's scales: 16 lanes)
            if (g < groups) {
                float s;
                if constexpr (CODES) {
                    const int64_t at = (int64_t)y * groups + g;
                    s = in && at < per_row ? p.S[(e * p.N + n) * per_row + at] : 0.f;
                } else {
                    const int j = g * (4 / groups);
                    s = j == 0 ? scale[0] : j == 1 ? scale[1] : j == 2 ? scale[2] : scale[3];
                }
                *(float *)(to + 1024 + ((lane & 15) * groups + g) * 4) = s * 16.f; // (the product's sums are of q / 16)
            }
        }
    }
}

template <class T, int G, int MT, int WN, int WK, int D, int XB> __global__ __launch_bounds__(64 * WN * WK) void i4_gemm(const I4GemmParams p) {
    using K = I4Gemm<T, G, MT, WN, WK, D, XB>;
    __shared__ __attribute__((aligned(16))) char smem[K::LDS_BYTES];
    K::run(p, (LCMA_LDS char *)smem);
}

} // namespace

// dtype: of the values; -1: codes
extern "C" int lcma_launch_i4_prepare(const lcma::I4PrepareParams *p, int dtype, int grid, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
    if (dtype < 0) i4_prepare<F32, true><<<dim3(grid), dim3(256), 0, s>>>(*p);
    else if (dtype == 0) i4_prepare<F32, false><<<dim3(grid), dim3(256), 0, s>>>(*p);
    else if (dtype == 1) i4_prepare<BF16, false><<<dim3(grid), dim3(256), 0, s>>>(*p);
    else i4_prepare<F16, false><<<dim3(grid), dim3(256), 0, s>>>(*p);
    return (int)hipGetLastError();
}

extern "C" int lcma_launch_i4_gemm(const lcma::I4GemmParams *p, int kernel, int group, int dtype, int grid, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
#define LCMA_I4_G(T, THREADS, ...)                                                                  \
    if (group == 32) i4_gemm<T, 32, __VA_ARGS__><<<dim3(grid), dim3(THREADS), 0, s>>>(*p);          \
    else if (group == 64) i4_gemm<T, 64, __VA_ARGS__><<<dim3(grid), dim3(THREADS), 0, s>>>(*p);     \
    else i4_gemm<T, 128, __VA_ARGS__><<<dim3(grid), dim3(THREADS), 0, s>>>(*p);
// (fp32: three parts of X in LDS)
#define LCMA_I4(MT, WN, WK, D, XB, D32, XB32)                                          \
    if (dtype == 0) { LCMA_I4_G(F32, 64 * WN * WK, MT, WN, WK, D32, XB32) }            \
    else if (dtype == 1) { LCMA_I4_G(BF16, 64 * WN * WK, MT, WN, WK, D, XB) }          \
    else { LCMA_I4_G(F16, 64 * WN * WK, MT, WN, WK, D, XB) }                           \
    break;
    switch (kernel) {
    case kI4Rows16K8: LCMA_I4(1, 1, 8, 2, 66048, 1, 99072)
    case kI4Rows16K4: LCMA_I4(1, 2, 4, 4, 66048, 1, 50048)
    case kI4Rows16: LCMA_I4(1, 4, 1, 4, 33024, 2, 50048)
    default: // (16 bit: three parts of 64 rows do not stay in registers)
        if (dtype == 1) { LCMA_I4_G(BF16, 512, 4, 4, 2, 2, 66560) }
        else { LCMA_I4_G(F16, 512, 4, 4, 2, 2, 66560) }
    }
#undef LCMA_I4
#undef LCMA_I4_G
    return (int)hipGetLastError();
}
