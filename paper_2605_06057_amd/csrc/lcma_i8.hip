// Rows quantised to 8-bit integers, and the instances of the 8-bit-integer product (csrc/lcma_i8.hpp).
#include "lcma_i8_few_rows.hpp"
#include "lcma_i8_pingpong.hpp"
#include "lcma_prepare_b.hpp"

using namespace lcma;

namespace {

// Quantisation of a row: amax = max |x|, scale amax / 127, codes rint(x (127 / amax)), ties to even, all in fp32.  A row of zeros has scale and
// codes zero; one with an infinity or a NaN has codes zero and amax / 127 (infinity, NaN) for its scale, so that its products are NaN.
// Magnitudes are compared as bits: NaN is above infinity there.  Rows below 2^-100 are scaled up first (127 / amax has to be finite).
// GATED: the row is 2 K long and x = silu(row[k]) row[K + k].
// A work-group of 256 per row; a thread takes eight values at a time.
template <class T> LCMA_DEV void eight(const char *at, int k, int K, float (&v)[8]) { // values k .. k + 7 of a row, zeros from K on
    if (k + 8 <= K) {
        if constexpr (T::ES == 4) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 raw;
                __builtin_memcpy(&raw, at + (int64_t)(k + 4 * h) * 4, 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[4 * h + i] = raw[i];
            }
        } else {
            u32x4 raw;
            __builtin_memcpy(&raw, at + (int64_t)k * 2, 16);
            Widen<T>::run(raw, v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0.f;
            if (k + i < K) {
                if constexpr (T::ES == 4) v[i] = ((const float *)at)[k + i];
                else if constexpr (std::is_same_v<T, F16>) v[i] = (float)((const _Float16 *)at)[k + i];
                else v[i] = __builtin_bit_cast(float, (uint32_t)((const uint16_t *)at)[k + i] << 16);
            }
        }
    }
}
template <class T, bool GATED> LCMA_DEV void values(const char *row, int k, int K, float (&v)[8]) {
    eight<T>(row, k, K, v);
    if constexpr (GATED) {
        float u[8];
        eight<T>(row + (int64_t)K * T::ES, k, K, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] / (1.f + __expf(-v[i])) * u[i];
    }
}
LCMA_DEV uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

struct RowScale {
    float up, inv, scale;
    bool finite;
};
LCMA_DEV RowScale row_scale(uint32_t bits) {
#pragma clang fp contract(off)
    RowScale s;
    const float amax = __builtin_bit_cast(float, bits);
    s.finite = bits < 0x7f800000u;
    s.up = amax < 0x1p-100f ? 0x1p100f : 1.f;
    s.inv = bits && s.finite ? 127.f / (amax * s.up) : 0.f;
    s.scale = amax / 127.f;
    return s;
}
LCMA_DEV uint64_t codes(const float (&v)[8], const RowScale &s) {
#pragma clang fp contract(off)
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = s.finite ? (uint32_t)(int)__builtin_rintf(v[i] * s.up * s.inv) & 255u : 0u;
    return (uint64_t)(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24) | (uint64_t)(c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24) << 32;
}

template <class T, bool GATED> __global__ __launch_bounds__(256) void i8_quantize(const I8QuantParams p) {
    __shared__ uint32_t part[4];
    const int64_t r = blockIdx.x;
    const char *row = (const char *)p.X + r * p.ldx_b;
    uint32_t most = 0;
    for (int k = threadIdx.x * 8; k < p.K; k += 2048) {
        float v[8];
        values<T, GATED>(row, k, p.K, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[i]));
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
    __syncthreads();
    const RowScale s = row_scale(max(max(part[0], part[1]), max(part[2], part[3])));
    for (int k = threadIdx.x * 8; k < p.pitch; k += 2048) {
        uint64_t c = 0;
        if (k < p.K) {
            float v[8];
            values<T, GATED>(row, k, p.K, v);
            c = codes(v, s);
        }
        if (!p.position) *(uint64_t *)(p.Q + r * p.pitch + k) = c;
        else
            for (int j = 0; j < p.top_k; ++j) {
                const int to = p.position[r * p.top_k + j];
                if (to >= 0) *(uint64_t *)(p.Q + (int64_t)to * p.pitch + k) = c;
            }
    }
    if (!p.position) {
        if (threadIdx.x == 0) p.S[r] = s.scale;
    } else {
        for (int j = threadIdx.x; j < p.top_k; j += 256)
            if (const int to = p.position[r * p.top_k + j]; to >= 0) p.S[to] = s.scale;
    }
}

#define LCMA_I8_RING(TM, TN, WGM, WGN, S)                                                                           \
    template <class OUT> __global__ __launch_bounds__(64 * WGM * WGN, 2) void i8_ring_##TM##_##TN(const I8GemmParams p) { \
        using G = I8Ring<TM, TN, WGM, WGN, S, OUT>;                                                                 \
        __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];                                            \
        G::run(p, (LCMA_LDS char *)smem);                                                                           \
    }
LCMA_I8_RING(64, 64, 2, 2, 4)
LCMA_I8_RING(64, 128, 2, 2, 3)
LCMA_I8_RING(128, 128, 2, 4, 4)
LCMA_I8_RING(128, 256, 2, 4, 3)
#define LCMA_I8_FEW(T, WK, S)                                                                               \
    template <class OUT> __global__ __launch_bounds__(64 * WK) void i8_few_##T(const I8GemmParams p) {      \
        using G = I8FewRows<T, WK, S, OUT>;                                                                 \
        __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];                                    \
        G::run(p, (LCMA_LDS char *)smem);                                                                   \
    }
LCMA_I8_FEW(16, 4, 2)
LCMA_I8_FEW(32, 4, 2)
template <class OUT> __global__ __launch_bounds__(512, 2) void i8_gemm_256(const I8GemmParams) {
    using G = I8PingPong<OUT>;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    G::run((LCMA_LDS char *)smem);
}

} // namespace

extern "C" int lcma_launch_i8_quantize(const lcma::I8QuantParams *p, int dtype, int gated, void *stream) {
    const dim3 grid(p->rows), block(256);
    const hipStream_t s = (hipStream_t)stream;
#define LCMA_QUANTIZE(T)                                       \
    if (gated) i8_quantize<T, true><<<grid, block, 0, s>>>(*p); \
    else i8_quantize<T, false><<<grid, block, 0, s>>>(*p);
    if (dtype == 0) { LCMA_QUANTIZE(F32) }
    else if (dtype == 1) { LCMA_QUANTIZE(BF16) }
    else { LCMA_QUANTIZE(F16) }
#undef LCMA_QUANTIZE
    return (int)hipGetLastError();
}

extern "C" int lcma_launch_i8_gemm(const lcma::I8GemmParams *p, int kernel, int dtype, int grid, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
#define LCMA_I8(KERNEL, THREADS)                                                \
    if (dtype == 0) KERNEL<F32><<<dim3(grid), dim3(THREADS), 0, s>>>(*p);       \
    else if (dtype == 1) KERNEL<BF16><<<dim3(grid), dim3(THREADS), 0, s>>>(*p); \
    else KERNEL<F16><<<dim3(grid), dim3(THREADS), 0, s>>>(*p);                  \
    break;
    switch (kernel) {
    case kI8Few16: LCMA_I8(i8_few_16, 256)
    case kI8Few32: LCMA_I8(i8_few_32, 256)
    case kI8Ring64: LCMA_I8(i8_ring_64_64, 256)
    case kI8Ring64x128: LCMA_I8(i8_ring_64_128, 256)
    case kI8Ring128: LCMA_I8(i8_ring_128_128, 512)
    case kI8Ring128x256: LCMA_I8(i8_ring_128_256, 512)
    default: LCMA_I8(i8_gemm_256, 512)
    }
#undef LCMA_I8
    return (int)hipGetLastError();
}
