// Rows quantised to 8-bit integers, and the instances of the 8-bit-integer product (csrc/lcma_i8.hpp).
#include "lcma_i8_few_rows.hpp"
#include "lcma_i8_narrow.hpp"
#include "lcma_prepare_b.hpp"

using namespace lcma;

namespace {

// Quantisation of a row: amax = max |x|, scale amax / 127, codes rint(x (127 / amax)), ties to even, all in fp32.  A row of zeros has scale and
// codes zero; one with an infinity or a NaN has codes zero and amax / 127 (infinity, NaN) for its scale, so that its products are NaN.
// Magnitudes are compared as bits: NaN is above infinity there.  Rows below 2^-100 are scaled up first (127 / amax has to be finite).
// GATED: the row is 2 K long and x = silu(row[k]) row[K + k].
// L threads per row (a wave, four or sixteen), eight values at a time: a thread keeps its first two eights in registers and reads others again.  Bound by
// the bytes it moves; the quotient is a product with 127 / amax and the rounding an addition of 1.5 * 2^23 (whose low byte is the code).
// Measured: 8192 x 4096 bf16 18.3 us (5.5 TB/s), gated 8192 x 14336 106 (5.5 TB/s; 208 with a true division and every value computed twice), gated 2 x 14336
// 4.5 (15 with a quarter of the threads), where the shortest launches take 2.8: a row is one work-group's, loads of all of it, a meeting of its 16 waves and its stores one after the other.
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
// silu(g) u = g / (1 + exp(-g)) u for gates far below zero.  exp(-g) leaves fp32 at g = -88.7, where silu is 2^-121 and u may be anything: so the exponential h is
// taken of -|g| / 2 and used twice, g h / (1 + h^2) u h, which holds down to g = -174.  Its argument, to base 2, is in two parts, the second one a linear term: rounded to
// one, it would cost 2^-24 |g| of the result.  |g| is held at 400, where h is zero, for the infinities.
LCMA_DEV float gated_far(float g, float u) {
#pragma clang fp contract(off)
    const float HALF_LOG2E = -0x1.715476p-1f, REST_LN2 = -0x1.4ae0cp-27f * 0x1.62e43p-1f; // -log2(e) / 2 in fp32, and what is left of it times ln(2)
    const float a = __builtin_fminf(__builtin_fabsf(g), 400.f), t = a * HALF_LOG2E;
    const float rest = __builtin_fmaf(a, REST_LN2, __builtin_fmaf(a, HALF_LOG2E, -t) * 0x1.62e43p-1f);
    const float e = __builtin_amdgcn_exp2f(t), h = __builtin_fmaf(e, rest, e), s = g < 0.f ? h : 1.f;
    return g * s * __builtin_amdgcn_rcpf(__builtin_fmaf(h, h, 1.f)) * u * s;
}
template <class T, bool GATED> LCMA_DEV void values(const char *row, int k, int K, float (&v)[8]) {
    eight<T>(row, k, K, v);
    if constexpr (GATED) {
        float u[8];
        eight<T>(row + (int64_t)K * T::ES, k, K, u);
        // eight ordinary gates, above -40, take the direct form (both are within 2^-18 of the value; 8192 x 14336 bf16 111 us, 122 were all gates
        // to take the other)
        float least = v[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) least = __builtin_fminf(least, v[i]);
        if (least < -40.f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = gated_far(v[i], u[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = v[i] * __builtin_amdgcn_rcpf(1.f + __expf(-v[i])) * u[i];
        }
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
LCMA_DEV uint64_t codes(float (&v)[8], const RowScale &s) {
#pragma clang fp contract(off)
    uint32_t c[8];
    if (s.up != 1.f)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= s.up;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = v[i] * s.inv; // (rounded on its own, as the definition says)
        c[i] = __builtin_bit_cast(uint32_t, q + 12582912.f);
    }
    const uint32_t lo = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[3], c[2], 0x0c0c0400), __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400), 0x05040100),
                   hi = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[7], c[6], 0x0c0c0400), __builtin_amdgcn_perm(c[5], c[4], 0x0c0c0400), 0x05040100);
    return s.finite ? (uint64_t)hi << 32 | lo : 0;
}

template <class T, bool GATED, int L> __global__ __launch_bounds__(L < 256 ? 256 : L) void i8_quantize(const I8QuantParams p) {
    constexpr int KEPT = 2, ROWS = L < 256 ? 256 / L : 1;
    __shared__ uint32_t part[L / 64];
    const int64_t r = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ROWS + threadIdx.x / L;
    const int lane = threadIdx.x % L;
    if (r >= p.rows) return; // (L >= 256: a work-group is a row)
    const char *row = (const char *)p.X + r * p.ldx_b;
    uint32_t most = 0;
    float kept[KEPT][8];
#pragma unroll
    for (int n = 0; n < KEPT; ++n) {
        const int k = (n * L + lane) * 8;
        if (k < p.K) values<T, GATED>(row, k, p.K, kept[n]);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) kept[n][i] = 0.f;
    }
#pragma unroll
    for (int n = 0; n < KEPT; ++n)
#pragma unroll
        for (int i = 0; i < 8; ++i) most = max(most, magnitude(kept[n][i]));
    for (int k = (KEPT * L + lane) * 8; k < p.K; k += L * 8) {
        float v[8];
        values<T, GATED>(row, k, p.K, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) most = max(most, magnitude(v[i]));
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d));
    if constexpr (L > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < L / 64; ++w) most = max(most, part[w]);
    }
    const RowScale s = row_scale(most);
    const int32_t *position = p.position ? p.position + r * p.top_k : nullptr;
    const uint32_t slots = (uint32_t)p.rows * p.top_k; // (a position that names none of them is left out, as a negative one)
    auto put = [&](int k, uint64_t c) {
        if (!position) *(uint64_t *)(p.Q + r * p.pitch + k) = c;
        else
            for (int j = 0; j < p.top_k; ++j)
                if (const uint32_t to = position[j]; to < slots) *(uint64_t *)(p.Q + (int64_t)to * p.pitch + k) = c;
    };
#pragma unroll
    for (int n = 0; n < KEPT; ++n) {
        const int k = (n * L + lane) * 8;
        if (k < p.pitch) put(k, codes(kept[n], s)); // (columns behind K: values 0, codes 0)
    }
    for (int k = (KEPT * L + lane) * 8; k < p.pitch; k += L * 8) {
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (k < p.K) values<T, GATED>(row, k, p.K, v);
        put(k, codes(v, s));
    }
    if (!position) {
        if (lane == 0) p.S[r] = s.scale;
    } else {
        for (int j = lane; j < p.top_k; j += L)
            if (const uint32_t to = position[j]; to < slots) p.S[to] = s.scale;
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
LCMA_I8_RING(128, 128, 4, 2, 4)
#define LCMA_I8_FEW(T, WK)                                                                                  \
    template <class OUT> __global__ __launch_bounds__(64 * WK) void i8_few_##T(const I8GemmParams p) {      \
        using G = I8FewRows<T, WK, OUT>;                                                                    \
        __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];                                    \
        G::run(p, (LCMA_LDS char *)smem);                                                                   \
    }
LCMA_I8_FEW(16, 4)
LCMA_I8_FEW(32, 4)
template <class OUT> __global__ __launch_bounds__(512, 2) void i8_narrow(const I8GemmParams) {
    using G = I8Narrow<OUT>;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    G::run((LCMA_LDS char *)smem);
}
template <class OUT> __global__ __launch_bounds__(512, 2) void i8_gemm_256(const I8GemmParams) {
    using G = I8PingPong<OUT>;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS_BYTES];
    G::run((LCMA_LDS char *)smem);
}

} // namespace

// threads: of a row
extern "C" int lcma_launch_i8_quantize(const lcma::I8QuantParams *p, int dtype, int gated, int threads, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
    const Groups g = groups_of(threads == 64 ? ((int64_t)p->rows + 3) / 4 : p->rows);
    const dim3 grid(g.along, g.across);
#define LCMA_QUANTIZE_L(T, G)                                                        \
    if (threads == 64) i8_quantize<T, G, 64><<<grid, dim3(256), 0, s>>>(*p);         \
    else if (threads == 256) i8_quantize<T, G, 256><<<grid, dim3(256), 0, s>>>(*p);  \
    else i8_quantize<T, G, 1024><<<grid, dim3(1024), 0, s>>>(*p);
#define LCMA_QUANTIZE(T)                    \
    if (gated) { LCMA_QUANTIZE_L(T, true) } \
    else { LCMA_QUANTIZE_L(T, false) }
    if (dtype == 0) { LCMA_QUANTIZE(F32) }
    else if (dtype == 1) { LCMA_QUANTIZE(BF16) }
    else { LCMA_QUANTIZE(F16) }
#undef LCMA_QUANTIZE
#undef LCMA_QUANTIZE_L
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
    case kI8Narrow: LCMA_I8(i8_narrow, 512)
    default: LCMA_I8(i8_gemm_256, 512)
    }
#undef LCMA_I8
    return (int)hipGetLastError();
}
