// Eight values of a row at a time, and the gate of an experts' layer, silu(g) u with silu(g) = g / (1 + exp(-g)), and its gradient.
#pragma once
#include "lcma_prepare_b.hpp"

namespace lcma {

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
// exp(-g) leaves fp32 at g = -88.7, where silu is 2^-121 and what it is multiplied with may be anything: so the exponential h is taken of -|g| / 2 and used twice.  Its
// argument, to base 2, is in two parts, the second one a linear term: rounded to one, it would cost 2^-24 |g| of the result.  |g| is held at 400, where h is zero,
// for the infinities.  r = 1 / (1 + h^2): 1 / (1 + exp(-g)) is r for g >= 0 and h r h below.
struct GateParts {
    float h, r;
};
LCMA_DEV GateParts gate_parts(float g) {
#pragma clang fp contract(off)
    const float HALF_LOG2E = -0x1.715476p-1f, REST_LN2 = -0x1.4ae0cp-27f * 0x1.62e43p-1f; // -log2(e) / 2 in fp32, and what is left of it times ln(2)
    const float a = __builtin_fminf(__builtin_fabsf(g), 400.f), t = a * HALF_LOG2E;
    const float rest = __builtin_fmaf(a, REST_LN2, __builtin_fmaf(a, HALF_LOG2E, -t) * 0x1.62e43p-1f);
    const float e = __builtin_amdgcn_exp2f(t), h = __builtin_fmaf(e, rest, e);
    return {h, __builtin_amdgcn_rcpf(__builtin_fmaf(h, h, 1.f))};
}
// silu(g) u, down to g = -174.
LCMA_DEV float gated_far(float g, float u) {
#pragma clang fp contract(off)
    const GateParts p = gate_parts(g);
    const float s = g < 0.f ? p.h : 1.f;
    return g * s * p.r * u * s;
}
// dy times d silu(g) u / d g = s (1 + g (1 - s)) u and times d / d u = s g, s = 1 / (1 + exp(-g)).  Below zero one h is multiplied in first and one last, so that
// no factor is lost below fp32 before the value is.  (Above it: where dy u itself is beyond fp32 a product on the way may be, and the result an infinity, whatever the value.)
LCMA_DEV void gated_back(float g, float u, float dy, float &dg, float &du) {
#pragma clang fp contract(off)
    const GateParts p = gate_parts(g);
    const float s = g < 0.f ? p.h : 1.f, rest = g < 0.f ? p.r : p.h * p.h * p.r; // (rest: 1 - s)
    const float back = dy * s * p.r;
    dg = back * u * __builtin_fmaf(g, rest, 1.f) * s;
    du = back * g * s;
}

} // namespace lcma
