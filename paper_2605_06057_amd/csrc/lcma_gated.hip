// The gate of an experts' layer and its gradient: rows X = (g, u) of 2 F values, Y = silu(g) u; dX = dY (silu'(g) u, silu(g)).
// Bound by the bytes it moves: three rows of F values forward, five back.  All arithmetic is in fp32, one rounding; the exponential is the accurate form for
// every type (about 20 operations forward and 30 back for a value, where the memory leaves room for 43 and 71).  bf16, 16384 x 14336: 244 us forward and 428 back, 5.8
// and 5.5 TB/s; passing the caches by made both together 727 -> 675 us (from 64 MiB written on: what follows finds less than that in them anyway); 2 rows: 3 us each, a launch.
#include "lcma_gated.hpp"
#include "lcma_i8.hpp"

using namespace lcma;

namespace {

typedef u32x4 u32x4_any __attribute__((aligned(2)));

// Values k .. k + 7 of a row, zeros from K on.  STREAM: past the caches.
template <class T, bool STREAM> LCMA_DEV void take_eight(const char *row, int k, int K, float (&v)[8]) {
    if (!STREAM || k + 8 > K) {
        eight<T>(row, k, K, v);
    } else if constexpr (T::ES == 4) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 raw = __builtin_bit_cast(f32x4, (u32x4)__builtin_nontemporal_load((const u32x4_any *)(row + (int64_t)(k + 4 * h) * 4)));
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * h + i] = raw[i];
        }
    } else {
        Widen<T>::run(__builtin_nontemporal_load((const u32x4_any *)(row + (int64_t)k * 2)), v);
    }
}
template <class T, bool STREAM> LCMA_DEV void put_sixteen(char *at, u32x4 v, int n) {
    if (STREAM && n >= T::CH) __builtin_nontemporal_store(v, (u32x4_any *)at);
    else i8_store16<T>(at, v, n);
}
template <class T, bool STREAM> LCMA_DEV void put_eight(char *at, const float (&v)[8], int n) { // n values, up to 8, from v on
    if constexpr (T::ES == 4) {
#pragma unroll
        for (int h = 0; h < 2; ++h) put_sixteen<T, STREAM>(at + h * 16, __builtin_bit_cast(u32x4, f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]}), n - 4 * h);
    } else {
        u32x4 raw;
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = Round<T>::run(v[2 * i]) | (Round<T>::run(v[2 * i + 1]) << 16);
        put_sixteen<T, STREAM>(at, raw, n);
    }
}

// A thread: eight values of every gridDim.x-th group of rows.
template <class T, bool BACK, bool STREAM> __global__ __launch_bounds__(256) void gated(const GatedParams p) {
    const int lanes = 1 << p.lane_shift, rows_of = 256 >> p.lane_shift, k = ((int)blockIdx.y * lanes + (int)(threadIdx.x & (lanes - 1))) * 8;
    if (k >= p.F) return;
    const int64_t up = (int64_t)p.F * T::ES, at = (int64_t)k * T::ES;
    for (int64_t r = (int64_t)blockIdx.x * rows_of + (threadIdx.x >> p.lane_shift); r < p.rows; r += (int64_t)gridDim.x * rows_of) {
        float g[8], u[8], y[8];
        const char *x = p.X + r * p.ldx_b;
        take_eight<T, STREAM>(x, k, p.F, g);
        take_eight<T, STREAM>(x + up, k, p.F, u);
        if constexpr (BACK) {
            float dg[8], du[8];
            take_eight<T, STREAM>(p.dY + r * p.lddy_b, k, p.F, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) gated_back(g[i], u[i], y[i], dg[i], du[i]);
            char *to = p.Y + r * p.ldy_b + at;
            put_eight<T, STREAM>(to, dg, p.F - k);
            put_eight<T, STREAM>(to + up, du, p.F - k);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = gated_far(g[i], u[i]);
            put_eight<T, STREAM>(p.Y + r * p.ldy_b + at, y, p.F - k);
        }
    }
}

} // namespace

extern "C" int lcma_launch_gated(const lcma::GatedParams *p, int dtype, int back, int gx, int gy, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
#define LCMA_GATED(T)                                                                  \
    if (back && p->stream) gated<T, true, true><<<dim3(gx, gy), dim3(256), 0, s>>>(*p);        \
    else if (back) gated<T, true, false><<<dim3(gx, gy), dim3(256), 0, s>>>(*p);               \
    else if (p->stream) gated<T, false, true><<<dim3(gx, gy), dim3(256), 0, s>>>(*p);          \
    else gated<T, false, false><<<dim3(gx, gy), dim3(256), 0, s>>>(*p);
    if (dtype == 0) { LCMA_GATED(F32) }
    else if (dtype == 1) { LCMA_GATED(BF16) }
    else { LCMA_GATED(F16) }
#undef LCMA_GATED
    return (int)hipGetLastError();
}
