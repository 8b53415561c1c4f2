// Tokens sorted by expert and back, for gfx950: the slots (t, j) of tokens x top_k expert numbers in expert order (stable), the rows of
// the tokens copied into that order, rows in that order summed into tokens with the router's weights, and the gradients of both.
//
//   dispatch         Y[position[t, j]] = X[t]                 gradient: combine without weights
//   combine          X[t] = sum_j w[t, j] Y[position[t, j]]   gradient: dY[position[t, j]] = w[t, j] dX[t], dw[t, j] = <dX[t], Y[position[t, j]]>
//
// A slot whose expert number is none of 0 .. experts - 1 has a row behind those of the experts; position holds -1 - row for it.  Such a
// row is written as zeros and never read.  All sums run in fp32 in a fixed order (j ascending; the gradient's dot product over fixed
// lanes), so results do not change from run to run.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lcma_experts_params.h"
#include "lcma_prepare_b.hpp"

namespace {
using namespace lcma;

// ------------------------------------------------------------------ sort
// A stable counting sort.  Eight waves own kSortSlots neighbouring slots, a wave the 512 from its first on; the slots of a round of 64 that
// name the same expert are found with one ballot per bit of the expert number, so a wave's counts need no atomics and the rank of a slot
// is the count before the round plus the lanes below with the same number.
constexpr int kSortWaves = 8, kSortRounds = kSortSlots / (64 * kSortWaves);

// What a wave's lanes wrote to LDS is there for the reads of its other lanes behind this (for the compiler: the LDS works in order).
LCMA_DEV void lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

LCMA_DEV uint64_t same_expert(int e, int bits, bool in) {
    uint64_t m = __ballot(in);
    for (int b = 0; b < bits; ++b) {
        const bool one = e >> b & 1;
        const uint64_t with = __ballot(one);
        m &= one ? with : ~with;
    }
    return m;
}

// Exclusive prefix sums of v[0 .. n) in LDS, by one wave.
LCMA_DEV void prefix_sums(LCMA_LDS int32_t *v, int n, int lane) {
    int carry = 0;
    for (int i = 0; i < n; i += 64) {
        const int mine = i + lane < n ? v[i + lane] : 0;
        int sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int below = __shfl_up(sum, d);
            if (lane >= d) sum += below;
        }
        if (i + lane < n) v[i + lane] = carry + sum - mine;
        carry += __shfl(sum, 63);
    }
}

// STAGE 0: all slots are one block's.  1: counts of every block.  2: rows, from the counts of the blocks before (made by block_prefix).
template <int STAGE> __global__ __launch_bounds__(64 * kSortWaves) void tokens_sort(const TokensSortParams p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int B = p.experts + 1, lane = threadIdx.x & 63, w = threadIdx.x >> 6, bits = 32 - __builtin_clz(p.experts);
    LCMA_LDS int32_t *counts = (LCMA_LDS int32_t *)smem, *first = counts + kSortWaves * B; // first row of every expert (and of the rest)
    LCMA_LDS int32_t *mine = counts + w * B;
    for (int i = threadIdx.x; i < kSortWaves * B; i += 64 * kSortWaves) counts[i] = 0;
    const int64_t slot0 = (int64_t)blockIdx.x * kSortSlots + w * 64 * kSortRounds + lane;
    int e[kSortRounds];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const int64_t slot = slot0 + r * 64;
        const int id = slot < p.n ? p.ids[slot] : 0;
        e[r] = (uint32_t)id < (uint32_t)p.experts ? id : p.experts;
    }
    __syncthreads();
    uint64_t same[kSortRounds];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        same[r] = same_expert(e[r], bits, slot0 + r * 64 < p.n);
        if (slot0 + r * 64 < p.n && (same[r] & ((1ull << lane) - 1)) == 0) mine[e[r]] += __popcll(same[r]);
        lanes_meet();
    }
    __syncthreads();
    // counts become, for every wave, the rows of the expert before its own; first: all of the block (the launch)
    const int32_t *before = p.counts + (int64_t)blockIdx.x * B, *totals = p.counts + (int64_t)p.blocks * B;
    for (int x = threadIdx.x; x < B; x += 64 * kSortWaves) {
        int sum = STAGE == 2 ? before[x] : 0;
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) {
            const int c = counts[k * B + x];
            counts[k * B + x] = sum;
            sum += c;
        }
        if (STAGE == 1) p.counts[(int64_t)blockIdx.x * B + x] = sum;
        else first[x] = STAGE == 2 ? totals[x] : sum;
    }
    if (STAGE == 1) return;
    __syncthreads();
    if (w == 0) prefix_sums(first, B, lane);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int x = threadIdx.x; x < B; x += 64 * kSortWaves) p.offsets[x] = first[x];
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const int64_t slot = slot0 + r * 64;
        if (slot < p.n) {
            const int below = __popcll(same[r] & ((1ull << lane) - 1)), row = first[e[r]] + mine[e[r]] + below;
            p.order[row] = (int32_t)slot;
            p.position[slot] = e[r] < p.experts ? row : -1 - row;
            lanes_meet();
            if (below == 0) mine[e[r]] += __popcll(same[r]);
        }
        lanes_meet();
    }
}

// counts[b][x] over the blocks b of one expert x become the sums before b; the total goes behind them.  One wave per expert.
__global__ __launch_bounds__(64) void block_prefix(const TokensSortParams p) {
    const int B = p.experts + 1, lane = threadIdx.x, x = blockIdx.x;
    int carry = 0;
    for (int b = 0; b < p.blocks; b += 64) {
        int32_t *at = p.counts + (int64_t)(b + lane) * B + x;
        const int mine = b + lane < p.blocks ? *at : 0;
        int sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int below = __shfl_up(sum, d);
            if (lane >= d) sum += below;
        }
        if (b + lane < p.blocks) *at = carry + sum - mine;
        carry += __shfl(sum, 63);
    }
    if (lane == 0) p.counts[(int64_t)p.blocks * B + x] = carry;
}

// ------------------------------------------------------------------ rows
// 16 bytes at any address that is aligned to an element: rows need not be whole vectors, nor start on one.
LCMA_DEV u32x4 load16(const char *at) {
    u32x4 v;
    __builtin_memcpy(&v, at, 16);
    return v;
}
LCMA_DEV void store16(char *at, u32x4 v) { __builtin_memcpy(at, &v, 16); }

template <class T> LCMA_DEV u32x4 packed(const float (&v)[16 / T::ES]) {
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (T::ES == 4) out[i] = __builtin_bit_cast(uint32_t, v[i]);
        else out[i] = Round<T>::run(v[2 * i]) | (Round<T>::run(v[2 * i + 1]) << 16);
    }
    return out;
}
// One element, for rows that are shorter than a vector.
template <class T> LCMA_DEV float element(const char *at) {
    if constexpr (T::ES == 4) return *(const float *)at;
    else if constexpr (std::is_same_v<T, F16>) return (float)*(const _Float16 *)at;
    else return __builtin_bit_cast(float, (uint32_t) * (const uint16_t *)at << 16);
}
template <class T> LCMA_DEV void put_element(char *at, float v) {
    if constexpr (T::ES == 4) *(float *)at = v;
    else *(uint16_t *)at = (uint16_t)Round<T>::run(v);
}

// Vector c of a row of H elements: the last one ends with the row, so it may repeat elements of the one before (which get the same values).
template <class T> LCMA_DEV int64_t vector_at(int c, int H) {
    constexpr int V = 16 / T::ES;
    return (int64_t)(c * V + V <= H ? c * V : H - V) * T::ES;
}

template <class T> __global__ __launch_bounds__(256) void tokens_dispatch(const TokensRowsParams p) {
    constexpr int V = 16 / T::ES;
    const int64_t t = (int64_t)blockIdx.x * (256 >> p.lane_shift) + (threadIdx.x >> p.lane_shift);
    const int c = blockIdx.y * (1 << p.lane_shift) + (threadIdx.x & ((1 << p.lane_shift) - 1));
    if (t >= p.tokens || c * V >= p.H) return;
    const char *x = (const char *)p.X + t * p.ldx_b;
    const int32_t *position = p.position + t * p.top_k;
    if (p.H >= V) {
        const int64_t at = vector_at<T>(c, p.H);
        const u32x4 v = load16(x + at);
        for (int j = 0; j < p.top_k; ++j) {
            const int row = position[j];
            store16((char *)p.Y + (int64_t)(row < 0 ? -1 - row : row) * p.ldy_b + at, row < 0 ? u32x4{0, 0, 0, 0} : v);
        }
    } else {
        for (int j = 0; j < p.top_k; ++j) {
            const int row = position[j];
            char *y = (char *)p.Y + (int64_t)(row < 0 ? -1 - row : row) * p.ldy_b;
            for (int i = 0; i < p.H; ++i) put_element<T>(y + i * T::ES, row < 0 ? 0.f : element<T>(x + i * T::ES));
        }
    }
}

template <class T> __global__ __launch_bounds__(256) void tokens_combine(const TokensRowsParams p) {
    constexpr int V = 16 / T::ES;
    const int64_t t = (int64_t)blockIdx.x * (256 >> p.lane_shift) + (threadIdx.x >> p.lane_shift);
    const int c = blockIdx.y * (1 << p.lane_shift) + (threadIdx.x & ((1 << p.lane_shift) - 1));
    if (t >= p.tokens || c * V >= p.H) return;
    char *y = (char *)p.Y + t * p.ldy_b;
    const int32_t *position = p.position + t * p.top_k;
    const float *weights = p.weights ? p.weights + t * p.top_k : nullptr;
    if (p.H >= V) {
        const int64_t at = vector_at<T>(c, p.H);
        float sum[V];
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] = 0.f;
        for (int j = 0; j < p.top_k; ++j) {
            const int row = position[j];
            if (row < 0) continue;
            const float w = weights ? weights[j] : 1.f;
            float v[V];
            Widen<T>::run(load16((const char *)p.X + (int64_t)row * p.ldx_b + at), v);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] += w * v[i];
        }
        store16(y + at, packed<T>(sum));
    } else {
        for (int i = 0; i < p.H; ++i) {
            float sum = 0.f;
            for (int j = 0; j < p.top_k; ++j)
                if (position[j] >= 0) sum += (weights ? weights[j] : 1.f) * element<T>((const char *)p.X + (int64_t)position[j] * p.ldx_b + i * T::ES);
            put_element<T>(y + i * T::ES, sum);
        }
    }
}

// A work-group per token: its four waves walk along the row, once for every slot.
template <class T> __global__ __launch_bounds__(256) void tokens_combine_grad(const TokensRowsParams p) {
    constexpr int V = 16 / T::ES;
    __shared__ float part[4];
    const int64_t t = blockIdx.x;
    const char *dx = (const char *)p.dX + t * p.lddx_b;
    for (int j = 0; j < p.top_k; ++j) {
        const int pos = p.position[t * p.top_k + j];
        const int64_t row = pos < 0 ? -1 - pos : pos;
        const float w = pos < 0 ? 0.f : p.weights[t * p.top_k + j];
        const char *x = (const char *)p.X + row * p.ldx_b;
        char *y = (char *)p.Y + row * p.ldy_b;
        float dot = 0.f;
        if (pos < 0) {
            for (int c = threadIdx.x; c < p.H; c += 256) put_element<T>(y + c * T::ES, 0.f);
        } else if (p.H >= V) {
            for (int c = threadIdx.x; c * V < p.H; c += 256) {
                const int64_t at = vector_at<T>(c, p.H);
                const int again = c * V - (int)(at / T::ES); // elements that the vector before has counted
                float g[V], v[V], out[V];
                Widen<T>::run(load16(dx + at), g);
                Widen<T>::run(load16(x + at), v);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    out[i] = w * g[i];
                    if (i >= again) dot += g[i] * v[i];
                }
                store16(y + at, packed<T>(out));
            }
        } else if ((int)threadIdx.x < p.H) {
            const float g = element<T>(dx + threadIdx.x * T::ES);
            dot = g * element<T>(x + threadIdx.x * T::ES);
            put_element<T>(y + threadIdx.x * T::ES, w * g);
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) dot += __shfl_xor(dot, d);
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = dot;
        __syncthreads();
        if (threadIdx.x == 0) p.dW[t * p.top_k + j] = (part[0] + part[1]) + (part[2] + part[3]);
        __syncthreads();
    }
}

} // namespace

extern "C" int lcma_launch_tokens_sort(const lcma::TokensSortParams *p, void *stream) {
    const size_t lds = (size_t)(kSortWaves + 1) * (p->experts + 1) * 4;
    const dim3 block(64 * kSortWaves);
    if (p->blocks == 1) {
        tokens_sort<0><<<dim3(1), block, lds, (hipStream_t)stream>>>(*p);
        return (int)hipGetLastError();
    }
    tokens_sort<1><<<dim3(p->blocks), block, lds, (hipStream_t)stream>>>(*p);
    if (const hipError_t e = hipGetLastError()) return (int)e;
    block_prefix<<<dim3(p->experts + 1), dim3(64), 0, (hipStream_t)stream>>>(*p);
    if (const hipError_t e = hipGetLastError()) return (int)e;
    tokens_sort<2><<<dim3(p->blocks), block, lds, (hipStream_t)stream>>>(*p);
    return (int)hipGetLastError();
}

#define LCMA_TOKENS_ROWS(NAME, KERNEL, GRID)                                                                             \
    extern "C" int lcma_launch_tokens_##NAME(const lcma::TokensRowsParams *p, int dtype, int gx, int gy, void *stream) { \
        if (dtype == 0) KERNEL<F32><<<GRID, dim3(256), 0, (hipStream_t)stream>>>(*p);                                    \
        else if (dtype == 1) KERNEL<BF16><<<GRID, dim3(256), 0, (hipStream_t)stream>>>(*p);                              \
        else KERNEL<F16><<<GRID, dim3(256), 0, (hipStream_t)stream>>>(*p);                                               \
        return (int)hipGetLastError();                                                                                   \
    }
LCMA_TOKENS_ROWS(dispatch, tokens_dispatch, dim3(gx, gy))
LCMA_TOKENS_ROWS(combine, tokens_combine, dim3(gx, gy))
LCMA_TOKENS_ROWS(combine_grad, tokens_combine_grad, dim3(gx, gy))
