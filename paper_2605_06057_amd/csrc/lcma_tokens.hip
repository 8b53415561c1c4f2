// Tokens sorted by expert and back, for gfx950: the slots (t, j) of tokens x top_k expert numbers in expert order (stable), the rows of
// the tokens copied into that order, rows in that order summed into tokens with the router's weights, and the gradients of both.
//
//   dispatch         Y[position[t, j]] = X[t]                 gradient: combine without weights
//   combine          X[t] = sum_j w[t, j] Y[position[t, j]]   gradient: dY[position[t, j]] = w[t, j] dX[t], dw[t, j] = <dX[t], Y[position[t, j]]>
//
// A slot whose expert number is none of 0 .. experts - 1 has a row behind those of the experts; position holds -1 - row for it.  Such a
// row is written as zeros and never read.  All sums run in fp32 in a fixed order (j ascending; the gradient's dot product over fixed
// lanes), so results do not change from run to run.
//
// The calls that move rows are bound by the bytes: 16384 tokens x 4 of 64 experts x 4096 bf16, one after the other: dispatch 125 us (671 MB), combine 111 (671), its
// gradient 230 (1208), the sort 11: 3.2 GB in 590, 5.5 TB/s, where a copy of 2 GiB runs at 4.9 and a read at 6.1.  A token's rows are read or written by
// the same threads, so the token's own row moves once; four rows are in flight together (one after the other: combine 165).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lcma_experts_params.h"
#include "lcma_lanes.hpp"
#include "lcma_prepare_b.hpp"

namespace {
using namespace lcma;

// ------------------------------------------------------------------ sort
// A stable counting sort.  A wave owns 64 R neighbouring slots; the slots of a round of 64 that name the same expert are found with one ballot per bit
// of the expert number, so a wave's counts need no atomics and the rank of a slot is the count before the round plus the lanes below with the
// same number.  What bounds it is latency: up to kSortOnce slots are one work-group's, 16 waves; above, a launch counts blocks of kSortSlots and
// another one places them, every block adding up the counts of those before it (more than kSortBlocks of them: a third launch in between does).
// Measured (us, launches included): 2000 slots of 64 experts 4.6, 4096 5.8, 6126 7.2, 65536 9.1, 131072 of 128 13.9.

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
        const int mine = i + lane < n ? v[i + lane] : 0, sum = lanes_upto(mine);
        if (i + lane < n) v[i + lane] = carry + sum - mine;
        carry += __shfl(sum, 63);
    }
}

// STAGE 0: all slots are one block's.  1: counts of every block.  2: rows, from the counts of all blocks.  3: rows, from what block_prefix made of
// them.  W waves of R rounds each; a wave's counts fit 16 bits.
template <int STAGE, int W, int R> __global__ __launch_bounds__(64 * W) void tokens_sort(const TokensSortParams p) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int B = p.experts + 1, lane = threadIdx.x & 63, w = threadIdx.x >> 6, bits = 32 - __builtin_clz(p.experts);
    LCMA_LDS int32_t *first = (LCMA_LDS int32_t *)smem, *base = first + B; // first row of every expert (and of the rest); rows of it before this block
    LCMA_LDS uint16_t *counts = (LCMA_LDS uint16_t *)(base + B), *mine = counts + w * B;
    for (int i = threadIdx.x; i < W * B; i += 64 * W) counts[i] = 0;
    for (int i = threadIdx.x; i < 2 * B; i += 64 * W) first[i] = 0;
    const int64_t slot0 = (int64_t)blockIdx.x * (64 * W * R) + w * 64 * R + lane;
    int e[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t slot = slot0 + r * 64;
        const int id = slot < p.n ? p.ids[slot] : 0;
        e[r] = (uint32_t)id < (uint32_t)p.experts ? id : p.experts;
    }
    __syncthreads();
    if (STAGE == 2) // (additions of whole numbers: in any order)
        for (int i = threadIdx.x; i < p.blocks * B; i += 64 * W) {
            const int c = p.counts[i], b = i / B, x = i - b * B;
            if (c) __hip_atomic_fetch_add(first + x, c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            if (c && b < (int)blockIdx.x) __hip_atomic_fetch_add(base + x, c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        }
    if (STAGE == 3)
        for (int x = threadIdx.x; x < B; x += 64 * W) {
            first[x] = p.counts[(int64_t)p.blocks * B + x];
            base[x] = p.counts[(int64_t)blockIdx.x * B + x];
        }
    if (STAGE == 1) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (slot0 + r * 64 < p.n) __hip_atomic_fetch_add(first + e[r], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        __syncthreads();
        for (int x = threadIdx.x; x < B; x += 64 * W) p.counts[(int64_t)blockIdx.x * B + x] = first[x];
        return;
    }
    uint64_t same[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        same[r] = same_expert(e[r], bits, slot0 + r * 64 < p.n);
        if (slot0 + r * 64 < p.n && (same[r] & ((1ull << lane) - 1)) == 0) mine[e[r]] += (uint16_t)__popcll(same[r]);
        lanes_meet();
    }
    __syncthreads();
    // counts become, for every wave, the rows of the expert that the waves before it have in this block
    for (int x = threadIdx.x; x < B; x += 64 * W) {
        int sum = 0;
#pragma unroll
        for (int k = 0; k < W; ++k) {
            const int c = counts[k * B + x];
            counts[k * B + x] = (uint16_t)sum;
            sum += c;
        }
        if (STAGE == 0) first[x] = sum;
    }
    __syncthreads();
    if (w == 0) prefix_sums(first, B, lane);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int x = threadIdx.x; x < B; x += 64 * W) p.offsets[x] = first[x];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t slot = slot0 + r * 64;
        if (slot < p.n) {
            const int below = __popcll(same[r] & ((1ull << lane) - 1)), row = first[e[r]] + base[e[r]] + mine[e[r]] + below;
            p.order[row] = (int32_t)slot;
            p.position[slot] = e[r] < p.experts ? row : -1 - row;
            lanes_meet();
            if (below == 0) mine[e[r]] += (uint16_t)__popcll(same[r]);
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
        const int mine = b + lane < p.blocks ? *at : 0, sum = lanes_upto(mine);
        if (b + lane < p.blocks) *at = carry + sum - mine;
        carry += __shfl(sum, 63);
    }
    if (lane == 0) p.counts[(int64_t)p.blocks * B + x] = carry;
}

// ------------------------------------------------------------------ rows
// 16 bytes at any address that is aligned to an element: rows need not be whole vectors, nor start on one.
// STREAM, bit 0: rows that are written, bit 1: rows in expert order that are read pass the caches by (kept there they would push each other out, and
// be written back under the next call's reads).  Measured on dispatch, combine and both gradients: 16384 tokens x 4 x 4096 bf16 646 us, stores alone 610, both
// 589; 4099 x 6 x 1543 fp32 198, 175, 184 (its rows, 152 MB, fit the Infinity Cache: the loads gain nothing by it).
typedef u32x4 u32x4_any __attribute__((aligned(2)));
template <int STREAM> LCMA_DEV u32x4 load16(const char *at) {
    if constexpr (STREAM & 2) return __builtin_nontemporal_load((const u32x4_any *)at);
    else return *(const u32x4_any *)at;
}
template <int STREAM> LCMA_DEV void store16(char *at, u32x4 v) {
    if constexpr (STREAM & 1) __builtin_nontemporal_store(v, (u32x4_any *)at);
    else *(u32x4_any *)at = v;
}

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

// Tokens are dealt out along x, and along z where they are more than x holds (y runs along the rows).
LCMA_DEV int64_t group_number() { return (int64_t)blockIdx.z * gridDim.x + blockIdx.x; }

// Vector c of a row of H elements: the last one ends with the row, so it may repeat elements of the one before (which get the same values).
template <class T> LCMA_DEV int64_t vector_at(int c, int H) {
    constexpr int V = 16 / T::ES;
    return (int64_t)(c * V + V <= H ? c * V : H - V) * T::ES;
}

// The row that a slot has, of `rows` of them; -1 for a position that names none (which is then neither read nor written).
LCMA_DEV int row_of(int position, int rows) {
    const int row = position < 0 ? -1 - position : position;
    return row < rows ? row : -1;
}

template <class T, int STREAM> __global__ __launch_bounds__(256) void tokens_dispatch(const TokensRowsParams p) {
    constexpr int V = 16 / T::ES;
    const int64_t t = group_number() * (256 >> p.lane_shift) + (threadIdx.x >> p.lane_shift);
    const int c = blockIdx.y * (1 << p.lane_shift) + (threadIdx.x & ((1 << p.lane_shift) - 1));
    if (t >= p.tokens || c * V >= p.H) return;
    const char *x = (const char *)p.X + t * p.ldx_b;
    const int32_t *position = p.position + t * p.top_k;
    const int rows = p.tokens * p.top_k;
    if (p.H >= V) {
        const int64_t at = vector_at<T>(c, p.H);
        const u32x4 v = load16<0>(x + at);
        for (int j = 0; j < p.top_k; ++j) {
            const int to = position[j], row = row_of(to, rows);
            if (row >= 0) store16<STREAM>((char *)p.Y + (int64_t)row * p.ldy_b + at, to < 0 ? u32x4{0, 0, 0, 0} : v);
        }
    } else {
        for (int j = 0; j < p.top_k; ++j) {
            const int to = position[j], row = row_of(to, rows);
            char *y = (char *)p.Y + (int64_t)row * p.ldy_b;
            if (row >= 0)
                for (int i = 0; i < p.H; ++i) put_element<T>(y + i * T::ES, to < 0 ? 0.f : element<T>(x + i * T::ES));
        }
    }
}

// Up to four slots of a token from j on: the rows that they have and, of those with an expert, that they read (-1: none), and their weights.
struct Four {
    int has[4], row[4];
    float w[4];
};
LCMA_DEV Four four_slots(const int32_t *position, const float *weights, int j, int top_k, int rows) {
    Four s;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int at = j + q < top_k ? position[j + q] : -1;
        s.has[q] = j + q < top_k ? row_of(at, rows) : -1;
        s.row[q] = at < 0 ? -1 : s.has[q];
        s.w[q] = s.row[q] < 0 ? 0.f : weights ? weights[j + q] : 1.f;
    }
    return s;
}

// A thread: two vectors of a token's row, those of four slots in flight together.
template <class T, int STREAM> __global__ __launch_bounds__(256) void tokens_combine(const TokensRowsParams p) {
    constexpr int V = 16 / T::ES, N = 2;
    const int64_t t = group_number() * (256 >> p.lane_shift) + (threadIdx.x >> p.lane_shift);
    const int lanes = 1 << p.lane_shift, c0 = blockIdx.y * (N * lanes) + (threadIdx.x & (lanes - 1));
    if (t >= p.tokens || c0 * V >= p.H) return;
    char *y = (char *)p.Y + t * p.ldy_b;
    const int32_t *position = p.position + t * p.top_k;
    const float *weights = p.weights ? p.weights + t * p.top_k : nullptr;
    const int rows = p.tokens * p.top_k;
    if (p.H >= V) {
        // (a second vector past the row is the first one again: the same values to the same place)
        const int64_t at[N] = {vector_at<T>(c0, p.H), vector_at<T>((c0 + lanes) * V < p.H ? c0 + lanes : c0, p.H)};
        float sum[N][V];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < V; ++i) sum[n][i] = 0.f;
        for (int j = 0; j < p.top_k; j += 4) {
            const Four s = four_slots(position, weights, j, p.top_k, rows);
            u32x4 raw[4][N];
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int n = 0; n < N; ++n)
                    raw[q][n] = s.row[q] >= 0 ? load16<STREAM>((const char *)p.X + (int64_t)s.row[q] * p.ldx_b + at[n]) : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    float v[V];
                    Widen<T>::run(raw[q][n], v);
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[n][i] += s.w[q] * v[i];
                }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) store16<STREAM>(y + at[n], packed<T>(sum[n]));
    } else {
        for (int i = 0; i < p.H; ++i) {
            float sum = 0.f;
            for (int j = 0; j < p.top_k; ++j)
                if (position[j] >= 0 && position[j] < rows) sum += (weights ? weights[j] : 1.f) * element<T>((const char *)p.X + (int64_t)position[j] * p.ldx_b + i * T::ES);
            put_element<T>(y + i * T::ES, sum);
        }
    }
}

// L threads per token, walking along the rows of four of its slots at a time.
template <class T, int L, int STREAM> __global__ __launch_bounds__(256) void tokens_combine_grad(const TokensRowsParams p) {
    constexpr int V = 16 / T::ES;
    __shared__ float part[4][4];
    const int64_t t = group_number() * (256 / L) + threadIdx.x / L;
    const int lane = threadIdx.x % L;
    if (t >= p.tokens) return; // (L = 256: a work-group is a token)
    const char *dx = (const char *)p.dX + t * p.lddx_b;
    for (int j = 0; j < p.top_k; j += 4) {
        const Four s = four_slots(p.position + t * p.top_k, p.weights + t * p.top_k, j, p.top_k, p.tokens * p.top_k);
        const char *x[4];
        char *y[4];
        float dot[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            x[q] = (const char *)p.X + (int64_t)s.row[q] * p.ldx_b;
            y[q] = (char *)p.Y + (int64_t)s.has[q] * p.ldy_b; // (zeros are written for a slot without an expert)
        }
        if (p.H >= V) {
            for (int c = lane; c * V < p.H; c += L) {
                const int64_t at = vector_at<T>(c, p.H);
                const int again = c * V - (int)(at / T::ES); // elements that the vector before has counted
                float g[V];
                u32x4 raw[4];
                const u32x4 mine = load16<0>(dx + at);
#pragma unroll
                for (int q = 0; q < 4; ++q) raw[q] = s.row[q] >= 0 ? load16<STREAM>(x[q] + at) : u32x4{0, 0, 0, 0};
                Widen<T>::run(mine, g);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (s.has[q] >= 0) {
                        float v[V], out[V];
                        Widen<T>::run(raw[q], v);
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            out[i] = s.row[q] >= 0 ? s.w[q] * g[i] : 0.f;
                            if (i >= again && s.row[q] >= 0) dot[q] += g[i] * v[i];
                        }
                        store16<STREAM>(y[q] + at, packed<T>(out));
                    }
            }
        } else if (lane < p.H) {
            const float g = element<T>(dx + lane * T::ES);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (s.has[q] >= 0) {
                    if (s.row[q] >= 0) dot[q] = g * element<T>(x[q] + lane * T::ES);
                    put_element<T>(y[q] + lane * T::ES, s.row[q] >= 0 ? s.w[q] * g : 0.f);
                }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int d = 32; d; d >>= 1) dot[q] += __shfl_xor(dot[q], d);
        if constexpr (L > 64) {
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int q = 0; q < 4; ++q) part[q][threadIdx.x >> 6] = dot[q];
            __syncthreads();
            if (lane < 4 && j + lane < p.top_k) p.dW[t * p.top_k + j + lane] = (part[lane][0] + part[lane][1]) + (part[lane][2] + part[lane][3]);
            __syncthreads();
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (lane == q && j + q < p.top_k) p.dW[t * p.top_k + j + q] = dot[q];
        }
    }
}

} // namespace

extern "C" int lcma_launch_tokens_sort(const lcma::TokensSortParams *p, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
    const int B = p->experts + 1;
    constexpr int W = 8, R = kSortSlots / (64 * W);
    const size_t lds = (size_t)B * (8 + 2 * W), lds_once = (size_t)B * (8 + 2 * 2 * W);
    if (p->n <= kSortOnce) { // (few slots: half the waves, which start and meet sooner)
        if (p->n <= kSortSlots) tokens_sort<0, W, R><<<dim3(1), dim3(64 * W), lds, s>>>(*p);
        else tokens_sort<0, 2 * W, R><<<dim3(1), dim3(128 * W), lds_once, s>>>(*p);
        return (int)hipGetLastError();
    }
    tokens_sort<1, W, R><<<dim3(p->blocks), dim3(64 * W), lds, s>>>(*p);
    if (const hipError_t e = hipGetLastError()) return (int)e;
    if (p->blocks > kSortBlocks) {
        block_prefix<<<dim3(B), dim3(64), 0, s>>>(*p);
        if (const hipError_t e = hipGetLastError()) return (int)e;
        tokens_sort<3, W, R><<<dim3(p->blocks), dim3(64 * W), lds, s>>>(*p);
    } else {
        tokens_sort<2, W, R><<<dim3(p->blocks), dim3(64 * W), lds, s>>>(*p);
    }
    return (int)hipGetLastError();
}

#define LCMA_TYPES(LAUNCH)         \
    if (dtype == 0) { LAUNCH(F32) } \
    else if (dtype == 1) { LAUNCH(BF16) } \
    else { LAUNCH(F16) }               \
    return (int)hipGetLastError();

static dim3 grid_of(int64_t groups, int gy) {
    const Groups g = groups_of(groups);
    return dim3(g.along, gy, g.across);
}

extern "C" int lcma_launch_tokens_dispatch(const lcma::TokensRowsParams *p, int dtype, int gx, int gy, void *stream) {
    const dim3 grid = grid_of(gx, gy), block(256);
    const hipStream_t s = (hipStream_t)stream;
#define LCMA_DISPATCH(T)                                            \
    if (p->stream) tokens_dispatch<T, 1><<<grid, block, 0, s>>>(*p); \
    else tokens_dispatch<T, 0><<<grid, block, 0, s>>>(*p);
    LCMA_TYPES(LCMA_DISPATCH)
}

extern "C" int lcma_launch_tokens_combine(const lcma::TokensRowsParams *p, int dtype, int gx, int gy, void *stream) {
    const dim3 grid = grid_of(gx, gy), block(256);
    const hipStream_t s = (hipStream_t)stream;
#define LCMA_COMBINE(T)                                                     \
    if (p->stream == 3) tokens_combine<T, 3><<<grid, block, 0, s>>>(*p);     \
    else if (p->stream == 2) tokens_combine<T, 2><<<grid, block, 0, s>>>(*p); \
    else if (p->stream == 1) tokens_combine<T, 1><<<grid, block, 0, s>>>(*p); \
    else tokens_combine<T, 0><<<grid, block, 0, s>>>(*p);
    LCMA_TYPES(LCMA_COMBINE)
}

// a wave per token where its row is no more than 128 vectors, else a work-group; as many rows in expert order are written as are read
extern "C" int lcma_launch_tokens_combine_grad(const lcma::TokensRowsParams *p, int dtype, int wave, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
    const dim3 block(256), tokens = grid_of(p->tokens, 1), fours = grid_of(((int64_t)p->tokens + 3) / 4, 1);
#define LCMA_GRAD(T)                                                                        \
    if (wave) {                                                                             \
        if (p->stream == 3) tokens_combine_grad<T, 64, 3><<<fours, block, 0, s>>>(*p);      \
        else if (p->stream) tokens_combine_grad<T, 64, 1><<<fours, block, 0, s>>>(*p);      \
        else tokens_combine_grad<T, 64, 0><<<fours, block, 0, s>>>(*p);                     \
    } else {                                                                                \
        if (p->stream == 3) tokens_combine_grad<T, 256, 3><<<tokens, block, 0, s>>>(*p);    \
        else if (p->stream) tokens_combine_grad<T, 256, 1><<<tokens, block, 0, s>>>(*p);    \
        else tokens_combine_grad<T, 256, 0><<<tokens, block, 0, s>>>(*p);                   \
    }
    LCMA_TYPES(LCMA_GRAD)
}
