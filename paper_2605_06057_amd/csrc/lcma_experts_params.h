// Argument blocks of the 8-bit-integer product and of the tokens' way to their experts and back, shared by the host launchers and
// the kernels.
#pragma once
#include <stdint.h>

namespace lcma {

// n work-groups as `along` x `across`: a dimension of a launch holds fewer than 2^32 threads.  Group number: across * along's extent + along.
struct Groups {
    uint32_t along, across;
};
inline Groups groups_of(int64_t n) {
    const int64_t most = 1 << 20; // (times 1024 threads: 2^30)
    return n <= most ? Groups{(uint32_t)n, 1} : Groups{(uint32_t)most, (uint32_t)((n + most - 1) / most)};
}

// lcma_tokens_sort (csrc/lcma_tokens.hip): n = tokens * top_k slots, up to kSortOnce in one launch, above in blocks of kSortSlots (more than
// kSortBlocks blocks: their counts are summed by a launch of its own).
constexpr int kSortSlots = 2048, kSortOnce = 4096, kSortBlocks = 128, kMaxExperts = 1024;
struct TokensSortParams {
    const int32_t *ids;
    int32_t *order, *position, *offsets;
    int32_t *counts; // blocks x (experts + 1), then (several blocks) experts + 1 totals
    int32_t n, experts, blocks;
};

// lcma_tokens_dispatch, lcma_tokens_combine, lcma_tokens_combine_grad: row pitches in bytes.
struct TokensRowsParams {
    const void *X;           // rows that are read: of tokens (dispatch), in expert order (combine and its gradient)
    const void *dX;          // gradient: of the tokens
    void *Y;                 // rows that are written: in expert order (dispatch, gradient), of tokens (combine)
    const int32_t *position; // tokens x top_k
    const float *weights;    // tokens x top_k, or null: ones
    float *dW;
    int64_t ldx_b, lddx_b, ldy_b;
    int32_t tokens, top_k, H;
    int32_t lane_shift; // 2^lane_shift neighbouring threads along a row
    int32_t stream;     // bit 0: what is written, bit 1: the rows in expert order that are read, pass the caches by
};

// lcma_i8_quantize, lcma_i8_quantize_dispatch (csrc/lcma_i8.hip).
struct I8QuantParams {
    const void *X;
    int8_t *Q;
    float *S;
    const int32_t *position; // dispatch: tokens x top_k rows of Q and S, a negative one is left out; null: row r of X is row r of Q
    int64_t ldx_b;
    int32_t rows, K, pitch, top_k;
};

// Kernels of the product: tiles of 16 x 16 and 32 x 32 (csrc/lcma_i8_few_rows.hpp), of the sizes named (csrc/lcma_i8.hpp), of 256 x 256 (csrc/lcma_i8_pingpong.hpp).
enum { kI8Few16 = 0, kI8Few32, kI8Ring64, kI8Ring64x128, kI8Ring128, kI8Narrow, kI8PingPong, kI8Kernels };

// lcma_i8_gemm_nt, lcma_i8_gemm_experts (csrc/lcma_i8.hpp): rows of A in groups, group e times the weights of expert e.
struct I8GemmParams {
    const int8_t *A, *W;
    const float *SA, *SW, *bias; // bias may be null
    void *C;
    const int32_t *offsets; // experts + 1; null: one group of all rows
    int64_t ldc;            // elements
    int32_t rows, N, pitch; // pitch: bytes of a row of A and W, a multiple of 128
    int32_t experts, steps; // steps of 128 bytes of K
    int32_t nz, panel;      // tiles along N, and the width of a column panel of the tile order
};

} // namespace lcma
