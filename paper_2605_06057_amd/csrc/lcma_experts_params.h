// Argument blocks of the 8-bit-integer product, of the tokens' way to their experts and back, of the experts' products in their own type and of their gate,
// shared by the host launchers and the kernels.
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

// Kernels of the experts' products: any sizes and alignments (csrc/lcma_experts.hpp, and in 16 bit
// lcma_experts_any.hpp); 16 bit in whole 16 bytes and fp32 (csrc/lcma_experts_ring.hpp); 16 bit in whole 16 bytes
// (csrc/lcma_experts_narrow.hpp, lcma_experts_pingpong.hpp).  Tiles of 16 x 16: 16 bit, weights N x K alone; of 64 x 128: 16 bit; of 16,
// 32 and 128 rows: no gradient of weights.
enum { kExpStaged64 = 0, kExpStaged128, kExpAnyFew32, kExpFew16, kExpFew32, kExpRing64, kExpRing64x128, kExpNarrow, kExpPingPong, kExpKernels };

// lcma_gemm_experts: rows of A (k-contiguous) in groups, group e times the matrix of expert e (N x K, or K x N).
// lcma_gemm_experts_grad: for every expert the product of its rows of A, transposed, and its rows of B: M x N, summed over the rows.
struct ExpertsGemmParams {
    const char *A, *B;
    char *C;
    const int32_t *offsets;         // experts + 1
    int64_t lda_b, ldb_b, ldc_b;    // bytes from a row of the stored matrices to the next
    int64_t expert_b;               // bytes from an expert's matrix to the next: of B (product), of C (gradient)
    int32_t rows, M, N, K, experts; // M: rows of an expert's C (gradient); K: what a product sums over
    int32_t nx, nz, panel;          // tiles along M (gradient) and N; width of a column panel of the tile order (product)
    int32_t stream, lines;          // the gradient passes the caches by; the 256 x 256 tiles' waves write whole lines of it
    int32_t by_expert;              // the gradient's tiles are dealt to the XCDs by experts, not by eighths of each
    int32_t from;                   // kernels with a work-group for each tile: the launch's first tile of each eighth of them
};

// lcma_gated_silu, lcma_gated_silu_grad: row pitches in bytes.
struct GatedParams {
    const char *X, *dY;
    char *Y; // or dX
    int64_t ldx_b, lddy_b, ldy_b;
    int32_t rows, F;
    int32_t lane_shift; // 2^lane_shift neighbouring threads along a row
    int32_t stream;     // the rows pass the caches by
};

// 4-bit weights (csrc/lcma_i4.hpp): blocks of 16 rows x 128 columns, a row of blocks behind the other; a block is its codes (1024 bytes) and the scales
// (fp32) of its 16 rows' groups.
inline int64_t i4_block_bytes(int group) { return 1024 + 128 / group * 64; }
// lcma_i4_quantize, lcma_i4_prepare: rows x K values, or codes and scales, laid out as blocks.
struct I4PrepareParams {
    const void *W;       // values in a storage type, or codes (int8)
    const float *S;      // scales (rows x groups), or null: quantise
    char *Q;
    int64_t ldw_b, expert_b, expert_q; // bytes from row to row, from expert to expert
    int32_t N, K, group, experts;
};
// Kernels of the product with them: rows of a tile; blocks of rows of the weights in it; waves along K.
enum { kI4Rows16K8 = 0, kI4Rows16K4, kI4Rows16, kI4Rows64, kI4Kernels };
// lcma_i4_gemm_nt, lcma_i4_gemm_experts.
struct I4GemmParams {
    const char *X, *Q;
    const float *bias;      // N, or experts x N; may be null
    char *C;
    const int32_t *offsets; // experts + 1; null: one group of all rows
    int64_t ldx_b, ldc, expert_q; // ldc: elements
    int32_t rows, N, K, experts;
    int32_t blocks;         // of 128 columns
    int32_t nz, panel;      // tiles along N
    int32_t from;           // the launch's first tile of each eighth of them
};

} // namespace lcma
