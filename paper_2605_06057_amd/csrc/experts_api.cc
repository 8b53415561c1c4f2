// Host side of the experts' products in their own type and of their gate: argument checks, launches.
#include "experts_host.h"

#include <cmath>
#include <cstring>

extern "C" int lcma_launch_experts_gemm(const lcma::ExpertsGemmParams *p, int form, int kernel, int dtype, int grid, void *stream);
extern "C" int lcma_launch_gated(const lcma::GatedParams *p, int dtype, int back, int gx, int gy, void *stream);

using namespace lcma;

namespace {

const int kTile[kExpKernels][2] = {{64, 64}, {128, 128}, {32, 32}, {16, 16}, {32, 32}, {64, 64}, {64, 128}, {128, 256}, {256, 256}}; // rows and columns of the kernels' tiles

int64_t span(int64_t rows, int64_t ld, int64_t cols, int es) { return rows > 0 && cols > 0 ? ((rows - 1) * ld + cols) * es : 0; }
int64_t tiles(int64_t n, int64_t of) { return (n + of - 1) / of; }

// Tiles, at most: every group of rows may end in one of its own that is not full.
int64_t product_tiles(int kernel, int64_t rows, int64_t N, int experts) {
    return (rows / kTile[kernel][0] + (rows < experts ? rows : experts)) * tiles(N, kTile[kernel][1]);
}
int64_t gradient_tiles(int kernel, int64_t M, int64_t N, int experts) { return experts * tiles(M, kTile[kernel][0]) * tiles(N, kTile[kernel][1]); }
bool needs_vectors(int kernel) { return kernel >= kExpFew16; }
bool walks(int kernel) { return kernel >= kExpNarrow; } // 256 work-groups walk through tiles; the other kernels have one for every tile
bool launches(int kernel, int64_t jobs) { return walks(kernel) ? several_launches(jobs) : one_launch(jobs); }
// Work-groups for `jobs` tiles, dealt out `whole` at a time (a multiple of eight); several launches where one does not hold them.
int launch(ExpertsGemmParams &p, int form, int kernel, int dtype, int64_t jobs, int64_t whole, void *stream) {
    if (walks(kernel)) return lcma_launch_experts_gemm(&p, form, kernel, dtype, 256, stream);
    const int64_t eighth = (jobs + whole - 1) / whole * whole / 8, most = one_launch(jobs) ? eighth : kLaunchEighth;
    for (int64_t from = 0; from < eighth; from += most) {
        p.from = (int32_t)from;
        if (const int err = lcma_launch_experts_gemm(&p, form, kernel, dtype, (int)((eighth - from < most ? eighth - from : most) * 8), stream)) return err;
    }
    return 0;
}
// What the kernels that load straight into LDS need: offsets inside a tile (256 rows of a k-contiguous operand, 128 rows along k of the other) below 2^30 bytes, and, 16-bit types,
// operands in whole 16 bytes (of a k-contiguous one K too, of the other form the rows).
const int64_t kShortRow = 1 << 22;
bool whole_vectors(int es, const void *A, int64_t lda_b, const void *B, int64_t ldb_b, int64_t k_b) {
    return es == 4 || !(((uintptr_t)A | (uintptr_t)B | (uint64_t)lda_b | (uint64_t)ldb_b | (uint64_t)k_b) & 15);
}

// What a kernel takes, in us: `start`; a tile: `end`, and `step` for every 128 bytes of K, 256 * `slots` tiles at a time; and no less than the bytes at `rate` GB/us take.  With rows that
// are no whole lines of 128 bytes a step takes `off` of its time more and the bytes half of that.  start 0: not taken.  Fitted to 164 layers in 16 bit, 94 in fp32 and 130 of sizes
// that are no whole 16 bytes, of 1 to 8192 tokens and 8 to 128 experts, timed on every kernel: a single time is predicted within 10 to 31 % (root mean square); the kernel with the smallest
// prediction is 1.2 to 2.4 % slower than the fastest one on average in whole 16 bytes (31 % at worst, of the gradient 65 %), 0.2 to 0.6 % in fp32 (18 %), 1.5 to 3 % in other sizes (52 %, one gradient 2.2 times).
// (The fp32 gradient's 64 x 64 came out as a line through the number of tiles, `slots` and `step` near nothing: it tells large ones apart, and nothing of less than a round of tiles.)
struct Cost {
    double start, end, step, rate, slots, off;
};
enum { kNt, kNn, kGrad, kForms };
const Cost kVectors[kForms][kExpKernels] = {
    {{}, {}, {}, {2.18, 0.29, 0.0312, 7.08, 0.655, 0.17}, {2.02, 0.655, 0.063, 6.15, 0.62, 0.118}, {2.06, 0.384, 0.209, 6.01, 0.812, 0.122}, {2.24, 0.706, 0.315, 5.88, 0.752, 0.133},
     {3.57, 1.83, 0.71, 5.44, 0.591, 0.0682}, {4.63, 0.567, 0.977, 4.55, 0.584, 0.0691}},
    {{}, {}, {}, {}, {1.97, 0.596, 0.0866, 5.53, 0.604, 0.0683}, {2.15, 0.344, 0.256, 6.65, 0.821, 0.0253}, {2.25, 0.764, 0.373, 6.08, 0.788, 0}, {3.23, 2.24, 0.768, 5.83, 0.633, 0},
     {4.99, 0.065, 1.01, 4.75, 0.615, 0}},
    {{}, {}, {}, {}, {}, {2.41, 1.19, 0.459, 3.86, 2.25, 0.284}, {2.77, 1.17, 0.448, 4.53, 1.31, 0.273}, {}, {5.47, 1.85, 0.977, 5.66, 0.552, 0.386}}};
const Cost kF32[kForms][kExpKernels] = {{{}, {}, {}, {}, {2.59, 0.891, 0.152, 5.93, 0.928, 0.0706}, {2.86, 0.396, 0.563, 6.81, 1.03, 0}},
                                        {{}, {}, {}, {}, {2.24, 1.22, 0.16, 7.18, 0.961, 0.0109}, {2.3, 0.878, 0.599, 5.28, 1.11, 0.0132}},
                                        {{3.11, 0.013, 1.09, 5.6, 1.5, 0.12}, {}, {}, {}, {}, {2.89, 0.000258, 0.000758, 4.66, 0.00135, 0.203}}};
const Cost kAny[kForms][kExpKernels] = {{{1.98, 1.45, 0.774, 5.02, 2.17, 0.208}, {2.21, 3.11, 1.37, 4.11, 1.51, 0.191}, {1.74, 3.17, 0.401, 3.66, 1.98, 0.05}},
                                        {{1.25, 0, 1.82, 3.62, 3.35, 0.25}, {}, {1.53, 1.51, 0.833, 2.71, 2.97, 0.193}}, // (128 x 128 was up to 1.8 x slower where it was taken and is up to 1.4 x faster on a tenth: 3.5 % over the fastest with it, 2.9 without)
                                        {{3.05, 0, 3.63, 2.73, 9.43, 0.315}, {3.94, 0, 5.06, 3.52, 3.62, 0.347}}};
double predicted_us(const Cost &c, double tiles, double steps, bool off, double bytes) {
    const double o = off ? c.off : 0, n = tiles / 256 / c.slots, t = c.start + (c.end + steps * c.step * (1 + o)) * (n > 1 ? n : 1), memory = c.start + bytes / (c.rate * 1e6) * (1 + 0.5 * o);
    return std::sqrt(std::sqrt(t * t * t * t + memory * memory * memory * memory));
}
// Whether a kernel takes the call at all: by name, one that the rule leaves out may be asked for.  short_rows: offsets inside a tile are below 2^30 bytes.
bool takes(int kernel, int form, bool vectors, bool short_rows, int es) {
    if (kernel < 0 || kernel >= kExpKernels) return false;
    if (kernel == kExpAnyFew32) return es == 2 && short_rows && form != kGrad;
    return !needs_vectors(kernel) || (vectors && (es == 2 ? kVectors : kF32)[form][kernel].start > 0);
}
// form, and the sizes of the call; -1: 2^31 tiles or more
int pick(int form, bool vectors, bool short_rows, int es, int64_t rows, int64_t N, int64_t K, int experts) {
    const Cost(&costs)[kExpKernels] = (!vectors ? kAny : es == 2 ? kVectors : kF32)[form];
    auto tiles_of = [&](int k) { return form == kGrad ? gradient_tiles(k, N, K, experts) : product_tiles(k, rows, N, experts); };
    // (the rows of each expert are known on the device alone: half a tile left over for each that can have any)
    const double hit = rows < experts ? (double)rows : experts;
    auto seconds = [&](int k) {
        const double tm = kTile[k][0];
        if (form == kGrad) return predicted_us(costs[k], (double)tiles_of(k), std::fmax(1, (double)rows / experts * es / 128 + 0.5), (N * es | K * es) & 127, ((double)experts * N * K + (double)rows * (N + K)) * es);
        const double nx = rows / tm + 0.5 * hit > hit ? rows / tm + 0.5 * hit : hit;
        return predicted_us(costs[k], nx * tiles(N, kTile[k][1]), (double)tiles(K * es, 128), ((form == kNt ? K : N) * es) & 127, (hit * N * K + (double)rows * (N + K)) * es);
    };
    int best = -1;
    double least = 0;
    for (int k = 0; k < kExpKernels; ++k)
        if (takes(k, form, vectors, short_rows, es) && costs[k].start > 0 && launches(k, tiles_of(k)))
            if (const double t = seconds(k); best < 0 || t < least) {
                least = t;
                best = k;
            }
    // (the fewest tiles of those that have a work-group each, in several launches; of the gradient, eight times the eighth of each expert's)
    if (best < 0 && several_launches(tiles_of(kExpStaged128) + (form == kGrad ? 7 * experts : 0))) best = kExpStaged128;
    return best;
}
lcma_status check_sizes(const char *who, int64_t rows, int64_t N, int64_t K, int experts, int dtype) {
    if (!dtype_size(dtype)) return fail(LCMA_ERR_DTYPE, "%s: unknown dtype %d", who, dtype);
    if (rows < 0 || N < 0 || K < 0) return fail(LCMA_ERR_ARG, "%s: negative size", who);
    if (experts < 1) return fail(LCMA_ERR_ARG, "%s: experts = %d must be at least 1", who, experts);
    if (experts > kMaxExperts) return fail(LCMA_ERR_SHAPE, "%s: experts = %d is more than %d", who, experts, kMaxExperts);
    if (rows >= kRowLimit) return fail(LCMA_ERR_SHAPE, "%s: 2^31 rows or more", who);
    if (N >= kPitchLimit || K >= kPitchLimit || N * K > kMatrixLimit) return fail(LCMA_ERR_SHAPE, "%s: 2^29 columns or more, or a matrix of more than 2^44 elements", who);
    return LCMA_OK;
}
lcma_status check_pitch(const char *who, int64_t ld, int64_t row) {
    if (ld < row) return fail(LCMA_ERR_ARG, "%s: leading dimension smaller than the row", who);
    if (ld >= kPitchLimit) return fail(LCMA_ERR_SHAPE, "%s: leading dimension of 2^29 or more", who);
    return LCMA_OK;
}

} // namespace

extern "C" lcma_status lcma_gemm_experts(int b_layout, int64_t rows, int64_t N, int64_t K, int experts, const int32_t *offsets, const void *A, int64_t lda, const void *B,
                                         void *C, int64_t ldc, lcma_dtype dtype, void *stream) {
    const char *who = "lcma_gemm_experts";
    if (b_layout != 0 && b_layout != 2) return fail(LCMA_ERR_ARG, "%s: b_layout = %d must be 0 (K x N) or 2 (N x K)", who, b_layout);
    if (const lcma_status st = check_sizes(who, rows, N, K, experts, dtype)) return st;
    if (rows == 0 || N == 0) return LCMA_OK;
    if (!offsets || !C || (K && (!A || !B))) return fail(LCMA_ERR_ARG, "%s: null pointer", who);
    if (const lcma_status st = check_pitch(who, lda, K)) return st;
    if (const lcma_status st = check_pitch(who, ldc, N)) return st;
    const int es = dtype_size(dtype);
    if (((uintptr_t)A | (uintptr_t)B | (uintptr_t)C) % es || ((uintptr_t)offsets & 3))
        return fail(LCMA_ERR_ARG, "%s: matrices must have the alignment of their elements, offsets 4-byte alignment", who);
    const int64_t c_bytes = span(rows, ldc, N, es);
    if (touch(C, c_bytes, A, span(rows, lda, K, es)) || touch(C, c_bytes, B, experts * N * K * es) || touch(C, c_bytes, offsets, ((int64_t)experts + 1) * 4))
        return fail(LCMA_ERR_ARG, "%s: C overlaps an operand", who);
    ExpertsGemmParams p;
    std::memset(&p, 0, sizeof p);
    p.A = (const char *)A;
    p.B = (const char *)B;
    p.C = (char *)C;
    p.offsets = offsets;
    p.lda_b = lda * es;
    p.ldb_b = (b_layout ? K : N) * es;
    p.ldc_b = ldc * es;
    p.expert_b = N * K * es;
    p.rows = (int32_t)rows;
    p.N = (int32_t)N;
    p.K = (int32_t)K;
    p.experts = experts;
    p.panel = 8;
    const bool short_rows = K > 0 && p.lda_b <= kShortRow && p.ldb_b <= kShortRow, vectors = short_rows && whole_vectors(es, A, p.lda_b, B, p.ldb_b, K * es);
    const int form = b_layout ? kNt : kNn;
    int kernel = tuning_experts_kernel();
    if (!takes(kernel, form, vectors, short_rows, es) || !launches(kernel, product_tiles(kernel, rows, N, experts))) kernel = pick(form, vectors, short_rows, es, rows, N, K, experts);
    if (kernel < 0) return fail(LCMA_ERR_SHAPE, "%s: 2^31 tiles or more", who);
    p.nz = (int32_t)tiles(N, kTile[kernel][1]);
    if (const int err = launch(p, form, kernel, dtype, product_tiles(kernel, rows, N, experts), 8, stream))
        return fail(LCMA_ERR_HIP, "%s: launch failed with HIP error %d", who, err);
    return LCMA_OK;
}

extern "C" lcma_status lcma_gemm_experts_grad(int64_t rows, int64_t N, int64_t K, int experts, const int32_t *offsets, const void *dC, int64_t lddc, const void *A, int64_t lda,
                                              void *dW, lcma_dtype dtype, void *stream) {
    const char *who = "lcma_gemm_experts_grad";
    if (const lcma_status st = check_sizes(who, rows, N, K, experts, dtype)) return st;
    if (N == 0 || K == 0) return LCMA_OK;
    if (!offsets || !dW || (rows && (!dC || !A))) return fail(LCMA_ERR_ARG, "%s: null pointer", who);
    if (const lcma_status st = check_pitch(who, lddc, N)) return st;
    if (const lcma_status st = check_pitch(who, lda, K)) return st;
    const int es = dtype_size(dtype);
    if (((uintptr_t)A | (uintptr_t)dC | (uintptr_t)dW) % es || ((uintptr_t)offsets & 3))
        return fail(LCMA_ERR_ARG, "%s: matrices must have the alignment of their elements, offsets 4-byte alignment", who);
    const int64_t w_bytes = experts * N * K * es;
    if (touch(dW, w_bytes, dC, span(rows, lddc, N, es)) || touch(dW, w_bytes, A, span(rows, lda, K, es)) || touch(dW, w_bytes, offsets, ((int64_t)experts + 1) * 4))
        return fail(LCMA_ERR_ARG, "%s: dW overlaps an operand", who);
    ExpertsGemmParams p;
    std::memset(&p, 0, sizeof p);
    p.A = (const char *)dC;
    p.B = (const char *)A;
    p.C = (char *)dW;
    p.offsets = offsets;
    p.lda_b = lddc * es;
    p.ldb_b = lda * es;
    p.ldc_b = K * es;
    p.expert_b = N * K * es;
    p.rows = (int32_t)rows;
    p.M = (int32_t)N;
    p.N = (int32_t)K;
    p.experts = experts;
    p.panel = 8;
    p.stream = !(((uintptr_t)dW | (uint64_t)p.ldc_b) & 127); // (rows of whole lines, which a wave's store, or two waves' at the same time, fill; lines filled part by part cost up to twice the time instead)
    p.lines = rows <= (int64_t)512 * experts; // (512 rows an expert: 88 -> 82 us at 2048 x 4096, 1024: 141 -> 145)
    const bool short_rows = p.lda_b <= kShortRow && p.ldb_b <= kShortRow, vectors = short_rows && whole_vectors(es, dC, p.lda_b, A, p.ldb_b, 0);
    int kernel = tuning_experts_kernel();
    if (!takes(kernel, kGrad, vectors, short_rows, es) || !launches(kernel, gradient_tiles(kernel, N, K, experts))) kernel = pick(kGrad, vectors, short_rows, es, rows, N, K, experts);
    if (kernel < 0) return fail(LCMA_ERR_SHAPE, "%s: 2^31 tiles or more", who);
    p.nx = (int32_t)tiles(N, kTile[kernel][0]);
    p.nz = (int32_t)tiles(K, kTile[kernel][1]);
    // (how the kernels deal out tiles, and what it measured: exp_gradient_tile)
    const int64_t of = (int64_t)p.nx * p.nz, all = gradient_tiles(kernel, N, K, experts), few = p.nx < p.nz ? p.nx : p.nz, many = p.nx < p.nz ? p.nz : p.nx;
    p.by_expert = es == 2 && (kernel == kExpRing64 || kernel == kExpRing64x128) && of < 64 && few >= 3 && many <= 4 * few;
    if (const int err = launch(p, kGrad, kernel, dtype, all, ((p.by_expert ? all : of) + 7) / 8 * 8, stream))
        return fail(LCMA_ERR_HIP, "%s: launch failed with HIP error %d", who, err);
    return LCMA_OK;
}

namespace {

// dY null: forward, Y from X; else Y is dX.
lcma_status gated(const char *who, int64_t rows, int64_t F, const void *dY, int64_t lddy, const void *X, int64_t ldx, void *Y, int64_t ldy, int dtype, bool back, void *stream) {
    const int es = dtype_size(dtype);
    if (!es) return fail(LCMA_ERR_DTYPE, "%s: unknown dtype %d", who, dtype);
    if (rows < 0 || F < 0) return fail(LCMA_ERR_ARG, "%s: negative size", who);
    if (rows >= kRowLimit) return fail(LCMA_ERR_SHAPE, "%s: 2^31 rows or more", who);
    if (F >= kPitchLimit / 8) return fail(LCMA_ERR_SHAPE, "%s: a row is too long", who);
    if (rows == 0 || F == 0) return LCMA_OK;
    if (!X || !Y || (back && !dY)) return fail(LCMA_ERR_ARG, "%s: null pointer", who);
    const int64_t width = back ? 2 * F : F;
    if (ldx < 2 * F || ldy < width || (back && lddy < F)) return fail(LCMA_ERR_ARG, "%s: leading dimension smaller than the row", who);
    if (ldx >= kPitchLimit || ldy >= kPitchLimit || (back && lddy >= kPitchLimit)) return fail(LCMA_ERR_SHAPE, "%s: leading dimension of 2^29 or more", who);
    if (((uintptr_t)X | (uintptr_t)Y | (uintptr_t)dY) % es) return fail(LCMA_ERR_ARG, "%s: rows must have the alignment of their elements", who);
    const int64_t y_bytes = span(rows, ldy, width, es);
    if (touch(Y, y_bytes, X, span(rows, ldx, 2 * F, es)) || (back && touch(Y, y_bytes, dY, span(rows, lddy, F, es)))) return fail(LCMA_ERR_ARG, "%s: the result overlaps an input", who);
    GatedParams p;
    std::memset(&p, 0, sizeof p);
    p.X = (const char *)X;
    p.dY = (const char *)dY;
    p.Y = (char *)Y;
    p.ldx_b = ldx * es;
    p.lddy_b = lddy * es;
    p.ldy_b = ldy * es;
    p.rows = (int32_t)rows;
    p.F = (int32_t)F;
    p.stream = rows * width * es >= (int64_t)64 << 20; // (a quarter of the Infinity Cache written)
    const int64_t vectors = (F + 7) / 8;
    while (p.lane_shift < 8 && ((int64_t)1 << p.lane_shift) < vectors) ++p.lane_shift;
    const int64_t per = 256 >> p.lane_shift, gx = (rows + per - 1) / per, gy = tiles(vectors, (int64_t)1 << p.lane_shift);
    const int64_t most = 1 << 20; // (work-groups along x; each then takes several groups of rows)
    if (const int err = lcma_launch_gated(&p, dtype, back, (int)(gx < most ? gx : most), (int)gy, stream)) return fail(LCMA_ERR_HIP, "%s: launch failed with HIP error %d", who, err);
    return LCMA_OK;
}

} // namespace

extern "C" lcma_status lcma_gated_silu(int64_t rows, int64_t F, const void *X, int64_t ldx, void *Y, int64_t ldy, lcma_dtype dtype, void *stream) {
    return gated("lcma_gated_silu", rows, F, nullptr, 0, X, ldx, Y, ldy, dtype, false, stream);
}

extern "C" lcma_status lcma_gated_silu_grad(int64_t rows, int64_t F, const void *dY, int64_t lddy, const void *X, int64_t ldx, void *dX, int64_t lddx, lcma_dtype dtype,
                                            void *stream) {
    return gated("lcma_gated_silu_grad", rows, F, dY, lddy, X, ldx, dX, lddx, dtype, true, stream);
}
