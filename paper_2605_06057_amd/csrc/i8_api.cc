// Host side of the 8-bit-integer linear layer, alone and over experts: argument checks, launches.
#include "experts_host.h"

#include <cmath>
#include <cstring>

extern "C" int lcma_launch_i8_quantize(const lcma::I8QuantParams *p, int dtype, int gated, int threads, void *stream);
extern "C" int lcma_launch_i8_gemm(const lcma::I8GemmParams *p, int kernel, int dtype, int grid, void *stream);

using namespace lcma;

namespace {

const int64_t kMostK = 131071; // 128 * 128 * K below 2^31

int64_t pitch_of(int64_t K) { return (K + 127) / 128 * 128; }

lcma_status quantize(const char *who, int64_t rows, int64_t K, const void *X, int64_t ldx, int dtype, bool gated, int top_k, const int32_t *position,
                     void *Q, float *S, void *stream) {
    const int es = dtype_size(dtype);
    if (!es) return fail(LCMA_ERR_DTYPE, "%s: unknown dtype %d", who, dtype);
    if (rows < 0 || K < 0) return fail(LCMA_ERR_ARG, "%s: negative size", who);
    if (top_k < 1) return fail(LCMA_ERR_ARG, "%s: top_k = %d must be at least 1", who, top_k);
    if (K > kMostK) return fail(LCMA_ERR_SHAPE, "%s: K = %lld is more than %lld", who, (long long)K, (long long)kMostK);
    if (rows >= kRowLimit || rows * top_k >= kRowLimit) return fail(LCMA_ERR_SHAPE, "%s: 2^31 rows or more", who);
    if (rows == 0) return LCMA_OK;
    const int64_t width = gated ? 2 * K : K;
    if (!S || (K && (!X || !Q))) return fail(LCMA_ERR_ARG, "%s: null pointer", who);
    if (ldx < width) return fail(LCMA_ERR_ARG, "%s: leading dimension smaller than the row", who);
    if (ldx >= kPitchLimit) return fail(LCMA_ERR_SHAPE, "%s: leading dimension of 2^29 or more", who);
    if ((uintptr_t)X % es || ((uintptr_t)Q & 15) || ((uintptr_t)S & 3) || ((uintptr_t)position & 3))
        return fail(LCMA_ERR_ARG, "%s: X must have the alignment of its elements, Q 16-byte and S 4-byte alignment", who);
    const int64_t to = rows * top_k, x_bytes = ((rows - 1) * ldx + width) * es, q_bytes = to * pitch_of(K);
    if (touch(Q, q_bytes, X, x_bytes) || touch(S, to * 4, X, x_bytes) || touch(Q, q_bytes, S, to * 4) ||
        (position && (touch(Q, q_bytes, position, to * 4) || touch(S, to * 4, position, to * 4))))
        return fail(LCMA_ERR_ARG, "%s: an output overlaps another operand", who);
    I8QuantParams p;
    std::memset(&p, 0, sizeof p);
    p.X = X;
    p.Q = (int8_t *)Q;
    p.S = S;
    p.position = position;
    p.ldx_b = ldx * es;
    p.rows = (int32_t)rows;
    p.K = (int32_t)K;
    p.pitch = (int32_t)pitch_of(K);
    p.top_k = top_k;
    // as many threads as keep the row in registers
    const int threads = K <= 1024 ? 64 : K <= 4096 ? 256 : 1024;
    if (const int err = lcma_launch_i8_quantize(&p, dtype, gated, threads, stream)) return fail(LCMA_ERR_HIP, "%s: launch failed with HIP error %d", who, err);
    return LCMA_OK;
}

// What a kernel takes, in us: `start` once; for every round of one tile per compute unit `end` and, for every step of 128 k, `step` with all units at work (the
// chip's power and what the units share bound it then), `alone` with few; and no less than the bytes at `rate` GB/us take.  Fitted to 110 products and 90 over experts of
// random sizes (1 to 8192 rows, 8 to 128 experts, 64 to 28672 columns, K 64 to 14336) timed on every kernel: a single time is predicted within 8 to
// 15 % (root mean square; 13 to 18 % with fp32 results).  On 200 other sizes the kernel with the smallest prediction is 2.0 % slower than the fastest one on
// average, 17 % at worst; on 200 with fp32 results 1.8 % and 33 %.  Left out because they choose no better: four bytes instead of two for an element of C in fp32 (1.9 % and 33 %),
// the halves of tiles that a last round of 256 x 256 may have (2.0 to 2.2 %; a whole one is charged, which is 10 % too much there).
const struct Cost {
    int rows, cols;
    double start, alone, step, end, rate;
    bool in_turn; // one work-group per compute unit: rounds count; else several, which share it
} kCost[kI8Kernels] = {{16, 16, 3.3, 0.026, 0.051, 0.40, 9.5, false},  {32, 32, 2.8, 0.041, 0.107, 1.07, 8.3, false},   {64, 64, 2.55, 0.168, 0.195, 1.44, 7.0, false},
                       {64, 128, 2.5, 0.292, 0.362, 1.50, 7.1, false}, {128, 128, 1.1, 0.387, 0.586, 3.29, 9.8, true},   {128, 256, 1.3, 0.506, 0.961, 4.88, 7.8, true},
                       {256, 256, 2.0, 0.861, 1.41, 5.82, 6.5, true}};
double predicted_us(const Cost &k, int64_t rows, int64_t N, int64_t K, int experts) {
    // (the rows of each expert are known on the device alone: half a tile left over for each that can have any)
    const double hit = experts < rows ? experts : (double)rows, nz = (double)((N + k.cols - 1) / k.cols);
    double nx = (double)((rows + k.rows - 1) / k.rows);
    if (experts > 1) nx = (double)rows / k.rows + 0.5 * hit > hit ? (double)rows / k.rows + 0.5 * hit : hit;
    const double n = nx * nz / 256, steps = (double)((K + 127) / 128);
    const double bytes = hit * N * K + (double)rows * K + 2.0 * rows * N, memory = k.start + bytes / (k.rate * 1e6);
    const double whole = k.in_turn ? (double)(int64_t)n : n >= 1 ? n : 0, part = n - whole;
    const double t = k.start + whole * (steps * k.step + k.end) + (part > 0 ? steps * (k.alone + (k.step - k.alone) * part) + k.end : 0);
    return std::sqrt(std::sqrt(t * t * t * t + memory * memory * memory * memory));
}
bool walks(int kernel) { return kernel >= kI8Narrow; } // 256 work-groups walk through the tiles; the other kernels have one for every tile
// Tiles, at most: every group of rows may end in one of its own that is not full.
int64_t tiles_along_rows(int kernel, int64_t rows, int experts, bool grouped) {
    const int64_t tm = kCost[kernel].rows;
    return grouped ? rows / tm + (rows < experts ? rows : experts) : (rows + tm - 1) / tm;
}
int64_t tiles_along_columns(int kernel, int64_t N) { return (N + kCost[kernel].cols - 1) / kCost[kernel].cols; }
bool launches(int kernel, int64_t rows, int64_t N, int experts, bool grouped) {
    const int64_t jobs = tiles_along_rows(kernel, rows, experts, grouped) * tiles_along_columns(kernel, N);
    return walks(kernel) ? jobs < kRowLimit - 1024 : (jobs + 8) * 512 < kGridLimit / 2; // (numbers of tiles are 32-bit on the device)
}
// Of the kernels whose launch holds the tiles; -1: none does.
int pick(int64_t rows, int64_t N, int64_t K, int experts, bool grouped) {
    if (K == 0) // (nothing to multiply: the smallest tiles that any number of steps suits, as long as they are not too many)
        return launches(kI8Ring64, rows, N, experts, grouped) ? kI8Ring64 : launches(kI8PingPong, rows, N, experts, grouped) ? kI8PingPong : -1;
    if (const int forced = tuning_i8_kernel(); forced >= 0 && launches(forced, rows, N, experts, grouped)) return forced;
    int best = -1;
    double least = 0;
    for (int k = 0; k < kI8Kernels; ++k)
        if (const double t = predicted_us(kCost[k], rows, N, K, experts); launches(k, rows, N, experts, grouped) && (best < 0 || t < least)) {
            least = t;
            best = k;
        }
    return best;
}

lcma_status gemm(const char *who, int64_t rows, int64_t N, int64_t K, int experts, const int32_t *offsets, const void *Aq, const float *Sa,
                 const void *Wq, const float *Sw, const float *bias, void *C, int64_t ldc, int dtype, void *stream) {
    const int es = dtype_size(dtype);
    if (!es) return fail(LCMA_ERR_DTYPE, "%s: unknown dtype %d", who, dtype);
    if (rows < 0 || N < 0 || K < 0) return fail(LCMA_ERR_ARG, "%s: negative size", who);
    if (K > kMostK) return fail(LCMA_ERR_SHAPE, "%s: K = %lld is more than %lld", who, (long long)K, (long long)kMostK);
    if (rows >= kRowLimit || N >= kRowLimit) return fail(LCMA_ERR_SHAPE, "%s: 2^31 rows or columns or more", who);
    if (rows == 0 || N == 0) return LCMA_OK;
    if (!Sa || !Sw || !C || (K && (!Aq || !Wq))) return fail(LCMA_ERR_ARG, "%s: null pointer", who);
    if (ldc < N) return fail(LCMA_ERR_ARG, "%s: leading dimension smaller than the row", who);
    if (ldc >= kPitchLimit) return fail(LCMA_ERR_SHAPE, "%s: leading dimension of 2^29 or more", who);
    if ((((uintptr_t)Aq | (uintptr_t)Wq) & 15) || (((uintptr_t)Sa | (uintptr_t)Sw | (uintptr_t)bias | (uintptr_t)offsets) & 3) || (uintptr_t)C % es)
        return fail(LCMA_ERR_ARG, "%s: code matrices must be 16-byte aligned, scales, bias and offsets 4-byte aligned, C as its elements", who);
    const int64_t pitch = pitch_of(K), channels = experts * N, c_bytes = ((rows - 1) * ldc + N) * es;
    if (touch(C, c_bytes, Aq, rows * pitch) || touch(C, c_bytes, Wq, channels * pitch) || touch(C, c_bytes, Sa, rows * 4) ||
        touch(C, c_bytes, Sw, channels * 4) || (bias && touch(C, c_bytes, bias, channels * 4)) || (offsets && touch(C, c_bytes, offsets, (experts + 1) * 4)))
        return fail(LCMA_ERR_ARG, "%s: C overlaps an operand", who);
    I8GemmParams p;
    std::memset(&p, 0, sizeof p);
    p.A = (const int8_t *)Aq;
    p.W = (const int8_t *)Wq;
    p.SA = Sa;
    p.SW = Sw;
    p.bias = bias;
    p.C = C;
    p.offsets = offsets;
    p.ldc = ldc;
    p.rows = (int32_t)rows;
    p.N = (int32_t)N;
    p.pitch = (int32_t)pitch;
    p.experts = experts;
    p.steps = (int32_t)(pitch / 128);
    const int kernel = pick(rows, N, K, experts, offsets != nullptr);
    if (kernel < 0) return fail(LCMA_ERR_SHAPE, "%s: too many tiles for a launch", who);
    const int64_t nz = tiles_along_columns(kernel, N), jobs = tiles_along_rows(kernel, rows, experts, offsets != nullptr) * nz;
    p.nz = (int32_t)nz;
    p.panel = kernel <= kI8Few32 ? 1 : 8;
    const int grid = walks(kernel) ? 256 : (int)((jobs + 7) / 8 * 8);
    if (const int err = lcma_launch_i8_gemm(&p, kernel, dtype, grid, stream))
        return fail(LCMA_ERR_HIP, "%s: launch failed with HIP error %d", who, err);
    return LCMA_OK;
}

} // namespace

extern "C" int64_t lcma_i8_code_pitch(int64_t K) { return K < 0 ? -1 : pitch_of(K); }

extern "C" lcma_status lcma_i8_quantize(int64_t rows, int64_t K, const void *X, int64_t ldx, lcma_dtype dtype, int gated, void *Q, float *S, void *stream) {
    return quantize("lcma_i8_quantize", rows, K, X, ldx, dtype, gated != 0, 1, nullptr, Q, S, stream);
}

extern "C" lcma_status lcma_i8_quantize_dispatch(int64_t tokens, int64_t K, const void *X, int64_t ldx, lcma_dtype dtype, int top_k, const int32_t *position,
                                                 void *Q, float *S, void *stream) {
    if (tokens > 0 && !position) return fail(LCMA_ERR_ARG, "lcma_i8_quantize_dispatch: null pointer");
    return quantize("lcma_i8_quantize_dispatch", tokens, K, X, ldx, dtype, false, top_k, position, Q, S, stream);
}

extern "C" lcma_status lcma_i8_gemm_nt(int64_t M, int64_t N, int64_t K, const void *Aq, const float *Sa, const void *Wq, const float *Sw, const float *bias,
                                       void *C, int64_t ldc, lcma_dtype dtype, void *stream) {
    return gemm("lcma_i8_gemm_nt", M, N, K, 1, nullptr, Aq, Sa, Wq, Sw, bias, C, ldc, dtype, stream);
}

extern "C" lcma_status lcma_i8_gemm_experts(int64_t rows, int64_t N, int64_t K, int experts, const int32_t *offsets, const void *Aq, const float *Sa,
                                            const void *Wq, const float *Sw, const float *bias, void *C, int64_t ldc, lcma_dtype dtype, void *stream) {
    const char *who = "lcma_i8_gemm_experts";
    if (experts < 1) return fail(LCMA_ERR_ARG, "%s: experts = %d must be at least 1", who, experts);
    if (experts > kMaxExperts) return fail(LCMA_ERR_SHAPE, "%s: experts = %d is more than %d", who, experts, kMaxExperts);
    if (rows > 0 && N > 0 && !offsets) return fail(LCMA_ERR_ARG, "%s: null pointer", who);
    return gemm(who, rows, N, K, experts, offsets, Aq, Sa, Wq, Sw, bias, C, ldc, dtype, stream);
}
