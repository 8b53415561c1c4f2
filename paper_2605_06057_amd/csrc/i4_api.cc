// Host side of the linear layer with 4-bit weights, alone and over experts: argument checks, launches.
#include "experts_host.h"

#include <cmath>
#include <cstring>

extern "C" int lcma_launch_i4_prepare(const lcma::I4PrepareParams *p, int dtype, int grid, void *stream);
extern "C" int lcma_launch_i4_gemm(const lcma::I4GemmParams *p, int kernel, int group, int dtype, int grid, void *stream);

using namespace lcma;

namespace {

const int kTile[kI4Kernels][2] = {{16, 16}, {16, 32}, {16, 64}, {64, 64}}; // rows and columns of the kernels' tiles

bool group_fits(int group) { return group == 32 || group == 64 || group == 128; }
int64_t row_blocks(int64_t N) { return (N + 15) / 16; }
int64_t column_blocks(int64_t K) { return (K + 127) / 128; }
int64_t bytes_of(int64_t N, int64_t K, int group) { return row_blocks(N) * column_blocks(K) * i4_block_bytes(group); }

lcma_status check_weights(const char *who, int64_t N, int64_t K, int group, int experts) {
    if (N < 0 || K < 0) return fail(LCMA_ERR_ARG, "%s: negative size", who);
    if (!group_fits(group)) return fail(LCMA_ERR_ARG, "%s: group = %d must be 32, 64 or 128", who, group);
    if (experts < 1) return fail(LCMA_ERR_ARG, "%s: experts = %d must be at least 1", who, experts);
    if (experts > kMaxExperts) return fail(LCMA_ERR_SHAPE, "%s: experts = %d is more than %d", who, experts, kMaxExperts);
    if (N >= kPitchLimit || K >= kPitchLimit || N * K > kMatrixLimit) return fail(LCMA_ERR_SHAPE, "%s: 2^29 rows or columns or more, or a matrix of more than 2^44 elements", who);
    return LCMA_OK;
}

lcma_status prepare(const char *who, int experts, int64_t N, int64_t K, int group, const void *W, int64_t ldw, int64_t es, const float *S, int dtype, void *Wp, void *stream) {
    if (const lcma_status st = check_weights(who, N, K, group, experts)) return st;
    if (N == 0 || K == 0) return LCMA_OK;
    if (!W || !Wp || (dtype < 0 && !S)) return fail(LCMA_ERR_ARG, "%s: null pointer", who);
    if (ldw < K) return fail(LCMA_ERR_ARG, "%s: leading dimension smaller than the row", who);
    if (ldw >= kPitchLimit || N * ldw > kMatrixLimit) return fail(LCMA_ERR_SHAPE, "%s: leading dimension of 2^29 or more, or a matrix that spans more than 2^44 elements", who);
    if ((uintptr_t)W % es || ((uintptr_t)S & 3) || ((uintptr_t)Wp & 15)) return fail(LCMA_ERR_ARG, "%s: W must have the alignment of its elements, scales 4-byte and Wp 16-byte alignment", who);
    const int64_t q_bytes = experts * bytes_of(N, K, group), w_bytes = ((experts * N - 1) * ldw + K) * es, s_bytes = experts * N * ((K + group - 1) / group) * 4;
    if (touch(Wp, q_bytes, W, w_bytes) || (S && touch(Wp, q_bytes, S, s_bytes))) return fail(LCMA_ERR_ARG, "%s: Wp overlaps an input", who);
    I4PrepareParams p;
    std::memset(&p, 0, sizeof p);
    p.W = W;
    p.S = S;
    p.Q = (char *)Wp;
    p.ldw_b = ldw * es;
    p.expert_b = N * ldw * es;
    p.expert_q = bytes_of(N, K, group);
    p.N = (int32_t)N;
    p.K = (int32_t)K;
    p.group = group;
    p.experts = experts;
    const int64_t all = row_blocks(N) * experts, most = 1 << 16;
    if (const int err = lcma_launch_i4_prepare(&p, dtype, (int)(all < most ? all : most), stream)) return fail(LCMA_ERR_HIP, "%s: launch failed with HIP error %d", who, err);
    return LCMA_OK;
}

// Tiles, at most: every group of rows may end in one of its own that is not full.
int64_t tiles_of(int kernel, int64_t rows, int64_t N, int experts, bool grouped) {
    const int64_t tm = kTile[kernel][0], tn = kTile[kernel][1];
    return (grouped ? rows / tm + (rows < experts ? rows : experts) : (rows + tm - 1) / tm) * ((N + tn - 1) / tn);
}

// What a kernel takes, in us: `start`; a tile: `end`, `step` for every turn of its waves along K (fp32: 2.2 of them, three parts of X), `stage` for every byte of a column
// of the rows of X that go through LDS, 256 * `slots` tiles at a time; and no less than the bytes at `rate` GB/us take.  Fitted to 268 products, alone and over experts, of 1 to 1024 rows, timed on every
// kernel: a single time is predicted within 14 % (root mean square), the kernel with the smallest prediction is 1.3 % slower than the fastest one on average, 38 % at worst.
const struct Cost {
    int along_k; // waves
    double start, end, step, stage, rate, slots;
} kCost[kI4Kernels] = {{8, 2.69, 0.768, 0.318, 0.00298, 16.4, 0.903}, {4, 2.49, 0.998, 0.279, 0.00407, 5.32, 1.08}, {1, 2.56, 0.819, 0.215, 0.00677, 4.86, 1.67}, {2, 2.73, 0.738, 0.67, 0.00475, 4.63, 0.831}};
double predicted_us(int kernel, int64_t rows, int64_t N, int64_t K, int group, int experts, bool grouped, int es) {
    const Cost &c = kCost[kernel];
    const double tm = kTile[kernel][0], hit = rows < experts ? (double)rows : experts, blocks = (double)column_blocks(K);
    // (the rows of each expert are known on the device alone: half a tile left over for each that can have any)
    double nx = std::ceil(rows / tm);
    if (grouped) nx = rows / tm + 0.5 * hit > hit ? rows / tm + 0.5 * hit : hit;
    const double nz = std::ceil((double)N / kTile[kernel][1]), per = rows / hit < tm ? rows / hit : tm, n = nx * nz / 256 / c.slots;
    const double tile = c.end + std::ceil(blocks / c.along_k) * c.step * (es == 4 ? 2.2 : 1) + blocks * per * c.stage * es;
    const double bytes = hit * N * (0.5 * K + 4.0 * K / group) + 2.0 * rows * (N + K);
    const double t = c.start + tile * (n > 1 ? n : 1), memory = c.start + bytes / (c.rate * 1e6);
    return std::sqrt(std::sqrt(t * t * t * t + memory * memory * memory * memory));
}

lcma_status gemm(const char *who, int64_t rows, int64_t N, int64_t K, int group, int experts, const int32_t *offsets, const void *X, int64_t ldx, const void *Wp, const float *bias,
                 void *C, int64_t ldc, int dtype, void *stream) {
    const int es = dtype_size(dtype);
    if (!es) return fail(LCMA_ERR_DTYPE, "%s: unknown dtype %d", who, dtype);
    if (rows < 0) return fail(LCMA_ERR_ARG, "%s: negative size", who);
    if (const lcma_status st = check_weights(who, N, K, group, experts)) return st;
    if (rows >= kRowLimit) return fail(LCMA_ERR_SHAPE, "%s: 2^31 rows or more", who);
    if (rows == 0 || N == 0) return LCMA_OK;
    if (!C || (K && (!X || !Wp))) return fail(LCMA_ERR_ARG, "%s: null pointer", who);
    if (ldx < K || ldc < N) return fail(LCMA_ERR_ARG, "%s: leading dimension smaller than the row", who);
    if (ldx >= kPitchLimit || ldc >= kPitchLimit) return fail(LCMA_ERR_SHAPE, "%s: leading dimension of 2^29 or more", who);
    if (((uintptr_t)X | (uintptr_t)C) % es || ((uintptr_t)Wp & 15) || (((uintptr_t)bias | (uintptr_t)offsets) & 3))
        return fail(LCMA_ERR_ARG, "%s: X and C must have the alignment of their elements, Wp 16-byte alignment, bias and offsets 4-byte alignment", who);
    const int64_t c_bytes = ((rows - 1) * ldc + N) * es, x_bytes = K ? ((rows - 1) * ldx + K) * es : 0;
    if (touch(C, c_bytes, X, x_bytes) || touch(C, c_bytes, Wp, experts * bytes_of(N, K, group)) || (bias && touch(C, c_bytes, bias, experts * N * 4)) ||
        (offsets && touch(C, c_bytes, offsets, ((int64_t)experts + 1) * 4)))
        return fail(LCMA_ERR_ARG, "%s: C overlaps an operand", who);
    I4GemmParams p;
    std::memset(&p, 0, sizeof p);
    p.X = (const char *)X;
    p.Q = (const char *)Wp;
    p.bias = bias;
    p.C = (char *)C;
    p.offsets = offsets;
    p.ldx_b = ldx * es;
    p.ldc = ldc;
    p.expert_q = bytes_of(N, K, group);
    p.rows = (int32_t)rows;
    p.N = (int32_t)N;
    p.K = (int32_t)K;
    p.experts = experts;
    p.blocks = (int32_t)column_blocks(K);
    p.panel = 1;
    auto fits = [&](int k, bool once) {
        const int64_t jobs = tiles_of(k, rows, N, experts, offsets != nullptr);
        return (es == 2 || k != kI4Rows64) && (once ? one_launch(jobs) : several_launches(jobs));
    };
    int kernel = tuning_i4_kernel();
    if (kernel < 0 || !fits(kernel, true)) kernel = -1;
    for (bool once : {true, false}) {
        if (kernel >= 0) break;
        double least = 0;
        for (int k = 0; k < kI4Kernels; ++k)
            if (const double t = predicted_us(k, rows, N, K, group, experts, offsets != nullptr, es); fits(k, once) && (kernel < 0 || t < least)) {
                least = t;
                kernel = k;
            }
    }
    if (kernel < 0) return fail(LCMA_ERR_SHAPE, "%s: 2^31 tiles or more", who);
    const int64_t jobs = tiles_of(kernel, rows, N, experts, offsets != nullptr), eighth = (jobs + 7) / 8, most = one_launch(jobs) ? eighth : kLaunchEighth;
    p.nz = (int32_t)((N + kTile[kernel][1] - 1) / kTile[kernel][1]);
    for (int64_t from = 0; from < eighth; from += most) {
        p.from = (int32_t)from;
        if (const int err = lcma_launch_i4_gemm(&p, kernel, group, dtype, (int)((eighth - from < most ? eighth - from : most) * 8), stream))
            return fail(LCMA_ERR_HIP, "%s: launch failed with HIP error %d", who, err);
    }
    return LCMA_OK;
}

} // namespace

extern "C" int64_t lcma_i4_prepared_bytes(int64_t N, int64_t K, int group) {
    return N < 0 || K < 0 || N >= kPitchLimit || K >= kPitchLimit || N * K > kMatrixLimit || !group_fits(group) ? -1 : bytes_of(N, K, group);
}

extern "C" lcma_status lcma_i4_quantize(int experts, int64_t N, int64_t K, int group, const void *W, int64_t ldw, lcma_dtype dtype, void *Wp, void *stream) {
    const int es = dtype_size(dtype);
    if (!es) return fail(LCMA_ERR_DTYPE, "lcma_i4_quantize: unknown dtype %d", (int)dtype);
    return prepare("lcma_i4_quantize", experts, N, K, group, W, ldw, es, nullptr, dtype, Wp, stream);
}

extern "C" lcma_status lcma_i4_prepare(int experts, int64_t N, int64_t K, int group, const int8_t *codes, const float *scales, void *Wp, void *stream) {
    return prepare("lcma_i4_prepare", experts, N, K, group, codes, K, 1, scales, -1, Wp, stream);
}

extern "C" lcma_status lcma_i4_gemm_nt(int64_t M, int64_t N, int64_t K, int group, const void *X, int64_t ldx, const void *Wp, const float *bias, void *C, int64_t ldc,
                                       lcma_dtype dtype, void *stream) {
    return gemm("lcma_i4_gemm_nt", M, N, K, group, 1, nullptr, X, ldx, Wp, bias, C, ldc, dtype, stream);
}

extern "C" lcma_status lcma_i4_gemm_experts(int64_t rows, int64_t N, int64_t K, int group, int experts, const int32_t *offsets, const void *X, int64_t ldx, const void *Wp,
                                            const float *bias, void *C, int64_t ldc, lcma_dtype dtype, void *stream) {
    if (rows > 0 && N > 0 && !offsets && experts >= 1 && experts <= kMaxExperts) return fail(LCMA_ERR_ARG, "lcma_i4_gemm_experts: null pointer");
    return gemm("lcma_i4_gemm_experts", rows, N, K, group, experts, offsets, X, ldx, Wp, bias, C, ldc, dtype, stream);
}
