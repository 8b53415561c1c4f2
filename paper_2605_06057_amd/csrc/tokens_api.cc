// Host side of the tokens' way to their experts and back: argument checks, launches.
#include "experts_host.h"

#include <cstring>

extern "C" int lcma_launch_tokens_sort(const lcma::TokensSortParams *p, void *stream);
extern "C" int lcma_launch_tokens_dispatch(const lcma::TokensRowsParams *p, int dtype, int gx, int gy, void *stream);
extern "C" int lcma_launch_tokens_combine(const lcma::TokensRowsParams *p, int dtype, int gx, int gy, void *stream);
extern "C" int lcma_launch_tokens_combine_grad(const lcma::TokensRowsParams *p, int dtype, int wave, void *stream);

using namespace lcma;

namespace {

bool sort_range(int64_t tokens, int top_k, int experts) {
    return tokens >= 0 && top_k >= 1 && experts >= 1 && experts <= kMaxExperts && tokens < kRowLimit && tokens * top_k < kRowLimit;
}

// What the three calls that move rows check alike.  wide: rows of tokens, long: rows in expert order.
lcma_status check_rows(const char *who, int64_t tokens, int top_k, int64_t H, const void *wide, int64_t ldw, const void *tall, int64_t ldt, int dtype,
                       const int32_t *position) {
    const int es = dtype_size(dtype);
    if (!es) return fail(LCMA_ERR_DTYPE, "%s: unknown dtype %d", who, dtype);
    if (tokens < 0 || H < 0) return fail(LCMA_ERR_ARG, "%s: negative size", who);
    if (top_k < 1) return fail(LCMA_ERR_ARG, "%s: top_k = %d must be at least 1", who, top_k);
    if (tokens >= kRowLimit || tokens * top_k >= kRowLimit) return fail(LCMA_ERR_SHAPE, "%s: 2^31 slots or more", who);
    if (tokens == 0) return LCMA_OK;
    if (!position || (H && (!wide || !tall))) return fail(LCMA_ERR_ARG, "%s: null pointer", who);
    if (ldw < H || ldt < H) return fail(LCMA_ERR_ARG, "%s: leading dimension smaller than the row", who);
    if (ldw >= kPitchLimit || ldt >= kPitchLimit || H >= kPitchLimit / 8) return fail(LCMA_ERR_SHAPE, "%s: a row is too long", who);
    if ((uintptr_t)wide % es || (uintptr_t)tall % es || ((uintptr_t)position & 3))
        return fail(LCMA_ERR_ARG, "%s: rows must have the alignment of their elements, positions 4-byte alignment", who);
    return LCMA_OK;
}
int64_t span(int64_t rows, int64_t ld, int64_t H, int dtype) { return rows > 0 ? ((rows - 1) * ld + H) * dtype_size(dtype) : 0; }

// Which rows pass the caches by (csrc/lcma_tokens.hip): those that are written from a quarter of the Infinity Cache on, those that are read from all of it on.
int streamed(int64_t written, int64_t read) { return (written >= ((int64_t)64 << 20) ? 1 : 0) | (read >= ((int64_t)256 << 20) ? 2 : 0); }

// Threads along a row: as many as it has 16-byte vectors, up to a work-group.
int lanes_of(int64_t vectors) {
    int s = 0;
    while (s < 8 && ((int64_t)1 << s) < vectors) ++s;
    return s;
}

} // namespace

extern "C" int64_t lcma_tokens_sort_workspace_bytes(int64_t tokens, int top_k, int experts) {
    if (!sort_range(tokens, top_k, experts)) return -1;
    const int64_t n = tokens * top_k, blocks = (n + kSortSlots - 1) / kSortSlots;
    return n > kSortOnce ? (blocks + 1) * (experts + 1) * 4 : 0;
}

extern "C" lcma_status lcma_tokens_sort(int64_t tokens, int top_k, int experts, const int32_t *ids, int32_t *order, int32_t *position, int32_t *offsets,
                                        void *workspace, int64_t workspace_bytes, void *stream) {
    const char *who = "lcma_tokens_sort";
    if (tokens < 0) return fail(LCMA_ERR_ARG, "%s: negative size", who);
    if (top_k < 1 || experts < 1) return fail(LCMA_ERR_ARG, "%s: top_k = %d and experts = %d must be at least 1", who, top_k, experts);
    if (!sort_range(tokens, top_k, experts))
        return fail(LCMA_ERR_SHAPE, "%s: more than %d experts, or 2^31 slots or more", who, kMaxExperts);
    const int64_t n = tokens * top_k, need = lcma_tokens_sort_workspace_bytes(tokens, top_k, experts);
    if (!offsets || (n && (!ids || !order || !position)) || (need && !workspace)) return fail(LCMA_ERR_ARG, "%s: null pointer", who);
    if (((uintptr_t)ids | (uintptr_t)order | (uintptr_t)position | (uintptr_t)offsets | (uintptr_t)workspace) & 3)
        return fail(LCMA_ERR_ARG, "%s: pointers must be 4-byte aligned", who);
    if (workspace_bytes < need)
        return fail(LCMA_ERR_ARG, "%s: the workspace holds %lld bytes, %lld are needed", who, (long long)workspace_bytes, (long long)need);
    const void *at[] = {ids, order, position, offsets, need ? workspace : nullptr};
    const int64_t bytes[] = {n * 4, n * 4, n * 4, ((int64_t)experts + 1) * 4, need};
    for (int i = 0; i < 5; ++i)
        for (int j = 0; j < i; ++j)
            if (touch(at[i], bytes[i], at[j], bytes[j])) return fail(LCMA_ERR_ARG, "%s: two operands overlap", who);
    TokensSortParams p;
    std::memset(&p, 0, sizeof p);
    p.ids = ids;
    p.order = order;
    p.position = position;
    p.offsets = offsets;
    p.counts = (int32_t *)workspace;
    p.n = (int32_t)n;
    p.experts = experts;
    p.blocks = (int32_t)((n + kSortSlots - 1) / kSortSlots);
    if (const int err = lcma_launch_tokens_sort(&p, stream)) return fail(LCMA_ERR_HIP, "%s: launch failed with HIP error %d", who, err);
    return LCMA_OK;
}

extern "C" lcma_status lcma_tokens_dispatch(int64_t tokens, int top_k, int64_t H, const void *X, int64_t ldx, lcma_dtype dtype, const int32_t *position,
                                            void *Y, int64_t ldy, void *stream) {
    const char *who = "lcma_tokens_dispatch";
    if (const lcma_status st = check_rows(who, tokens, top_k, H, X, ldx, Y, ldy, dtype, position)) return st;
    if (tokens == 0 || H == 0) return LCMA_OK;
    const int64_t n = tokens * top_k, y_bytes = span(n, ldy, H, dtype);
    if (touch(Y, y_bytes, X, span(tokens, ldx, H, dtype)) || touch(Y, y_bytes, position, n * 4)) return fail(LCMA_ERR_ARG, "%s: Y overlaps an input", who);
    const int es = dtype_size(dtype);
    const int64_t vectors = (H * es + 15) / 16;
    TokensRowsParams p;
    std::memset(&p, 0, sizeof p);
    p.X = X;
    p.Y = Y;
    p.position = position;
    p.ldx_b = ldx * es;
    p.ldy_b = ldy * es;
    p.tokens = (int32_t)tokens;
    p.top_k = top_k;
    p.H = (int32_t)H;
    p.lane_shift = lanes_of(vectors);
    p.stream = streamed(n * H * es, 0);
    const int64_t per = 256 >> p.lane_shift, gy = (vectors + (1 << p.lane_shift) - 1) >> p.lane_shift;
    if (gy > 65535) return fail(LCMA_ERR_SHAPE, "%s: a row is too long", who);
    if (const int err = lcma_launch_tokens_dispatch(&p, dtype, (int)((tokens + per - 1) / per), (int)gy, stream))
        return fail(LCMA_ERR_HIP, "%s: launch failed with HIP error %d", who, err);
    return LCMA_OK;
}

extern "C" lcma_status lcma_tokens_combine(int64_t tokens, int top_k, int64_t H, const void *Y, int64_t ldy, lcma_dtype dtype, const int32_t *position,
                                           const float *weights, void *X, int64_t ldx, void *stream) {
    const char *who = "lcma_tokens_combine";
    if (const lcma_status st = check_rows(who, tokens, top_k, H, X, ldx, Y, ldy, dtype, position)) return st;
    if (tokens == 0 || H == 0) return LCMA_OK;
    if ((uintptr_t)weights & 3) return fail(LCMA_ERR_ARG, "%s: weights must be 4-byte aligned", who);
    const int64_t n = tokens * top_k, x_bytes = span(tokens, ldx, H, dtype);
    if (touch(X, x_bytes, Y, span(n, ldy, H, dtype)) || touch(X, x_bytes, position, n * 4) || touch(X, x_bytes, weights, n * 4))
        return fail(LCMA_ERR_ARG, "%s: X overlaps an input", who);
    const int es = dtype_size(dtype);
    const int64_t vectors = (H * es + 15) / 16;
    TokensRowsParams p;
    std::memset(&p, 0, sizeof p);
    p.X = Y;
    p.Y = X;
    p.position = position;
    p.weights = weights;
    p.ldx_b = ldy * es;
    p.ldy_b = ldx * es;
    p.tokens = (int32_t)tokens;
    p.top_k = top_k;
    p.H = (int32_t)H;
    p.lane_shift = lanes_of((vectors + 1) / 2); // (a thread takes two)
    p.stream = streamed(tokens * H * es, n * H * es);
    const int64_t per = 256 >> p.lane_shift, gy = (vectors + (2 << p.lane_shift) - 1) >> (p.lane_shift + 1);
    if (gy > 65535) return fail(LCMA_ERR_SHAPE, "%s: a row is too long", who);
    if (const int err = lcma_launch_tokens_combine(&p, dtype, (int)((tokens + per - 1) / per), (int)gy, stream))
        return fail(LCMA_ERR_HIP, "%s: launch failed with HIP error %d", who, err);
    return LCMA_OK;
}

extern "C" lcma_status lcma_tokens_combine_grad(int64_t tokens, int top_k, int64_t H, const void *dX, int64_t lddx, const void *Y, int64_t ldy,
                                                lcma_dtype dtype, const int32_t *position, const float *weights, void *dY, int64_t lddy, float *dweights,
                                                void *stream) {
    const char *who = "lcma_tokens_combine_grad";
    if (const lcma_status st = check_rows(who, tokens, top_k, H, dX, lddx, Y, ldy, dtype, position)) return st;
    if (const lcma_status st = check_rows(who, tokens, top_k, H, dX, lddx, dY, lddy, dtype, position)) return st;
    if (tokens == 0) return LCMA_OK;
    if (!weights || !dweights) return fail(LCMA_ERR_ARG, "%s: null pointer", who);
    if (((uintptr_t)weights | (uintptr_t)dweights) & 3) return fail(LCMA_ERR_ARG, "%s: weights must be 4-byte aligned", who);
    const int64_t n = tokens * top_k, y_bytes = span(n, lddy, H, dtype);
    const void *in[] = {dX, Y, position, weights};
    const int64_t bytes[] = {span(tokens, lddx, H, dtype), span(n, ldy, H, dtype), n * 4, n * 4};
    for (int i = 0; i < 4; ++i)
        if (touch(dY, y_bytes, in[i], bytes[i]) || touch(dweights, n * 4, in[i], bytes[i])) return fail(LCMA_ERR_ARG, "%s: an output overlaps an input", who);
    if (touch(dY, y_bytes, dweights, n * 4)) return fail(LCMA_ERR_ARG, "%s: the outputs overlap", who);
    const int es = dtype_size(dtype);
    TokensRowsParams p;
    std::memset(&p, 0, sizeof p);
    p.X = Y;
    p.dX = dX;
    p.Y = dY;
    p.position = position;
    p.weights = weights;
    p.dW = dweights;
    p.ldx_b = ldy * es;
    p.lddx_b = lddx * es;
    p.ldy_b = lddy * es;
    p.tokens = (int32_t)tokens;
    p.top_k = top_k;
    p.H = (int32_t)H;
    p.stream = streamed(n * H * es, n * H * es);
    if (const int err = lcma_launch_tokens_combine_grad(&p, dtype, H * es <= 128 * 16, stream))
        return fail(LCMA_ERR_HIP, "%s: launch failed with HIP error %d", who, err);
    return LCMA_OK;
}
