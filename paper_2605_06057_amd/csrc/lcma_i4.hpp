// C = X W^T (+ bias) with weights of 4 bits for gfx950: W[n][k] = (u[n][k] - 8) S[n][k / G], codes u of 0 .. 15, a scale (fp32) for every G = 32, 64 or 128 columns of a row.
// X and C are bf16, fp16 or fp32; sums in fp32, one rounding.  With offsets the rows of X are in groups, group e times the weights of expert e.
//
// Weights are laid out once, in the order in which a wave takes them: blocks of 16 rows x 128 columns, those of 16 rows one behind the other, so that a wave reads
// memory from front to back.  A block is 1024 bytes of codes, 16 for every lane (row lane % 16; four dwords, dword j the columns 32 j + 8 (lane / 16) .. + 7, which are what
// the lane holds of a 16x16x32 instruction), and then the scales of its groups, 16 rows each.  Column i of the eight is nibble i / 2 + 4 (i % 2): shifted to place,
// the nibbles p and p + 4 are the two halves of a register.
//
// A code becomes a 16-bit float by its bits alone: u under the exponent of one is 1 + u / 16 = (24 + q) / 16 with q = u - 8, exactly, in bf16 and fp16: a shift and an
// and-or for two codes.  The 1.5 too much comes off as a sum of its own, of -1.5 x over the same columns, on the matrix pipe too, which the sum of a group starts with.  The group's
// sum is then 1/16 of sum q x in fp32 and is added to the row's times 16 S.  (What that costs: the terms are up to 1.94 x where q x / 16 is up to 0.5 x, so roundings
// of the fp32 sums count about eight times: 2^-21 of sum |x|, where C's own rounding is 2^-9 or 2^-12.)  fp32 activations are three bf16 numbers, whose sum is the value.
#pragma once
#include "lcma_i8.hpp"

namespace lcma {

// Types of the multiplication: bits of 1.0 twice, of -1.5 twice, where a nibble goes.
template <class T> struct I4Type {
    using Mul = BF16;
    static constexpr uint32_t ONE = 0x3F803F80u, MINUS = 0xBFC0BFC0u, MASK = 0x00780078u;
    static constexpr int UP = 3;
    static constexpr int PARTS = T::ES == 4 ? 3 : 1;
};
template <> struct I4Type<F16> {
    using Mul = F16;
    static constexpr uint32_t ONE = 0x3C003C00u, MINUS = 0xBE00BE00u, MASK = 0x03C003C0u;
    static constexpr int UP = 6, PARTS = 1;
};
template <class T> LCMA_DEV u32x4 i4_widened(uint32_t v) {
    using I = I4Type<T>;
    u32x4 r;
#pragma unroll
    for (int p = 0; p < 4; ++p) r[p] = ((I::UP >= 4 * p ? v << (I::UP - 4 * p) : v >> (4 * p - I::UP)) & I::MASK) | I::ONE;
    return r;
}

// WN x WK waves: the first along N, NB blocks of rows each, the others along K, a block of columns to a wave in turn.  MT x 16 rows of X, chunks of KC blocks of columns of
// them in LDS.  Rows past the tile's are whatever is in LDS: their sums are dropped.
template <class T, int G, int MT, int NB, int WN, int WK, int KC> struct I4Gemm {
    using I = I4Type<T>;
    using Mul = typename I::Mul;
    using Frag = typename Mma16<Mul>::frag;
    static constexpr int NT = 64 * WN * WK, TM = 16 * MT, TN = 16 * NB * WN, GROUPS = 128 / G, BLOCK = 1024 + GROUPS * 64;
    static constexpr int PITCH = KC * 256 + 16, PART = TM * PITCH; // (16: 16 rows at one column meet different banks)
    static constexpr int SUMS = (WK - 1) * WN * NB * MT * 1024, X_BYTES = I::PARTS * PART, LDS_BYTES = SUMS > X_BYTES ? SUMS : X_BYTES;
    static_assert(LDS_BYTES <= 160 * 1024, "LDS budget of one CU");

    // Columns k .. k + 7 of a row of X as the parts that are multiplied; zeros from K on.
    static LCMA_DEV void stage(const char *row, int k, int K, LCMA_LDS char *to) {
        constexpr int ES = T::ES;
        if constexpr (ES == 2) {
            u32x4 v = {0, 0, 0, 0};
            if (k + 8 <= K) __builtin_memcpy(&v, row + (int64_t)k * 2, 16);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (k + i < K) v[i / 2] |= (uint32_t)((const uint16_t *)row)[k + i] << (i & 1) * 16;
            *(LCMA_LDS u32x4 *)to = v;
        } else {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
            if (k + 8 <= K) __builtin_memcpy(v, row + (int64_t)k * 4, 32);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (k + i < K) v[i] = ((const float *)row)[k + i];
#pragma unroll
            for (int part = 0; part < 3; ++part) { // the upper 8 bits of what is left, twice, and the rest: each exact
                u32x4 w;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t top = __builtin_bit_cast(uint32_t, v[i]) & 0xffff0000u;
                    if (i & 1) w[i / 2] |= top;
                    else w[i / 2] = top >> 16;
                    v[i] -= __builtin_bit_cast(float, top);
                }
                *(LCMA_LDS u32x4 *)(to + part * PART) = w;
            }
        }
    }

    struct Block {
        u32x4 codes;
        f32x4 scales[GROUPS];
    };
    static LCMA_DEV void fetch(const char *at, Block &b) { // at: of the block
        const int lane = threadIdx.x & 63;
        b.codes = *(const u32x4 *)(at + lane * 16);
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) b.scales[g] = *(const f32x4 *)(at + 1024 + g * 64 + (lane >> 4) * 16);
    }

    static LCMA_DEV void run(const I4GemmParams &p, LCMA_LDS char *lds) {
        const I8Rows<TM, I4GemmParams> groups(p);
        i8_zero_behind<T>(p, groups.behind, gridDim.x, NT);
        const int nx = groups.tiles, jobs = nx * p.nz, per = (jobs + 7) / 8;
        const int job = (blockIdx.x & 7) * per + (blockIdx.x >> 3); // an eighth of the tiles to every XCD, row tiles that share weights next to each other
        if ((int)(blockIdx.x >> 3) >= per || job >= jobs) return;
        int x, z;
        i8_tile_of_job(nx, p.nz, p.panel, job, x, z);
        const I8Place at = groups.place(p, x);
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = w / WN, wn = w % WN, m = lane & 15, kb = lane >> 4;
        const int first = (z * WN + wn) * NB, all = (p.N + 15) / 16; // blocks of rows
        const char *q[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) q[b] = p.Q + at.expert * p.expert_q + (int64_t)(first + b < all ? first + b : all - 1) * p.blocks * BLOCK; // (past the last: the last again, dropped)
        f32x4 acc[NB][MT];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        const Frag minus = __builtin_bit_cast(Frag, u32x4{I::MINUS, I::MINUS, I::MINUS, I::MINUS});
        for (int c0 = 0; c0 < p.blocks; c0 += KC) {
            const int chunk = p.blocks - c0 < KC ? p.blocks - c0 : KC;
            if (c0) __syncthreads(); // all have read the chunk before
            for (int i = threadIdx.x; i < at.rows * chunk * 16; i += NT) {
                const int row = i / (chunk * 16), v = i % (chunk * 16);
                stage(p.X + (int64_t)(at.row0 + row) * p.ldx_b, c0 * 128 + v * 8, p.K, lds + row * PITCH + v * 16);
            }
            __syncthreads();
            for (int y = wk; y < chunk; y += WK) {
                Block blk[NB];
#pragma unroll
                for (int b = 0; b < NB; ++b) fetch(q[b] + (int64_t)(c0 + y) * BLOCK, blk[b]);
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    Frag xf[4 / GROUPS][MT][I::PARTS];
                    f32x4 off[MT], sum[NB][MT];
#pragma unroll
                    for (int j = 0; j < 4 / GROUPS; ++j)
#pragma unroll
                        for (int i = 0; i < MT; ++i)
#pragma unroll
                            for (int part = 0; part < I::PARTS; ++part)
                                xf[j][i][part] = __builtin_bit_cast(
                                    Frag, *(const LCMA_LDS u32x4 *)(lds + part * PART + (i * 16 + m) * PITCH + y * 256 + (g * (4 / GROUPS) + j) * 64 + kb * 16));
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        off[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int j = 0; j < 4 / GROUPS; ++j)
#pragma unroll
                            for (int part = 0; part < I::PARTS; ++part) off[i] = Mma16<Mul>::run(minus, xf[j][i][part], off[i]);
                    }
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
#pragma unroll
                        for (int i = 0; i < MT; ++i) sum[b][i] = off[i];
#pragma unroll
                        for (int j = 0; j < 4 / GROUPS; ++j) {
                            const Frag wf = __builtin_bit_cast(Frag, i4_widened<T>(blk[b].codes[g * (4 / GROUPS) + j]));
#pragma unroll
                            for (int i = 0; i < MT; ++i)
#pragma unroll
                                for (int part = 0; part < I::PARTS; ++part) sum[b][i] = Mma16<Mul>::run(wf, xf[j][i][part], sum[b][i]);
                        }
#pragma unroll
                        for (int i = 0; i < MT; ++i)
#pragma unroll
                            for (int v = 0; v < 4; ++v) acc[b][i][v] = __builtin_fmaf(sum[b][i][v], blk[b].scales[g][v], acc[b][i][v]);
                    }
                }
            }
        }
        if constexpr (WK > 1) { // the sums of the waves along K, in ascending order
            __syncthreads();
            LCMA_LDS f32x4 *sums = (LCMA_LDS f32x4 *)lds;
            if (wk)
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < MT; ++i) sums[((((wk - 1) * WN + wn) * NB + b) * MT + i) * 64 + lane] = acc[b][i];
            __syncthreads();
            if (wk) return;
#pragma unroll
            for (int k = 1; k < WK; ++k)
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[b][i] += sums[((((k - 1) * WN + wn) * NB + b) * MT + i) * 64 + lane];
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int col = (first + b) * 16 + kb * 4;
            if (col >= p.N) continue;
            f32x4 bias = {0.f, 0.f, 0.f, 0.f};
            if (p.bias) bias = i8_four(p.bias + (int64_t)at.expert * p.N, col, p.N);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const int row = i * 16 + m;
                if (row < at.rows) i8_store4<T>(p.C + ((int64_t)(at.row0 + row) * p.ldc + col) * T::ES, acc[b][i] + bias, p.N - col);
            }
        }
    }
};

} // namespace lcma
