// C = X W^T (+ bias) with weights of 4 bits for gfx950: W[n][k] = (u[n][k] - 8) S[n][k / G], codes u of 0 .. 15, a scale (fp32) for every G = 32, 64 or 128 columns of a row.
// X and C are bf16, fp16 or fp32; sums in fp32, one rounding.  With offsets the rows of X are in groups, group e times the weights of expert e.
//
// Weights are laid out once, in the order in which a wave takes them: blocks of 16 rows x 128 columns, those of 16 rows one behind the other, so that a wave reads
// memory from front to back.  A block is 1024 bytes of codes, 16 for every lane (row lane % 16; four dwords, dword j the columns 32 j + 8 (lane / 16) .. + 7, which are what
// the lane holds of a 16x16x32 instruction), and then the scales of every row's groups.  Column i of the eight is nibble i / 2 + 4 (i % 2): shifted to place,
// the nibbles p and p + 4 are the two halves of a register.
//
// A code becomes a 16-bit float by its bits alone: u under the exponent of one is 1 + u / 16 = (24 + q) / 16 with q = u - 8, exactly, in bf16 and fp16: a shift and an
// and-or for two codes.  The 1.5 too much comes off as a sum of its own, of -1.5 x over the same columns, on the matrix pipe too, which the sum of a group starts with.  The group's
// sum is then 1/16 of sum q x in fp32 and is added to the row's times 16 S.  (What that costs: the terms are up to 1.94 x and the sums on
// the way up to 2 sum |x|, where q x / 16 is up to 0.5 x.  2 group additions, each off by up to 2^-23 of such a sum, times 16 S: group * 2^-20 of sum |x| 8 S at the very worst, three times that in fp32.  Measured, C in
// fp32, 128 to 8192 columns, x of one sign or of both: up to 2^-19.6 in groups of 128, 2^-20.4 of 64, 2^-20.2 of 32; a plain fp32 sum over all columns 2^-19.4.  C's own rounding in 16 bit is 2^-8 or 2^-11 of C.)
// fp32 activations are three bf16 numbers, whose sum is the value.
#pragma once
#include "lcma_experts.hpp"

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

// WN x WK waves: the first along N, a block of rows (of the weights) each, the others along K, a block of columns to a wave in turn; the weights of D of a wave's blocks are in
// flight.  MT x 16 rows of X; as many blocks of columns of them are in LDS at a time as XB bytes hold.
// bf16, groups of 128: a row, 14336 x 4096: 9.1 us (31 MB at 3.4 TB/s, 6.6 without the 2.5 of an empty launch: 448 tiles of 16 x 32, all at once, no second round to hide a start behind);
// 16 rows over 8 experts, 28672 x 4096: 80 us, 5.6 TB/s; fp16, groups of 64, 366 rows over 64 experts, 2816 x 2048: 48 us, 4.3 TB/s.
// What bounds it is the latency of the weights' way from memory, not the arithmetic: a block takes a wave about 60 vector instructions, 240 of the 420 clocks in which a CU's fourth of the
// memory's rate brings it.
template <class T, int G, int MT, int WN, int WK, int D, int XB> struct I4Gemm {
    using I = I4Type<T>;
    using Mul = typename I::Mul;
    using Frag = typename Mma16<Mul>::frag;
    static constexpr int NT = 64 * WN * WK, TM = 16 * MT, TN = 16 * WN, GROUPS = 128 / G, BLOCK = 1024 + GROUPS * 64, PER = 4 / GROUPS; // PER: instructions of a group
    static constexpr int PITCH = TN + 4, SUMS = WK * TM * PITCH * 4, LDS_BYTES = SUMS > XB ? SUMS : XB;
    static_assert(LDS_BYTES <= 160 * 1024 && I::PARTS * TM * (WK * D * 256 + 16) <= XB, "LDS budget of one CU; a turn of all waves");

    // Columns k .. k + 7 of a row of X, zeros from K on; put into LDS as the parts that are multiplied.
    struct Eight {
        u32x4 v[T::ES / 2];
    };
    static LCMA_DEV Eight take(const char *row, int k, int K) {
        Eight e;
#pragma unroll
        for (int h = 0; h < T::ES / 2; ++h) e.v[h] = exp_chunk<T>(row + (int64_t)(k + h * T::CH) * T::ES, K - (k + h * T::CH));
        return e;
    }
    static LCMA_DEV void put(const Eight &e, LCMA_LDS char *to, int part_bytes) {
        if constexpr (T::ES == 2) {
            *(LCMA_LDS u32x4 *)to = e.v[0];
        } else {
            const f32x4 half[2] = {__builtin_bit_cast(f32x4, e.v[0]), __builtin_bit_cast(f32x4, e.v[T::ES / 2 - 1])};
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = half[i / 4][i % 4];
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
                *(LCMA_LDS u32x4 *)(to + part * part_bytes) = w;
            }
        }
    }
    // Blocks c0 .. end - 1 of the tile's rows of X, by all threads, four loads of each in flight.
    static LCMA_DEV void stage(const I4GemmParams &p, const I8Place &at, int c0, int end, int pitch, int part_bytes, LCMA_LDS char *lds) {
        constexpr int U = 4;
        const int vectors = (end - c0) * 16, n = at.rows * vectors;
        const char *x = p.X + (int64_t)at.row0 * p.ldx_b;
        for (int i0 = threadIdx.x; i0 < n; i0 += U * NT) {
            Eight e[U];
            int to[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * NT, row = (int)((uint32_t)i / (uint32_t)vectors), v = i - row * vectors;
                to[u] = i < n ? row * pitch + v * 16 : -1;
                if (i < n) e[u] = take(x + (int64_t)row * p.ldx_b, c0 * 128 + v * 8, p.K);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (to[u] >= 0) put(e[u], lds + to[u], part_bytes);
        }
    }

    struct Block {
        u32x4 codes;
        float scales[GROUPS]; // of row lane % 16
    };
    static LCMA_DEV void fetch(const char *at, Block &b) { // at: of the block
        const int lane = threadIdx.x & 63;
        b.codes = *(const u32x4 *)(at + lane * 16);
        __builtin_memcpy(b.scales, __builtin_assume_aligned(at + 1024 + (lane & 15) * (GROUPS * 4), GROUPS * 4), GROUPS * 4);
    }

    // A block of columns: x, this lane's row of X in LDS (`row` of every 16), at the block's columns.
    static LCMA_DEV void multiply(const LCMA_LDS char *(&x)[MT], int at, int part_bytes, const Block &blk, f32x4 (&acc)[MT]) {
        const Frag minus = __builtin_bit_cast(Frag, u32x4{I::MINUS, I::MINUS, I::MINUS, I::MINUS});
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            Frag xf[PER][MT][I::PARTS];
            f32x4 sum[MT];
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int part = 0; part < I::PARTS; ++part) xf[j][i][part] = __builtin_bit_cast(Frag, *(const LCMA_LDS u32x4 *)(x[i] + at + part * part_bytes + (g * PER + j) * 64));
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                sum[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < PER; ++j)
#pragma unroll
                    for (int part = 0; part < I::PARTS; ++part) sum[i] = Mma16<Mul>::run(xf[j][i][part], minus, sum[i]);
            }
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const Frag wf = __builtin_bit_cast(Frag, i4_widened<T>(blk.codes[g * PER + j]));
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int part = 0; part < I::PARTS; ++part) sum[i] = Mma16<Mul>::run(xf[j][i][part], wf, sum[i]);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][v] = __builtin_fmaf(sum[i][v], blk.scales[g], acc[i][v]);
        }
    }

    static LCMA_DEV void run(const I4GemmParams &p, LCMA_LDS char *lds) {
        const I8Rows<TM, I4GemmParams> groups(p);
        if (!p.from) i8_zero_behind<T>(p, groups.behind, gridDim.x, NT);
        const int nx = groups.within(p), jobs = nx * p.nz, per = (jobs + 7) / 8, i = p.from + (int)(blockIdx.x >> 3);
        const int job = (int)(blockIdx.x & 7) * per + i; // an eighth of the tiles to every XCD, row tiles that share weights next to each other
        if (i >= per || job >= jobs) return;
        int tile, z;
        i8_tile_of_job(nx, p.nz, p.panel, job, tile, z);
        const I8Place at = groups.place(p, tile);
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = w / WN, wn = w % WN;
        const int first = z * WN + wn, all = (p.N + 15) / 16, blocks = p.blocks; // blocks of rows; of columns
        const char *q = p.Q + at.expert * p.expert_q + (int64_t)(first < all ? first : all - 1) * blocks * BLOCK; // (past the last: the last again, dropped)
        auto fetch_from = [&](int y, Block &blk) { fetch(q + (int64_t)(y < blocks ? y : blocks - 1) * BLOCK, blk); }; // (past the last: the last again, not used)
        f32x4 acc[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (blocks) {
            Block now[D], next[D];
            int y = wk;
#pragma unroll
            for (int d = 0; d < D; ++d) fetch_from(y + d * WK, next[d]);
            // whole turns of all waves in LDS at a time, D blocks each, as often as the rows there are leave room for
            const int room = (XB / (I::PARTS * at.rows) - 16) / (WK * D * 256) * (WK * D), chunk = room < blocks ? room : blocks, pitch = chunk * 256 + 16; // (16: 16 rows at one column meet different banks)
            const int part_bytes = at.rows * pitch;
            const LCMA_LDS char *x[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) { // (rows past the tile's: the last one again, dropped)
                const int row = i * 16 + (lane & 15);
                x[i] = lds + (row < at.rows ? row : at.rows - 1) * pitch + (lane >> 4) * 16;
            }
            for (int c0 = 0; c0 < blocks; c0 += chunk) {
                const int end = c0 + chunk < blocks ? c0 + chunk : blocks;
                if (c0) __syncthreads(); // all have read the blocks before
                stage(p, at, c0, end, pitch, part_bytes, lds);
                __syncthreads();
                for (; y < end; y += WK * D) {
#pragma unroll
                    for (int d = 0; d < D; ++d) now[d] = next[d];
                    if (y + WK * D < blocks)
#pragma unroll
                        for (int d = 0; d < D; ++d) fetch_from(y + (D + d) * WK, next[d]);
#pragma unroll
                    for (int d = 0; d < D; ++d)
                        if (y + d * WK < end) multiply(x, (y + d * WK - c0) * 256, part_bytes, now[d], acc);
                }
            }
            __syncthreads(); // the sums take the place of X
        }
        // lane: column lane % 16 of rows 4 (lane / 16) .. + 3
        LCMA_LDS float *mine = (LCMA_LDS float *)lds + wk * (TM * PITCH) + (lane >> 4) * 4 * PITCH + wn * 16 + (lane & 15);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) mine[(i * 16 + v) * PITCH] = acc[i][v];
        __syncthreads();
        for (int t = threadIdx.x; t < TM * TN / 4; t += NT) { // four neighbouring columns of a row; the waves along K in ascending order
            const int row = t / (TN / 4), n = t % (TN / 4) * 4, col = z * TN + n;
            if (row >= at.rows || col >= p.N) continue;
            const LCMA_LDS float *of = (const LCMA_LDS float *)lds + row * PITCH + n;
            f32x4 sum = *(const LCMA_LDS f32x4 *)of;
#pragma unroll
            for (int k = 1; k < WK; ++k) sum += *(const LCMA_LDS f32x4 *)(of + k * TM * PITCH);
            if (p.bias) sum += i8_four(p.bias + (int64_t)at.expert * p.N, col, p.N);
            i8_store4<T>(p.C + ((int64_t)(at.row0 + row) * p.ldc + col) * T::ES, sum, p.N - col);
        }
    }
};

} // namespace lcma
