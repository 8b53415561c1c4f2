// Products of experts in their own type (bf16, fp16, fp32) for gfx950:
//   product   C[r][n] = sum_k A[r][k] W_e[n][k]  (or A[r][k] B_e[k][n])  for the rows r of expert e; rows behind the last expert's are zero
//   gradient  C_e[m][n] = sum_r A[r][m] B[r][n]  over the rows r of expert e (none: zeros)
// Sums in fp32, one rounding.  How many rows an expert has is known on the device alone.
//
// An operand of a tile comes in one of two forms: its rows (of the tile) are k-contiguous, or, COL, its columns are what is contiguous and k goes from
// row to row of the stored matrix.  A step is 128 bytes of k (64, fp32: 32); in LDS R rows of a k-contiguous operand are R x 128 bytes, R columns of the other
// form are 64 (32) rows of R elements: both R * 128 bytes.  Fragments of the first are read 16 bytes at a time, those of the second with the transposing
// read of 16-bit types, or element by element.
// Addresses are 64-bit bases of a tile, so matrices may be of any size.
#pragma once
#include "lcma_i8.hpp"

namespace lcma {

// A tile's operands and where its result goes; k: what is summed over; am, bn: rows and columns of C that are there.
struct ExpJob {
    const char *a, *b;
    char *c;
    int am, bn, k;
};

template <class T, bool BCOL, int TM, int TN> LCMA_DEV ExpJob product_job(const ExpertsGemmParams &p, const I8Place &at, int col0) {
    ExpJob j;
    j.a = p.A + (int64_t)at.row0 * p.lda_b;
    j.b = p.B + (int64_t)at.expert * p.expert_b + (BCOL ? (int64_t)col0 * T::ES : (int64_t)col0 * p.ldb_b);
    j.c = p.C + (int64_t)at.row0 * p.ldc_b + (int64_t)col0 * T::ES;
    j.am = at.rows;
    j.bn = p.N - col0 < TN ? p.N - col0 : TN;
    j.k = p.K;
    return j;
}
// Tile `job` of the gradient: expert by expert.
template <class T, int TM, int TN> LCMA_DEV ExpJob gradient_job(const ExpertsGemmParams &p, int job) {
    const int of = p.nx * p.nz, e = job / of;
    int x, z;
    i8_tile_of_job(p.nx, p.nz, p.panel, job - e * of, x, z);
    const int begin = i8_row(p, e), end = i8_row(p, e + 1);
    ExpJob j;
    j.a = p.A + (int64_t)begin * p.lda_b + (int64_t)x * TM * T::ES;
    j.b = p.B + (int64_t)begin * p.ldb_b + (int64_t)z * TN * T::ES;
    j.c = p.C + (int64_t)e * p.expert_b + (int64_t)x * TM * p.ldc_b + (int64_t)z * TN * T::ES;
    j.am = p.M - x * TM < TM ? p.M - x * TM : TM;
    j.bn = p.N - z * TN < TN ? p.N - z * TN : TN;
    j.k = end > begin ? end - begin : 0;
    return j;
}

// Tiles of the gradient to work-groups, one each (work-groups go to the eight XCDs in turn); -1: none.  An expert's tiles take as long as it has rows, so an XCD that had whole experts would
// be done long before another: eighths of each expert's tiles to every XCD, in turn (the launch holds whole eights of them).  fp32, 2331 rows spread unequally over 12 experts, 1001 x 515: 41 us by experts, 37 by
// eighths; 120 narrow matrices with a router's counts 16 % less by eighths on average.
// But then an expert's rows, which one L2 would hold, go to eight.  `by_expert` (16 bit, matrices of a few tiles along both sides, where every eighth reads most of the rows): by experts, one behind the other.  bf16, 42342 rows
// over 8, 304 x 1104: 100.7 us by eighths, 70.3 by experts, 39392 rows in equal shares, 384 x 1152: 88.6 and 46.3; 59 such matrices with a router's counts 13 % less on average by experts and 1.2 times at worst (15574 x 4 of 8, 752 x 320: 97.8 and 117), in equal shares
// 27 % less.  Where it is left at eighths, 16 bit: 1 to 5 % less by eighths with a router's counts (0.55 to 1.3 times), 5 to 15 % more in equal shares.
LCMA_DEV int exp_gradient_tile(const ExpertsGemmParams &p) {
    const int of = p.nx * p.nz, jobs = p.experts * of, q = p.by_expert ? (jobs + 7) >> 3 : (of + 7) >> 3, i = p.from + (int)(blockIdx.x >> 3), job = (i / q * 8 + (int)(blockIdx.x & 7)) * q + i % q;
    return job < jobs ? job : -1;
}

// Where 16-byte chunk c of a row lies in LDS.  k-contiguous rows of 128 bytes: 16 rows at one chunk column meet all banks once.  Rows of columns, 16 bit: the four
// rows (k) of a transposing read, 64 bytes of each, meet different banks (rows of 64 bytes do so by themselves; fp32 needs nothing).
LCMA_DEV constexpr int exp_row_chunk(int row, int c) { return c ^ ((row >> 1) & 7); }
template <class T, int R> LCMA_DEV constexpr int exp_col_chunk(int k, int c) {
    static_assert(T::ES == 4 || R <= 32 || R == 64 || R == 128, "rows of 64, 128 or 256 bytes");
    return T::ES == 4 || R <= 32 ? c : R == 64 ? c ^ ((k >> 1 & 1) << 2) : c ^ ((k & 3) << 2);
}

// Fragments of 32 columns, 32 block and on, of R columns in LDS for the four instructions of a step (16 bit): eight k of a column are two transposing reads of four.
// Sixteen lanes of such a read give the addresses of four rows (k) x 16 columns, four lanes to a row, and get a column each.  One block of instructions that waits for
// its own results: the compiler's form of the read carries no alias information and would wait for every load in flight.
template <class T, int R> LCMA_DEV void exp_columns(const LCMA_LDS char *tile, int block, u32x4 (&f)[4]) {
    constexpr int P = R * 2;
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4, k = i >> 2, c = block * 4 + (g & 1) * 2 + ((i & 3) >> 1);
    const uint32_t at = (uint32_t)(uintptr_t)tile + ((g >> 1) * 8 + k) * P + exp_col_chunk<T, R>(k, c) * 16 + (i & 1) * 8;
    u32x2 r[4][2];
    asm volatile("ds_read_b64_tr_b16 %0, %8\n"
                 "ds_read_b64_tr_b16 %1, %8 offset:%9\n"
                 "ds_read_b64_tr_b16 %2, %8 offset:%10\n"
                 "ds_read_b64_tr_b16 %3, %8 offset:%11\n"
                 "ds_read_b64_tr_b16 %4, %8 offset:%12\n"
                 "ds_read_b64_tr_b16 %5, %8 offset:%13\n"
                 "ds_read_b64_tr_b16 %6, %8 offset:%14\n"
                 "ds_read_b64_tr_b16 %7, %8 offset:%15\n"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(r[0][0]), "=&v"(r[0][1]), "=&v"(r[1][0]), "=&v"(r[1][1]), "=&v"(r[2][0]), "=&v"(r[2][1]), "=&v"(r[3][0]), "=&v"(r[3][1])
                 : "v"(at), "n"(4 * P), "n"(16 * P), "n"(20 * P), "n"(32 * P), "n"(36 * P), "n"(48 * P), "n"(52 * P)
                 : "memory");
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = u32x4{r[j][0][0], r[j][0][1], r[j][1][0], r[j][1][1]};
}
// Two blocks of 32 columns, `block` even: one wait for both (gradient of 8192 x 2 of 8, 4096 x 14336: 1594 -> 1565 us).
template <class T, int R> LCMA_DEV void exp_columns_pair(const LCMA_LDS char *tile, int block, u32x4 (&f0)[4], u32x4 (&f1)[4]) {
    constexpr int P = R * 2;
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4, k = i >> 2, c = block * 4 + (g & 1) * 2 + ((i & 3) >> 1);
    const uint32_t row = (uint32_t)(uintptr_t)tile + ((g >> 1) * 8 + k) * P + (i & 1) * 8, a0 = row + exp_col_chunk<T, R>(k, c) * 16, a1 = row + exp_col_chunk<T, R>(k, c + 4) * 16;
    u32x2 r[4][2], s[4][2];
    asm volatile("ds_read_b64_tr_b16 %0, %16\n"
                 "ds_read_b64_tr_b16 %1, %16 offset:%18\n"
                 "ds_read_b64_tr_b16 %8, %17\n"
                 "ds_read_b64_tr_b16 %9, %17 offset:%18\n"
                 "ds_read_b64_tr_b16 %2, %16 offset:%19\n"
                 "ds_read_b64_tr_b16 %3, %16 offset:%20\n"
                 "ds_read_b64_tr_b16 %10, %17 offset:%19\n"
                 "ds_read_b64_tr_b16 %11, %17 offset:%20\n"
                 "ds_read_b64_tr_b16 %4, %16 offset:%21\n"
                 "ds_read_b64_tr_b16 %5, %16 offset:%22\n"
                 "ds_read_b64_tr_b16 %12, %17 offset:%21\n"
                 "ds_read_b64_tr_b16 %13, %17 offset:%22\n"
                 "ds_read_b64_tr_b16 %6, %16 offset:%23\n"
                 "ds_read_b64_tr_b16 %7, %16 offset:%24\n"
                 "ds_read_b64_tr_b16 %14, %17 offset:%23\n"
                 "ds_read_b64_tr_b16 %15, %17 offset:%24\n"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(r[0][0]), "=&v"(r[0][1]), "=&v"(r[1][0]), "=&v"(r[1][1]), "=&v"(r[2][0]), "=&v"(r[2][1]), "=&v"(r[3][0]), "=&v"(r[3][1]), "=&v"(s[0][0]),
                   "=&v"(s[0][1]), "=&v"(s[1][0]), "=&v"(s[1][1]), "=&v"(s[2][0]), "=&v"(s[2][1]), "=&v"(s[3][0]), "=&v"(s[3][1])
                 : "v"(a0), "v"(a1), "n"(4 * P), "n"(16 * P), "n"(20 * P), "n"(32 * P), "n"(36 * P), "n"(48 * P), "n"(52 * P)
                 : "memory");
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f0[j] = u32x4{r[j][0][0], r[j][0][1], r[j][1][0], r[j][1][1]};
        f1[j] = u32x4{s[j][0][0], s[j][0][1], s[j][1][0], s[j][1][1]};
    }
}
// The four fragments of 32 rows (columns) from 32 block on of an operand with R of them.
template <class T, bool COL, int R> LCMA_DEV void exp_fragments(const LCMA_LDS char *tile, int block, u32x4 (&f)[4]) {
    const int lane = threadIdx.x & 63, l32 = lane & 31, lh = lane >> 5;
    if constexpr (!COL) {
        const int row = block * 32 + l32;
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = *(const LCMA_LDS u32x4 *)(tile + row * 128 + exp_row_chunk(row, k * 2 + lh) * 16);
    } else if constexpr (T::ES == 2) {
        exp_columns<T, R>(tile, block, f);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t) f[k][t] = *(const LCMA_LDS uint32_t *)(tile + ((k * 8 + lh * 4 + t) * R + block * 32 + l32) * 4);
    }
}

// A wave's part of a tile of C (NMI x NNI blocks of 32 x 32; rows, cols: of C from its first element on) rounded and stored: through SR rows of 128 bytes of LDS that are the
// wave's own, so that it leaves as whole lines, 16 bytes a lane.  The right operand is the left one of the matrix instruction: a lane holds four neighbouring columns.
// Blocks of rows follow each other, or, TWO, the second pair of them is 128 rows on; the blocks of columns are GAP columns apart.
// FULL: all of it lies inside C.  STREAM: and passes the caches by, in rows that are whole lines in memory (64 x 128 tiles, gradient of 1021 x 6 of 64, 2816 x 2048: 355 -> 292 us).  A wave's store is whole
// lines of it, or, with one block of columns in 16 bit (64 x 64 tiles), halves that the wave beside it completes at about the same time: through the caches these took 1.07 times as long on average over 57 gradients
// (1.33 at most, 0.98 at least), off 16 bytes 1.04 (1.2, 0.99).  Halves that nothing completes soon (256 x 256 tiles whose waves' columns lie apart) were 340 -> 540 past the caches, at 2 rows of 8 experts, 28672 x 4096.
template <class T, int NMI, int NNI, bool TWO, int GAP, int SR, bool FULL, bool STREAM>
LCMA_DEV void exp_store_rows(LCMA_LDS char *strip, char *c, int64_t ldc_b, int rows, int cols, const f32x16 (&acc)[NMI][NNI]) {
    constexpr int ES = T::ES, BLOCKS = ES == 4 ? 1 : NNI == 1 ? 1 : 2, L = BLOCKS * 32 * ES / 16, RPS = 64 / L; // 32-column blocks of a pass; lanes of a row, rows of a store
    static_assert(NNI % BLOCKS == 0 && SR % RPS == 0, "whole passes");
    // (the lane number anew, hidden: what derives from it would otherwise be kept in registers through the steps)
    int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(lane));
    const int l32 = lane & 31, lh = lane >> 5, row_of = lane / L, ch = lane % L;
    if (!FULL && (rows <= 0 || cols <= 0)) return;
    char *const at = c + (int64_t)row_of * ldc_b;
#pragma unroll
    for (int mi = 0; mi < NMI; ++mi) {
        const int row0 = TWO ? mi / 2 * 128 + mi % 2 * 32 : mi * 32;
        if (!FULL && row0 >= rows) return;
#pragma unroll
        for (int n0 = 0; n0 < NNI; n0 += BLOCKS) {
#pragma unroll
            for (int h = 0; h < 32 / SR; ++h) {
                if (SR == 32 || l32 / SR == h) {
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const f32x16 &v = acc[mi][n0 + b];
                            const int byte = (b * 32 + g * 8 + lh * 4) * ES;
                            LCMA_LDS char *to = strip + l32 % SR * (L * 16) + ((byte >> 4) ^ (l32 & (L - 1))) * 16 + (byte & 15);
                            if constexpr (ES == 2) {
                                const uint32_t lo = Round<T>::run(v[g * 4]) | (Round<T>::run(v[g * 4 + 1]) << 16), hi = Round<T>::run(v[g * 4 + 2]) | (Round<T>::run(v[g * 4 + 3]) << 16);
                                *(LCMA_LDS uint64_t *)to = (uint64_t)hi << 32 | lo;
                            } else {
                                *(LCMA_LDS f32x4 *)to = f32x4{v[g * 4], v[g * 4 + 1], v[g * 4 + 2], v[g * 4 + 3]};
                            }
                        }
                }
                lanes_meet();
#pragma unroll
                for (int it = 0; it < SR / RPS; ++it) {
                    const int in = it * RPS + row_of, row = h * SR + in, of = ch * (16 / ES), col = (n0 + of / 32) * GAP + of % 32;
                    const u32x4 v = *(const LCMA_LDS u32x4 *)(strip + in * (L * 16) + (ch ^ (row & (L - 1))) * 16);
                    char *to = at + (int64_t)(row0 + h * SR + it * RPS) * ldc_b + col * ES;
                    if constexpr (STREAM) __builtin_nontemporal_store(v, (u32x4 *)to);
                    else if constexpr (FULL) __builtin_memcpy(to, &v, 16);
                    else if (row0 + row < rows && col < cols) i8_store16<T>(to, v, cols - col);
                }
                lanes_meet();
            }
        }
    }
}
template <class T, int NMI, int NNI, bool TWO = false, int GAP = 32, int SR = 32, bool GRAD = false>
LCMA_DEV void exp_store(LCMA_LDS char *strip, char *c, int64_t ldc_b, int rows, int cols, const f32x16 (&acc)[NMI][NNI], bool stream = false) {
    const bool full = rows >= (TWO ? (NMI - 1) / 2 * 128 + (NMI - 1) % 2 * 32 : (NMI - 1) * 32) + 32 && cols >= (NNI - 1) * GAP + 32;
    if (GRAD && full && stream) exp_store_rows<T, NMI, NNI, TWO, GAP, SR, true, GRAD>(strip, c, ldc_b, rows, cols, acc);
    else if (full) exp_store_rows<T, NMI, NNI, TWO, GAP, SR, true, false>(strip, c, ldc_b, rows, cols, acc);
    else exp_store_rows<T, NMI, NNI, TWO, GAP, SR, false, false>(strip, c, ldc_b, rows, cols, acc);
}

// Rows of C behind the last expert's are zero: the work-groups of the launch share them.
template <class T, int NT> LCMA_DEV void exp_zero_behind(const ExpertsGemmParams &p, int behind) {
    for (uint32_t row = behind + blockIdx.x; row < (uint32_t)p.rows; row += gridDim.x) // (past 2^31 before it ends)
        for (int n = threadIdx.x * T::CH; n < p.N; n += NT * T::CH) i8_store16<T>(p.C + (int64_t)row * p.ldc_b + (int64_t)n * T::ES, u32x4{0, 0, 0, 0}, p.N - n);
}

// `n` (up to 16 / ES, none: not read) elements from `at`, which has the alignment of an element, zeros behind.
template <class T> LCMA_DEV u32x4 exp_chunk(const char *at, int n) {
    u32x4 v = {0, 0, 0, 0};
    if (n >= T::CH) {
        __builtin_memcpy(&v, at, 16);
    } else {
#pragma unroll
        for (int i = 0; i < T::CH; ++i)
            if (i < n) {
                if constexpr (T::ES == 4) v[i] = ((const uint32_t *)at)[i];
                else v[i / 2] |= (uint32_t)((const uint16_t *)at)[i] << (i & 1) * 16;
            }
    }
    return v;
}

// Any sizes, leading dimensions and alignments: a tile per work-group, operands through registers into two stages of LDS, the loads of a step one step ahead.
// Bound by the way of the operands: a load and an LDS store of each chunk, and one step of loads in flight, where direct loads have two.  bf16, rows of 8192 x 2 of 8, 4096 x 14336: 3980 us on
// 64 x 64 against 3310 of the ring on the same tile; 128 x 2 of 8, 2048 x 1024: 16.4 against 8.3.  What it is for, fp16 1021 x 6 of 64, 2815 x 2055: products 300 us on 128 x 128 and 358 on 64 x 64,
// with K x N weights 728 and 535, gradient 425 and 507.
template <class T, bool ACOL, bool BCOL, bool GRAD, int TM, int TN, int WGM, int WGN> struct ExpStaged {
    static constexpr int NT = 64 * WGM * WGN, NMI = TM / WGM / 32, NNI = TN / WGN / 32, KS = 128 / T::ES;
    static constexpr int A_STAGE = TM * 128, STAGE = (TM + TN) * 128, LDS_BYTES = 2 * STAGE, QA = TM * 8 / NT, QB = TN * 8 / NT;
    static_assert(NT / 64 * 4096 <= LDS_BYTES && TM * 8 % NT == 0 && TN * 8 % NT == 0, "strips; whole loads");

    template <bool COL, int R, int Q> static LCMA_DEV void load(const char *at, int64_t ld_b, int wide, int k, int y, u32x4 (&v)[Q]) {
        constexpr int CPR = R * T::ES / 16;
        const int left = k - y * KS; // (k may be up to 2^31 - 1: the numbers past it do not fit)
        at += (int64_t)y * KS * (COL ? ld_b : T::ES);
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int i = q * NT + (int)threadIdx.x;
            if constexpr (!COL) {
                const int row = i >> 3, k0 = (i & 7) * T::CH;
                v[q] = exp_chunk<T>(at + (int64_t)row * ld_b + k0 * T::ES, row < wide ? left - k0 : 0);
            } else {
                const int k0 = i / CPR, col = i % CPR * T::CH;
                v[q] = exp_chunk<T>(at + (int64_t)k0 * ld_b + col * T::ES, k0 < left ? wide - col : 0);
            }
        }
    }
    template <bool COL, int R, int Q> static LCMA_DEV void put(LCMA_LDS char *to, const u32x4 (&v)[Q]) {
        constexpr int CPR = R * T::ES / 16;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int i = q * NT + (int)threadIdx.x;
            if constexpr (!COL) *(LCMA_LDS u32x4 *)(to + (i >> 3) * 128 + exp_row_chunk(i >> 3, i & 7) * 16) = v[q];
            else *(LCMA_LDS u32x4 *)(to + i / CPR * (R * T::ES) + exp_col_chunk<T, R>(i / CPR, i % CPR) * 16) = v[q];
        }
    }

    static LCMA_DEV void run(const ExpertsGemmParams &p, LCMA_LDS char *lds) {
        ExpJob j;
        if constexpr (GRAD) {
            const int job = exp_gradient_tile(p);
            if (job < 0) return;
            j = gradient_job<T, TM, TN>(p, job);
        } else {
            const I8Rows<TM, ExpertsGemmParams> groups(p);
            if (!p.from) exp_zero_behind<T, NT>(p, groups.behind);
            const int nx = groups.within(p), jobs = nx * p.nz, per = (jobs + 7) / 8, i = p.from + (int)(blockIdx.x >> 3), job = (int)(blockIdx.x & 7) * per + i;
            if (i >= per || job >= jobs) return;
            int x, z;
            i8_tile_of_job(nx, p.nz, p.panel, job, x, z);
            j = product_job<T, BCOL, TM, TN>(p, groups.place(p, x), z * TN);
        }
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w / WGN, wn = w % WGN, steps = (int)(((uint32_t)j.k + (KS - 1)) / KS);
        f32x16 acc[NMI][NNI];
#pragma unroll
        for (int i = 0; i < NMI; ++i)
#pragma unroll
            for (int n = 0; n < NNI; ++n) zero(acc[i][n]);
        u32x4 va[QA], vb[QB];
        if (steps) {
            load<ACOL, TM>(j.a, p.lda_b, j.am, j.k, 0, va);
            load<BCOL, TN>(j.b, p.ldb_b, j.bn, j.k, 0, vb);
        }
        for (int y = 0; y < steps; ++y) {
            LCMA_LDS char *st = lds + (y & 1) * STAGE;
            put<ACOL, TM>(st, va);
            put<BCOL, TN>(st + A_STAGE, vb);
            __syncthreads(); // the stage is whole, and all have read the other one, which the next step writes
            if (y + 1 < steps) {
                load<ACOL, TM>(j.a, p.lda_b, j.am, j.k, y + 1, va);
                load<BCOL, TN>(j.b, p.ldb_b, j.bn, j.k, y + 1, vb);
            }
            u32x4 a[NMI][4], b[NNI][4];
#pragma unroll
            for (int i = 0; i < NMI; ++i) exp_fragments<T, ACOL, TM>(st, wm * NMI + i, a[i]);
#pragma unroll
            for (int n = 0; n < NNI; ++n) exp_fragments<T, BCOL, TN>(st + A_STAGE, wn * NNI + n, b[n]);
            using Frag = typename Mma<T>::frag;
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < NMI; ++i)
#pragma unroll
                    for (int n = 0; n < NNI; ++n) Mma<T>::run(__builtin_bit_cast(Frag, b[n][k]), __builtin_bit_cast(Frag, a[i][k]), acc[i][n]);
        }
        __syncthreads(); // the strips take the place of the stages
        const int row = wm * NMI * 32, col = wn * NNI * 32;
        exp_store<T, NMI, NNI, false, 32, 32, GRAD>(lds + w * 4096, j.c + (int64_t)row * p.ldc_b + (int64_t)col * T::ES, p.ldc_b, j.am - row, j.bn - col, acc, p.stream);
    }
};

} // namespace lcma
