// The experts' product of 16-bit types on few rows, at sizes, leading dimensions and alignments that are no whole 16 bytes: operands come into registers, where loads take any address, and go on
// into LDS from there.  Where a chunk of 16 bytes lies inside what there is, it is one load (rows past a tile's last one: the last one again, their sums are dropped); in the last step of K, and where
// columns are contiguous in a tile that has not all of them, element by element.
#pragma once
#include "lcma_experts_ring.hpp"

namespace lcma {

// Chunk c (16 bytes) of `line` of an operand of a tile: a row of it from k = y * 64 on, or, COL, row y * 64 + line of the stored matrix.  whole: the step is not the last one, and all columns are there.
template <class T, bool COL> LCMA_DEV u32x4 exp_take(const char *at, uint32_t ld_b, int wide, int k, int y, int line, int c, bool whole) {
    u32x4 v;
    if (whole) {
        const uint32_t row = COL ? line : line < wide ? line : wide - 1;
        const char *from = COL ? at + (int64_t)y * 64 * ld_b : at + (int64_t)y * 128;
        __builtin_memcpy(&v, from + (row * ld_b + c * 16), 16);
    } else {
        const int k0 = y * 64 + (COL ? line : c * 8), n = COL ? (k0 < k ? wide - c * 8 : 0) : line < wide ? k - k0 : 0;
        v = exp_chunk<T>(COL ? at + (int64_t)k0 * ld_b + c * 16 : at + (int64_t)line * ld_b + (int64_t)k0 * 2, n);
    }
    return v;
}

// Few rows: a work-group owns a tile of 32 x 32 of C and its waves split K between them, a step to a wave in turn, as ExpFewRows; a wave has 8 KB of LDS, and the registers that
// a step's operands leave take those of its next one.
// Bound by the loads' latency, one step of a wave in flight, and off lines by half-used ones.  bf16, us, against the 64 x 64 tile above: 2 rows of 8 experts, K x N weights 28671 x 4099
// 351 : 887 (N x K 168 : 102, which the time model sees); 32 rows, 2049 x 1025 14.4 : 19.7, K x N 25.4 : 52.9.  One load a chunk where it lies inside: 28671 x 4099 took 890 element by element.
template <class T, bool BCOL, int WK> struct ExpAnyFewRows {
    static constexpr int R = 32, HALF = R * 128, STAGE = 2 * HALF, PITCH = R + 4, SUMS = WK * R * PITCH * 4, LDS_BYTES = SUMS > WK * STAGE ? SUMS : WK * STAGE;
    static_assert(T::ES == 2, "16-bit types");
    using Frag = typename Mma<T>::frag;

    static LCMA_DEV void run(const ExpertsGemmParams &p, LCMA_LDS char *lds) {
        const int lane = threadIdx.x & 63, l32 = lane & 31, lh = lane >> 5, wk = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const I8Rows<R, ExpertsGemmParams> groups(p);
        exp_zero_behind<T, 64 * WK>(p, groups.behind);
        const int nx = groups.within(p), jobs = nx * p.nz, per = (jobs + 7) / 8;
        const int job = (blockIdx.x & 7) * per + (blockIdx.x >> 3); // an eighth of the tiles to every XCD, row tiles that share weights next to each other
        if ((int)(blockIdx.x >> 3) >= per || job >= jobs) return;
        int x, z;
        i8_tile_of_job(nx, p.nz, p.panel, job, x, z);
        ExpJob j = product_job<T, BCOL, R, R>(p, groups.place(p, x), z * R);
        j.a = exp_uniform(j.a);
        j.b = exp_uniform(j.b);
        const uint32_t lda = (uint32_t)p.lda_b, ldb = (uint32_t)p.ldb_b;
        const int steps = (int)(((uint32_t)j.k + 63) / 64);
        f32x16 acc;
        zero(acc);
        LCMA_LDS char *st = lds + wk * STAGE;
        u32x4 va[4], vb[4];
        auto take = [&](int y) {
            const bool inside = y < steps - 1, b_whole = inside && (!BCOL || j.bn == R);
#pragma unroll
            for (int q = 0; q < 4; ++q) { // 8 rows of 128 bytes, or 16 rows (k) of 64
                va[q] = exp_take<T, false>(j.a, lda, j.am, j.k, y, q * 8 + (lane >> 3), lane & 7, inside);
                vb[q] = BCOL ? exp_take<T, true>(j.b, ldb, j.bn, j.k, y, q * 16 + (lane >> 2), lane & 3, b_whole) : exp_take<T, false>(j.b, ldb, j.bn, j.k, y, q * 8 + (lane >> 3), lane & 7, b_whole);
            }
        };
        if (wk < steps) take(wk);
        for (int y = wk; y < steps; y += WK) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int row = q * 8 + (lane >> 3), at = row * 128 + exp_row_chunk(row, lane & 7) * 16;
                *(LCMA_LDS u32x4 *)(st + at) = va[q];
                *(LCMA_LDS u32x4 *)(st + HALF + (BCOL ? (q * 64 + lane) * 16 : at)) = vb[q];
            }
            lanes_meet();
            u32x4 a[4], b[4];
            exp_fragments<T, false, R>(st, 0, a);
            exp_fragments<T, BCOL, R>(st + HALF, 0, b);
            if (y + WK < steps) take(y + WK);
#pragma unroll
            for (int k = 0; k < 4; ++k) Mma<T>::run(__builtin_bit_cast(Frag, b[k]), __builtin_bit_cast(Frag, a[k]), acc);
            lanes_meet();
        }
        __syncthreads(); // every wave has read its last step: the sums take the place of the stages
        LCMA_LDS float *mine = (LCMA_LDS float *)lds + wk * (R * PITCH);
#pragma unroll
        for (int g = 0; g < 4; ++g) *(LCMA_LDS f32x4 *)(mine + l32 * PITCH + g * 8 + lh * 4) = f32x4{acc[g * 4], acc[g * 4 + 1], acc[g * 4 + 2], acc[g * 4 + 3]}; // four neighbouring columns
        __syncthreads();
        for (int t = threadIdx.x; t < R * R / 4; t += 64 * WK) {
            const int row = t / (R / 4), n = t % (R / 4) * 4;
            if (row >= j.am || n >= j.bn) continue;
            const LCMA_LDS float *of = (const LCMA_LDS float *)lds + row * PITCH + n;
            f32x4 sum = *(const LCMA_LDS f32x4 *)of;
#pragma unroll
            for (int k = 1; k < WK; ++k) sum += *(const LCMA_LDS f32x4 *)(of + k * R * PITCH);
            i8_store4<T>(j.c + (int64_t)row * p.ldc_b + n * T::ES, sum, j.bn - n);
        }
    }
};

} // namespace lcma
