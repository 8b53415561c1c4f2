// The experts' products on tiles below 256 x 256, operands straight into LDS (either form of both, csrc/lcma_experts.hpp): 16-bit types in whole 16 bytes, fp32 at any
// sizes (a load needs the alignment of four bytes).  What lies past a tile's rows or columns may be anything: it reaches elements of C alone that are not there.  What lies past the
// last k is zero on both sides: by the extent where k goes from row to row; in k-contiguous rows 16 bytes at a time from past the extent (16 bit), or in
// the fragments of the last step (fp32).
#pragma once
#include "lcma_experts.hpp"

namespace lcma {

// A pointer that is the same in all lanes, in scalar registers.  (Global memory, said so: the compiler takes a pointer made of two numbers for one into any memory, and stores through it
// count as LDS accesses too.)
template <class P> LCMA_DEV P *exp_uniform(P *at) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)at >> 32));
    return (P *)(__attribute__((address_space(1))) P *)((uint64_t)hi << 32 | lo);
}
// The rows of the stored matrix from step y on, `steps` steps of them; none past the last k.  The extent ends behind the dword of the last column: the range is checked by whole dwords, and a 16-bit
// gradient's columns may be odd in rows of whole 16 bytes (what the dword holds besides belongs to a column that is not there).
template <class T> LCMA_DEV __amdgpu_buffer_rsrc_t exp_columns_from(const char *at, int wide, int k, uint32_t ld_b, int y, int steps) {
    constexpr int KS = 128 / T::ES;
    const int left = (int)((uint32_t)k - (uint32_t)y * KS), n = left < steps * KS ? left : steps * KS; // (unsigned: y * KS may lie past 2^31, behind k)
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(at) + (int64_t)y * KS * ld_b, 0, n > 0 ? (n - 1) * (int)ld_b + ((wide * T::ES + 3) & ~3) : 0, 0x00020000);
}
template <class T> LCMA_DEV __amdgpu_buffer_rsrc_t exp_rows_of(const char *at, int wide, int k, uint32_t ld_b) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(at), 0, k > 0 ? (wide - 1) * (int)ld_b + k * T::ES : 0, 0x00020000);
}
// fp32: zeros in the place of what is past the `left` k of the last step.
template <int N> LCMA_DEV void exp_end_of_k(u32x4 (&f)[N][4], int left) {
    const int lh = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int t = 0; t < 4; ++t) f[n][k][t] = k * 8 + lh * 4 + t < left ? f[n][k][t] : 0;
}

// One tile of TM x TN per work-group of WGM x WGN waves.  A step is 64 k (fp32: 32); three stages of LDS hold the steps in flight, the loads run two steps ahead and are waited for by
// count, and one barrier a step says that all waves' parts of it have landed and that all have read the stage that is loaded anew (csrc/lcma_i8.hpp has the
// same with its measurements).  Bound by memory at hundreds of rows, by the loads' way through LDS above: bf16, rows of 128 x 2 of 8, 2048 x 1024: 8.3 us on 64 x 64 (weights at 4.0 TB/s; 32 x 32 takes
// 11.1), 9.0 on 64 x 128; fp16 1021 x 6 of 64, 2816 x 2056: 287 and 255 against 213 on 128 x 256.  fp32 (64 x 64 alone, by the matrix pipe, 68 % of which is at work): 777 x 3 of 12, 1001 x 515: 33 us,
// gradients 39 and 35; 4096 x 2 of 8, 2048 x 2048: 538 (128 TFLOP/s).
template <class T, bool ACOL, bool BCOL, bool GRAD, int TM, int TN, int WGM, int WGN> struct ExpRing {
    static constexpr int NT = 64 * WGM * WGN, NMI = TM / WGM / 32, NNI = TN / WGN / 32, KS = 128 / T::ES;
    static constexpr int A_STAGE = TM * 128, STAGE = (TM + TN) * 128, LDS_BYTES = 3 * STAGE, QA = TM * 8 / NT, QB = TN * 8 / NT;
    static_assert(NT / 64 * 4096 <= LDS_BYTES && TM * 8 % NT == 0 && TN * 8 % NT == 0 && LDS_BYTES <= 160 * 1024 && 2 * (QA + QB) <= 63, "tile and wave grid");
    using Frag = typename Mma<T>::frag;
    static constexpr uint32_t NONE = 1u << 30; // an offset past any extent

    static LCMA_DEV void run(const ExpertsGemmParams &p, LCMA_LDS char *lds) {
        ExpJob j;
        if constexpr (GRAD) {
            const int job = exp_gradient_tile(p);
            if (job < 0) return;
            j = gradient_job<T, TM, TN>(p, job);
        } else {
            const I8Rows<TM, ExpertsGemmParams> groups(p);
            exp_zero_behind<T, NT>(p, groups.behind);
            const int nx = groups.within(p), jobs = nx * p.nz, per = (jobs + 7) / 8, job = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
            if ((int)(blockIdx.x >> 3) >= per || job >= jobs) return;
            int x, z;
            i8_tile_of_job(nx, p.nz, p.panel, job, x, z);
            j = product_job<T, BCOL, TM, TN>(p, groups.place(p, x), z * TN);
        }
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w / WGN, wn = w % WGN;
        f32x16 acc[NMI][NNI];
#pragma unroll
        for (int i = 0; i < NMI; ++i)
#pragma unroll
            for (int n = 0; n < NNI; ++n) zero(acc[i][n]);
        multiply(p, j, w, wm, wn, acc, lds, lds + STAGE, lds + 2 * STAGE);
        __syncthreads(); // no load is in flight and every wave has read its last step: the strips take the place of the stages
        const int row = wm * NMI * 32, col = wn * NNI * 32;
        exp_store<T, NMI, NNI, false, 32, 32, GRAD>(lds + w * 4096, j.c + (int64_t)row * p.ldc_b + (int64_t)col * T::ES, p.ldc_b, j.am - row, j.bn - col, acc, p.stream);
    }
    // restrict: the loads in flight towards one stage do not touch what is read from another (the compiler would otherwise wait for all of them in
    // front of every read)
    static LCMA_DEV void multiply(const ExpertsGemmParams &p, const ExpJob &j, int w, int wm, int wn, f32x16 (&acc)[NMI][NNI], LCMA_LDS char *__restrict__ s0,
                                  LCMA_LDS char *__restrict__ s1, LCMA_LDS char *__restrict__ s2) {
        constexpr int CA = TM * T::ES / 16, CB = TN * T::ES / 16; // 16-byte chunks of a row of the other form
        const int tid = threadIdx.x, steps = (int)(((uint32_t)j.k + (KS - 1)) / KS), chunk = exp_row_chunk(tid >> 3, tid & 7) * 16;
        const uint32_t lda = (uint32_t)p.lda_b, ldb = (uint32_t)p.ldb_b;
        const auto rows_a = exp_rows_of<T>(j.a, j.am, j.k, lda), rows_b = exp_rows_of<T>(j.b, j.bn, j.k, ldb);
        const uint32_t a_voff = ACOL ? tid / CA * lda + exp_col_chunk<T, TM>(tid / CA, tid % CA) * 16 : (uint32_t)(tid >> 3) * lda + chunk;
        const uint32_t b_voff = BCOL ? tid / CB * ldb + exp_col_chunk<T, TN>(tid / CB, tid % CB) * 16 : (uint32_t)(tid >> 3) * ldb + chunk;
        const int in_last = (j.k - 1) % KS + 1;
        const bool past = T::ES == 2 && chunk >= in_last * 2; // (of the last step, k-contiguous)
        const uint32_t a_last = !ACOL && past ? NONE : a_voff, b_last = !BCOL && past ? NONE : b_voff;
        const uint32_t a_down = NT / (ACOL ? CA : 8) * lda, b_down = NT / (BCOL ? CB : 8) * ldb;
        auto load = [&](LCMA_LDS char *st, int y) { // a step past the end: zeros, from past the extents
            const uint32_t off = y < steps ? (uint32_t)y * 128 : NONE, av = y == steps - 1 ? a_last : a_voff, bv = y == steps - 1 ? b_last : b_voff;
            const auto ra = ACOL ? exp_columns_from<T>(j.a, j.am, j.k, lda, y, 1) : rows_a, rb = BCOL ? exp_columns_from<T>(j.b, j.bn, j.k, ldb, y, 1) : rows_b;
#pragma unroll
            for (int q = 0; q < QB; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (LCMA_LDS void *)(st + A_STAGE + (q * NT + w * 64) * 16), 16, (int)bv, (int)((BCOL ? 0 : off) + q * b_down), 0, 0);
#pragma unroll
            for (int q = 0; q < QA; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (LCMA_LDS void *)(st + (q * NT + w * 64) * 16), 16, (int)av, (int)((ACOL ? 0 : off) + q * a_down), 0, 0);
        };
        auto step = [&](LCMA_LDS char *st, LCMA_LDS char *before, int y) {
            wait_loads<QA + QB>();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            load(before, y + 2);
            u32x4 a[NMI][4], b[NNI][4];
#pragma unroll
            for (int n = 0; n < NNI; ++n) exp_fragments<T, BCOL, TN>(st + A_STAGE, wn * NNI + n, b[n]);
#pragma unroll
            for (int i = 0; i < NMI; ++i) exp_fragments<T, ACOL, TM>(st, wm * NMI + i, a[i]);
            if (T::ES == 4 && y == steps - 1) {
                if constexpr (!ACOL) exp_end_of_k(a, in_last);
                if constexpr (!BCOL) exp_end_of_k(b, in_last);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < NMI; ++i)
#pragma unroll
                    for (int n = 0; n < NNI; ++n) Mma<T>::run(__builtin_bit_cast(Frag, b[n][k]), __builtin_bit_cast(Frag, a[i][k]), acc[i][n]);
            __builtin_amdgcn_sched_barrier(0); // (the multiplications stay in front of the next wait; what they read has left LDS)
        };
        load(s0, 0);
        load(s1, 1);
        for (int y = 0; y < steps; ++y) {
            step(s0, s2, y);
            if (++y >= steps) break;
            step(s1, s0, y);
            if (++y >= steps) break;
            step(s2, s1, y);
        }
        wait_loads<0>(); // the loads past the end land before the LDS is another work-group's
    }
};

// Few rows: a work-group owns a tile of R x R of C and its waves split K between them, a step (64 k, fp32: 32, 128 bytes of every row) to a wave in turn; nothing is shared between
// waves, so there is no barrier in the loop, and the waves' sums are added at the end, in fp32 and in ascending order (csrc/lcma_few_rows.hpp has the same for one product,
// with the reasons and measurements).  Two steps of a wave in flight.  Bound by memory: bf16, 2 rows of 8 experts, 28672 x 4096: 77 us, 6.1 TB/s, which is what a large read reaches; weights K x N
// 113 (32 columns are half a line; 64 x 64 takes 164).
template <class T, bool BCOL, int R, int WK> struct ExpFewRows {
    static constexpr int KF = 64 / (512 / R), KS = 128 / T::ES; // 16x16x32 or 32x32x16 instructions; fragments of a step along K
    static constexpr int LOADS = R / 8, HALF = R * 128, STAGE = 2 * HALF, PITCH = R + 4, SUMS = WK * R * PITCH * 4, STAGES = WK * 2 * STAGE, LDS_BYTES = SUMS > STAGES ? SUMS : STAGES;
    static_assert((R == 32 || (R == 16 && !BCOL && T::ES == 2)) && LDS_BYTES <= 160 * 1024 && 4 * LOADS <= 63, "LDS budget of one CU; counter of loads");
    using Frag = typename Mma<T>::frag;
    using Acc = std::conditional_t<R == 16, f32x4, f32x16>;
    static constexpr uint32_t NONE = 1u << 30;

    static LCMA_DEV void run(const ExpertsGemmParams &p, LCMA_LDS char *lds) {
        const int lane = threadIdx.x & 63, fr = lane & (R - 1), fk = lane / R, wk = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const I8Rows<R, ExpertsGemmParams> groups(p);
        exp_zero_behind<T, 64 * WK>(p, groups.behind);
        const int nx = groups.within(p), jobs = nx * p.nz, per = (jobs + 7) / 8;
        const int job = (blockIdx.x & 7) * per + (blockIdx.x >> 3); // an eighth of the tiles to every XCD, row tiles that share weights next to each other
        if ((int)(blockIdx.x >> 3) >= per || job >= jobs) return;
        int x, z;
        i8_tile_of_job(nx, p.nz, p.panel, job, x, z);
        const ExpJob j = product_job<T, BCOL, R, R>(p, groups.place(p, x), z * R);
        Acc acc;
#pragma unroll
        for (int v = 0; v < R * R / 64; ++v) acc[v] = 0.f;
        LCMA_LDS char *st = lds + wk * (2 * STAGE);
        steps_of_wave(p, j, wk, acc, st, st + STAGE);
        __syncthreads(); // no load is in flight and every wave has read its last step: the sums take the place of the stages
        LCMA_LDS float *mine = (LCMA_LDS float *)lds + wk * (R * PITCH);
#pragma unroll
        for (int g = 0; g < R * R / 256; ++g) // four neighbouring columns of row fr
            *(LCMA_LDS f32x4 *)(mine + fr * PITCH + g * 8 + fk * 4) = f32x4{acc[g * 4], acc[g * 4 + 1], acc[g * 4 + 2], acc[g * 4 + 3]};
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
    // Steps `y`, y + WK, ...
    static LCMA_DEV void steps_of_wave(const ExpertsGemmParams &p, const ExpJob &j, int y, Acc &acc, LCMA_LDS char *__restrict__ s0, LCMA_LDS char *__restrict__ s1) {
        constexpr int CPR = R * T::ES / 16, RPL = 64 / CPR; // the other form: 16-byte chunks of a row, rows of a load
        const int lane = threadIdx.x & 63, fr = lane & (R - 1), fk = lane / R, steps = (int)(((uint32_t)j.k + (KS - 1)) / KS), in_last = (j.k - 1) % KS + 1;
        const uint32_t lda = (uint32_t)p.lda_b, ldb = (uint32_t)p.ldb_b;
        const auto ra = exp_rows_of<T>(j.a, j.am, j.k, lda), rows_b = exp_rows_of<T>(j.b, j.bn, j.k, ldb);
        // a load brings 8 rows of 128 bytes, lanes 8 i to 8 i + 7 one row; `last`: what is past K from past the extents
        uint32_t av[2], bv[2], al[2], bl[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t c = ((lane & 7) ^ (lane >> 4) ^ (4 * i)) * 16;
            const bool past = T::ES == 2 && c >= (uint32_t)in_last * 2;
            av[i] = (uint32_t)(lane >> 3) * lda + c;
            al[i] = past ? NONE : av[i];
            bv[i] = BCOL ? (uint32_t)(lane / CPR) * ldb + exp_col_chunk<T, R>(lane / CPR, lane % CPR) * 16 : (uint32_t)(lane >> 3) * ldb + c;
            bl[i] = !BCOL && past ? NONE : bv[i];
        }
        auto load = [&](LCMA_LDS char *st, int y) { // a step past the end: zeros, from past the extents
            const uint32_t off = y < steps ? (uint32_t)y * 128 : NONE;
            const bool last = y == steps - 1;
            const auto rb = BCOL ? exp_columns_from<T>(j.b, j.bn, j.k, ldb, y, 1) : rows_b;
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (LCMA_LDS void *)(st + HALF + i * 1024), 16, (int)(last ? bl[i & 1] : bv[i & 1]), (int)(BCOL ? i * RPL * ldb : off + i * 8 * ldb), 0, 0);
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (LCMA_LDS void *)(st + i * 1024), 16, (int)(last ? al[i & 1] : av[i & 1]), (int)(off + i * 8 * lda), 0, 0);
        };
        uint32_t frag[KF]; // of this lane's 16 bytes in k-contiguous rows
#pragma unroll
        for (int k = 0; k < KF; ++k) frag[k] = fr * 128 + ((k * (64 / R) + fk) ^ (fr >> 1 & 7)) * 16;
        auto step = [&](LCMA_LDS char *st, int y) {
            u32x4 a[1][KF], b[1][KF];
            wait_loads<2 * LOADS>();
            if constexpr (BCOL) exp_fragments<T, true, R>(st + HALF, 0, b[0]);
#pragma unroll
            for (int k = 0; k < KF; ++k) {
                a[0][k] = *(const LCMA_LDS u32x4 *)(st + frag[k]);
                if constexpr (!BCOL) b[0][k] = *(const LCMA_LDS u32x4 *)(st + HALF + frag[k]);
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0xC07F); // lgkmcnt(0): what was read has left LDS, so its place may be loaded anew
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            load(st, y + 2 * WK);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (T::ES == 4)
                if (y == steps - 1) {
                    exp_end_of_k(a, in_last);
                    if constexpr (!BCOL) exp_end_of_k(b, in_last);
                }
#pragma unroll
            for (int k = 0; k < KF; ++k) {
                const Frag fa = __builtin_bit_cast(Frag, a[0][k]), fb = __builtin_bit_cast(Frag, b[0][k]);
                if constexpr (R == 16) acc = Mma16<T>::run(fb, fa, acc);
                else Mma<T>::run(fb, fa, acc);
            }
        };
        load(s0, y);
        load(s1, y + WK);
        for (; y < steps; y += WK) {
            step(s0, y);
            if ((y += WK) >= steps) break;
            step(s1, y);
        }
        wait_loads<0>();
    }
};

} // namespace lcma
