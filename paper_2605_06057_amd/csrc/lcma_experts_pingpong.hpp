// The experts' products in 16 bit on tiles of 256 x 256, the two waves of every SIMD in turn: what csrc/lcma_pingpong.hpp does for one product (phases, slots, waits and the
// placing of the operand halves are described there), for rows in groups, either form of both operands (csrc/lcma_experts.hpp), 64-bit bases, and as many steps as the rows of
// an expert take (the gradient).
// Half h of a k-contiguous operand holds the tile's rows 128 wm + 64 h .. + 63 of both wm (right operand: 64 wn + 32 h .. + 31 of all wn); of the other form it holds the columns
// 128 h .. + 127, so a wave has rows 64 wm .. + 63 of both halves (right operand: columns 32 wn .. + 31).  LINES (gradients of few rows, which their stores bound): the right operand
// is cut as a k-contiguous one all the same, so that a wave's 64 columns of C lie together and leave as whole lines, past the caches where they are such in memory; what it costs is loads of half lines
// (1021 x 6 of 64, 2816 x 2048: 226 -> 179 us, 2816 x 2056, off lines: 272 -> 260; 1024 x 2 of 8, 4096 x 14336: 402 -> 324, but with 8192 tokens 1529 -> 1596; weights K x N, which come from
// memory: 3 to 14 % slower).  What lies past a tile's rows or columns may be anything: it
// reaches elements of C alone that are not there.  What lies past the last k reads as zero, on both sides: k-contiguous, 16 bytes at a time from past the extent; else by the extent.
// Every work-group walks through tiles of its own, in turn; the loads run two steps ahead, into the next tile too.
// Bound by power, as one large product: bf16, 8192 x 2 of 8, 4096 x 14336: 1620 us, 1.19 PFLOP/s (128 x 256 takes 1960, 64 x 128 2790), gradients 1550 and 1570; the matrix pipe is at work in 83, 83 and
// 71 % of the clocks, of which there are 1.5 to 1.8 in a nanosecond.
#pragma once
#include "lcma_experts_ring.hpp"

namespace lcma {

template <class T, bool ACOL, bool BCOL, bool GRAD, bool LINES = false> struct ExpPingPong {
    static constexpr int NT = 512, ROW = 128, NK = 4, TM = 256, TN = 256, NMI = 4, NNI = 2, KS = 64;
    static constexpr int HALF = 128 * ROW, LDS_BYTES = 8 * HALF + 8 * 4096;
    static constexpr int B_GAP = BCOL && !LINES ? 128 : 32; // columns of C from a wave's first 32 to its others
    static_assert(LDS_BYTES <= 160 * 1024 && T::ES == 2 && (GRAD || !LINES), "LDS budget of one CU");
    static constexpr uint32_t NONE = 1u << 30; // an offset past any extent
    using Frag = typename Mma<T>::frag;
    typedef const __attribute__((address_space(4))) ExpertsGemmParams *Args;

    // (the argument block is read where it is needed: its fields, kept through the steps, would push the offsets of the loads out of the scalar registers)
    static LCMA_DEV ExpertsGemmParams arguments(Args at) {
        asm volatile("" : "+s"(at));
        return ExpertsGemmParams{at->A, at->B, at->C, at->offsets, at->lda_b, at->ldb_b, at->ldc_b, at->expert_b, at->rows, at->M, at->N, at->K, at->experts, at->nx, at->nz, at->panel, at->stream};
    }
    static LCMA_DEV void slot_end() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    }
    // lgkmcnt(0), vmcnt(12): the fragments are read, and all but the six youngest pairs of loads have landed
    static LCMA_DEV void memory_slot_end() {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x007C);
        slot_end();
    }
    static LCMA_DEV void load_half(__amdgpu_buffer_rsrc_t r, LCMA_LDS char *dst, int wave_chunk, uint32_t voff, uint32_t off, uint32_t rows) {
#pragma unroll
        for (int q = 0; q < 2; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LCMA_LDS void *)(dst + (q * NT + wave_chunk) * 16), 16, (int)voff, (int)(off + q * rows), 0, 0);
    }
    // A half's fragments of 32 rows: block i of a wave's two (left operand), or its one.
    template <bool COL> static LCMA_DEV void read(const LCMA_LDS char *half, int block, u32x4 (&f)[NK]) { exp_fragments<T, COL, 128>(half, block, f); }
    static LCMA_DEV void multiply(const u32x4 (&a)[2][NK], const u32x4 (&b)[NK], f32x16 &c0, f32x16 &c1) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            Mma<T>::run(__builtin_bit_cast(Frag, b[k]), __builtin_bit_cast(Frag, a[0][k]), c0);
            Mma<T>::run(__builtin_bit_cast(Frag, b[k]), __builtin_bit_cast(Frag, a[1][k]), c1);
        }
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
    }

    // Where the operands of a tile are: bases, and what there is of them (k: 0 without a tile: nothing is read then).
    struct Source {
        const char *a, *b;
        char *c;
        int am, bn, k;
    };
    template <int TM, int TN> static LCMA_DEV Source source(Args args, int nx, int jobs, int job) {
        ExpJob j = {nullptr, nullptr, nullptr, 0, 0, 0};
        if (job < jobs) {
            const ExpertsGemmParams p = arguments(args);
            if constexpr (GRAD) {
                j = gradient_job<T, TM, TN>(p, job);
            } else {
                int x, z;
                i8_tile_of_job(nx, p.nz, p.panel, job, x, z);
                j = product_job<T, BCOL, TM, TN>(p, I8Rows<TM, ExpertsGemmParams>(p).place(p, x), z * TN);
            }
        }
        // (uniform anyway; said here so that the descriptors stay in scalar registers)
        return {exp_uniform(j.a), exp_uniform(j.b), exp_uniform(j.c), __builtin_amdgcn_readfirstlane(j.am), __builtin_amdgcn_readfirstlane(j.bn), __builtin_amdgcn_readfirstlane(j.k)};
    }
    // The operand from step y on, for two steps: k-contiguous rows with their steps as offsets, or the rows of the stored matrix from k = 64 y on.
    template <bool COL> static LCMA_DEV __amdgpu_buffer_rsrc_t operand(const char *at, int wide, int k, uint32_t ld_b, int y) {
        if constexpr (COL) return exp_columns_from<T>(at, wide, k, ld_b, y, 2);
        else return exp_rows_of<T>(at, wide, k, ld_b);
    }

    static LCMA_DEV void run(LCMA_LDS char *lds) { // (the argument block has to be the kernel's first argument)
        pipeline((Args)__builtin_amdgcn_kernarg_segment_ptr(), lds, lds + HALF, lds + 2 * HALF, lds + 3 * HALF, lds + 4 * HALF, lds + 5 * HALF, lds + 6 * HALF, lds + 7 * HALF,
                 lds + 8 * HALF);
    }

    // restrict: the loads in flight towards one half do not touch what is read from another, without which the compiler waits for all of them in front of every read.
    static LCMA_DEV void pipeline(Args args, LCMA_LDS char *__restrict__ A00, LCMA_LDS char *__restrict__ A10, LCMA_LDS char *__restrict__ A01,
                                  LCMA_LDS char *__restrict__ A11, LCMA_LDS char *__restrict__ B00, LCMA_LDS char *__restrict__ B10,
                                  LCMA_LDS char *__restrict__ B01, LCMA_LDS char *__restrict__ B11, LCMA_LDS char *__restrict__ strips) {
        const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w >> 2, wn = w & 3, wave_chunk = w * 64;
        int nx, jobs;
        {
            const ExpertsGemmParams p = arguments(args);
            if constexpr (GRAD) {
                nx = p.nx;
                jobs = p.experts * p.nx * p.nz;
            } else {
                const I8Rows<TM, ExpertsGemmParams> groups(p);
                exp_zero_behind<T, NT>(p, groups.behind);
                nx = groups.within(p);
                jobs = nx * p.nz;
            }
        }
        const int units = gridDim.x;
        // tiles in rounds of one per work-group; inside a round an XCD (work-groups go to the eight in turn) has consecutive ones
        const int per = units >> 3;
        const int unit = (int)blockIdx.x < (per << 3) ? (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
        const int whole = jobs / units * units;
        int job = unit < whole ? unit : (int)blockIdx.x;
        if (job >= jobs) return;
        const uint32_t lda = (uint32_t)args->lda_b, ldb = (uint32_t)args->ldb_b;
        // load q of a thread fills row q * 64 + tid / 8 of a half, position tid % 8; of the other form row (k) q * 32 + tid / 16, position tid % 16 (LINES, right
        // operand: four chunks of every 64 columns)
        const int row = tid >> 3, pos = exp_row_chunk(row, tid & 7), k16 = tid >> 4, pos16 = exp_col_chunk<T, 128>(k16, tid & 15);
        const uint32_t a_voff = ACOL ? k16 * lda + pos16 * 16 : row * lda + pos * 16, b_voff = BCOL ? k16 * ldb + (LINES ? (pos16 >> 2) * 128 + (pos16 & 3) * 16 : pos16 * 16) : (uint32_t)((row >> 5) * 64 + (row & 31)) * ldb + pos * 16;
        const uint32_t a_rows = (ACOL ? 32 : 128) * lda, b_rows = (BCOL ? 32 : 128) * ldb, a_half = ACOL ? 256 : 64 * lda, b_half = LINES ? 64 : BCOL ? 256 : 32 * ldb;
        const uint32_t a_step = ACOL ? KS * lda : ROW, b_step = BCOL ? KS * ldb : ROW;
        // k-contiguous: the 16 bytes past the last k in the last step, read from past the extent
        auto last_voff = [&](bool col, uint32_t voff, int k) { return !col && (uint32_t)pos * 8 >= (uint32_t)((k - 1) % KS + 1) ? NONE : voff; };
        Source cur = source<TM, TN>(args, nx, jobs, job), nxt;
        u32x4 fa0[2][NK], fa1[2][NK], fb0[NK], fb1[NK];
        f32x16 acc[NMI][NNI];
        auto read_a = [&](const LCMA_LDS char *half, u32x4 (&f)[2][NK]) {
            if constexpr (ACOL) {
                exp_columns_pair<T, 128>(half, wm * 2, f[0], f[1]);
            } else {
                read<false>(half, wm * 2, f[0]);
                read<false>(half, wm * 2 + 1, f[1]);
            }
        };
        auto read_b = [&](const LCMA_LDS char *half, u32x4 (&f)[NK]) { read<BCOL>(half, wn, f); };
        auto steps_of = [&](int k) { return k > KS ? (int)(((uint32_t)k + (KS - 1)) / KS) : 1; };
        auto load_step = [&](__amdgpu_buffer_rsrc_t ra, __amdgpu_buffer_rsrc_t rb, LCMA_LDS char *A0, LCMA_LDS char *A1, LCMA_LDS char *B0, LCMA_LDS char *B1, uint32_t av, uint32_t bv,
                             uint32_t a, uint32_t b) {
            load_half(rb, B0, wave_chunk, bv, b, b_rows);
            load_half(ra, A0, wave_chunk, av, a, a_rows);
            load_half(ra, A1, wave_chunk, av, a + a_half, a_rows);
            load_half(rb, B1, wave_chunk, bv, b + b_half, b_rows);
        };
        {
            const int ny = steps_of(cur.k);
            const auto ra = operand<ACOL>(cur.a, cur.am, cur.k, lda, 0), rb = operand<BCOL>(cur.b, cur.bn, cur.k, ldb, 0);
            const uint32_t al = last_voff(ACOL, a_voff, cur.k), bl = last_voff(BCOL, b_voff, cur.k);
            load_step(ra, rb, A00, A10, B00, B10, ny == 1 ? al : a_voff, ny == 1 ? bl : b_voff, 0, 0);
            load_step(ra, rb, A01, A11, B01, B11, ny == 2 ? al : a_voff, ny == 2 ? bl : b_voff, ny > 1 ? a_step : NONE, ny > 1 ? b_step : NONE);
        }
        memory_slot_end();
        read_b(B00, fb0);
        memory_slot_end();
        if (wm) slot_end(); // the second group runs one slot behind the first
        while (true) {
            int next = job + units;
            if (next >= whole && job < whole && whole < jobs) next = whole + (int)blockIdx.x;
            nxt = source<TM, TN>(args, nx, jobs, next);
            const int ny = steps_of(cur.k), n2 = (ny + 1) & ~1, ny_next = steps_of(nxt.k);
#pragma unroll
            for (int mi = 0; mi < NMI; ++mi)
#pragma unroll
                for (int ni = 0; ni < NNI; ++ni) zero(acc[mi][ni]);
            for (int y = 0;;) {
                const bool in = y + 2 < n2;
                const int from = in ? y + 2 : 0, of = in ? ny : ny_next, k = in ? cur.k : nxt.k; // the two steps whose loads go out: of this tile or of the next
                const auto ra = operand<ACOL>(in ? cur.a : nxt.a, in ? cur.am : nxt.am, k, lda, from), rb = operand<BCOL>(in ? cur.b : nxt.b, in ? cur.bn : nxt.bn, k, ldb, from);
                const uint32_t a_off = ACOL ? 0 : (uint32_t)from * ROW, b_off = BCOL ? 0 : (uint32_t)from * ROW;
                // one step out of stage (A0, A1, B0, B1); nextB0: half 0 of B of the next step; av, bv, a, b: of the loads into this stage
                auto step = [&](LCMA_LDS char *A0, LCMA_LDS char *A1, LCMA_LDS char *B0, LCMA_LDS char *B1, LCMA_LDS char *nextB0, uint32_t av, uint32_t bv, uint32_t a, uint32_t b) {
                    if constexpr (!ACOL) read_a(A0, fa0);
                    load_half(rb, B0, wave_chunk, bv, b, b_rows);
                    if constexpr (ACOL) read_a(A0, fa0); // (these wait for their results: behind the loads)
                    memory_slot_end();
                    multiply(fa0, fb0, acc[0][0], acc[1][0]);
                    slot_end();
                    if constexpr (!ACOL) read_a(A1, fa1);
                    load_half(ra, A0, wave_chunk, av, a, a_rows);
                    if constexpr (ACOL) read_a(A1, fa1);
                    memory_slot_end();
                    multiply(fa1, fb0, acc[2][0], acc[3][0]);
                    slot_end();
                    if constexpr (!BCOL) read_b(B1, fb1);
                    load_half(ra, A1, wave_chunk, av, a + a_half, a_rows);
                    if constexpr (BCOL) read_b(B1, fb1);
                    memory_slot_end();
                    multiply(fa1, fb1, acc[2][1], acc[3][1]);
                    slot_end();
                    if constexpr (!BCOL) read_b(nextB0, fb0);
                    load_half(rb, B1, wave_chunk, bv, b + b_half, b_rows);
                    if constexpr (BCOL) read_b(nextB0, fb0);
                    memory_slot_end();
                    multiply(fa0, fb1, acc[0][1], acc[1][1]);
                };
                const bool l0 = from + 1 == of, l1 = from + 2 == of, none = from + 1 >= of; // (an odd number of steps: one of zeros behind)
                const uint32_t al = last_voff(ACOL, a_voff, k), bl = last_voff(BCOL, b_voff, k);
                step(A00, A10, B00, B10, B01, l0 ? al : a_voff, l0 ? bl : b_voff, a_off, b_off);
                slot_end();
                step(A01, A11, B01, B11, B00, l1 ? al : a_voff, l1 ? bl : b_voff, none ? NONE : a_off + a_step, none ? NONE : b_off + b_step);
                y += 2;
                if (y >= n2) break;
                slot_end();
            }
            if (!wm) slot_end(); // both groups write their halves of the tile in one slot
            if (next >= jobs) __builtin_amdgcn_s_waitcnt(0x0070); // loads past the end land before the LDS is another work-group's
            {
                const ExpertsGemmParams p = arguments(args);
                const int64_t ldc_b = p.ldc_b;
                const int r0 = wm * (ACOL ? 64 : 128), c0 = wn * (B_GAP == 128 ? 32 : 64);
                exp_store<T, NMI, NNI, ACOL, B_GAP, 32, LINES>(strips + w * 4096, cur.c + r0 * ldc_b + c0 * T::ES, ldc_b, cur.am - r0, cur.bn - c0, acc, p.stream);
            }
            if (wm) slot_end();
            if (next >= jobs) break;
            job = next;
            cur = nxt;
        }
        if (!wm) slot_end();
    }
};

} // namespace lcma
