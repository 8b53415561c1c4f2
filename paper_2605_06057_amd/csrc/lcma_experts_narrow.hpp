// The experts' products in 16 bit on tiles of 128 x 256, two groups of waves in turn (csrc/lcma_i8_narrow.hpp does so for 8-bit integers): for experts with fewer rows than a
// 256 x 256 tile has, and where there are too few of those to fill the chip or to end its last round.  Wave tiles of 64 x 64, the two groups below each other; a step of 64 k is two
// phases (the upper and the lower 32 rows of the wave tile) of eight matrix instructions.  Loads go two whole steps ahead into one of three stages (144 KB), and the wait
// for them is the count of one step's.  Work-groups walk through tiles and the loads run on into the next one; so that every tile starts in the first stage its steps are rounded up to
// threes by steps that load zeros and multiply nothing.  K x N weights lie in LDS in halves of 128 columns.
// fp16, 1021 x 6 of 64, 2816 x 2056: 213 us, 333 TFLOP/s and the weights at 3.5 TB/s (256 x 256 as fast, 64 x 128 takes 255); gradient of the rows 196 against 208 and 225.  An expert has about a hundred
// rows: half the tile's sums are dropped, and what bounds it is the weights' way in, of which each work-group has two steps in flight; weights four waves' own, five steps ahead, took 215 where this took 190,
// straight into registers 222 to 249.
#pragma once
#include "lcma_experts_pingpong.hpp"

namespace lcma {

template <class T, bool BCOL> struct ExpNarrow {
    using Turns = ExpPingPong<T, false, BCOL, false>;
    using Args = typename Turns::Args;
    using Frag = typename Mma<T>::frag;
    static constexpr int NT = 512, TM = 128, TN = 256, NK = 4, KS = 64, HALF = 128 * 128, STAGE = 3 * HALF, STRIP = 16 * 128, LDS_BYTES = 3 * STAGE + 8 * STRIP;
    static_assert(LDS_BYTES <= 160 * 1024 && T::ES == 2, "LDS budget of one CU");
    static constexpr uint32_t NONE = 1u << 30; // an offset past any extent

    static LCMA_DEV void multiply(const u32x4 (&a)[NK], const u32x4 (&b)[2][NK], f32x16 (&c)[2]) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            Mma<T>::run(__builtin_bit_cast(Frag, b[0][k]), __builtin_bit_cast(Frag, a[k]), c[0]);
            Mma<T>::run(__builtin_bit_cast(Frag, b[1][k]), __builtin_bit_cast(Frag, a[k]), c[1]);
        }
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
    }
    static LCMA_DEV void run(LCMA_LDS char *lds) { // (the argument block has to be the kernel's first argument)
        pipeline((Args)__builtin_amdgcn_kernarg_segment_ptr(), lds, lds + STAGE, lds + 2 * STAGE, lds + 3 * STAGE);
    }
    // restrict: the loads in flight towards one stage do not touch what is read from another (the compiler would otherwise wait for all of them in
    // front of every read)
    static LCMA_DEV void pipeline(Args args, LCMA_LDS char *__restrict__ s0, LCMA_LDS char *__restrict__ s1, LCMA_LDS char *__restrict__ s2, LCMA_LDS char *__restrict__ strips) {
        const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w >> 2, wn = w & 3; // (wm: also the group; waves w and w + 4 share a SIMD)
        int nx, jobs;
        {
            const ExpertsGemmParams p = Turns::arguments(args);
            const I8Rows<TM, ExpertsGemmParams> groups(p);
            exp_zero_behind<T, NT>(p, groups.behind);
            nx = groups.within(p);
            jobs = nx * p.nz;
        }
        const int units = gridDim.x, per = units >> 3; // rounds of one tile per work-group, as in ExpPingPong
        const int unit = (int)blockIdx.x < (per << 3) ? (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
        const int whole = jobs / units * units;
        int job = unit < whole ? unit : (int)blockIdx.x;
        if (job >= jobs) return;
        const uint32_t lda = (uint32_t)args->lda_b, ldb = (uint32_t)args->ldb_b;
        // load q of a thread fills row q * 64 + tid / 8 of an operand, position tid % 8; where B's columns are contiguous row (k) q % 2 * 32 + tid / 16 of half q / 2, position tid % 16
        const int row = tid >> 3, pos = exp_row_chunk(row, tid & 7), k16 = tid >> 4, pos16 = exp_col_chunk<T, 128>(k16, tid & 15);
        const uint32_t a_voff = row * lda + pos * 16, b_voff = BCOL ? k16 * ldb + pos16 * 16 : row * ldb + pos * 16;
        using Source = typename Turns::Source;
        auto source = [&](int job) { return Turns::template source<TM, TN>(args, nx, jobs, job); };
        Source cur = source(job), nxt;
        auto steps_of = [&](int k) { return k > KS ? (int)(((uint32_t)k + (KS - 1)) / KS) : 1; };
        // loads FROM .. TO of step y: first those of A, then those of B
        auto load = [&](auto from, auto to, const Source &s, LCMA_LDS char *st, int y) {
            const int ny = steps_of(s.k);
            const uint32_t off = y < ny ? (uint32_t)y * 128 : NONE;
            const bool past = y == ny - 1 && (uint32_t)pos * 8 >= (uint32_t)((s.k - 1) % KS + 1); // 16 bytes past the last k
            const uint32_t av = past ? NONE : a_voff, bv = !BCOL && past ? NONE : b_voff;
            const auto ra = exp_rows_of<T>(s.a, s.am, s.k, lda);
            const auto rb = BCOL ? exp_columns_from<T>(s.b, s.bn, s.k, ldb, y, 1) : exp_rows_of<T>(s.b, s.bn, s.k, ldb);
#pragma unroll
            for (int q = from; q < to; ++q) {
                const int i = q - 2; // of B
                if (q < 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (LCMA_LDS void *)(st + (q * NT + w * 64) * 16), 16, (int)av, (int)(off + q * 64 * lda), 0, 0);
                else __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (LCMA_LDS void *)(st + (q * NT + w * 64) * 16), 16, (int)bv, (int)(BCOL ? i % 2 * 32 * ldb + i / 2 * 256 : off + i * 64 * ldb), 0, 0);
            }
        };
        constexpr std::integral_constant<int, 0> c0{};
        constexpr std::integral_constant<int, 3> c3{};
        constexpr std::integral_constant<int, 6> c6{};
        load(c0, c6, cur, s0, 0);
        load(c0, c6, cur, s1, 1);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0076); // vmcnt(6)
        Turns::slot_end();
        if (wm) Turns::slot_end(); // the second group runs one slot behind the first
        f32x16 acc[2][2];
        u32x4 a[NK], b[2][NK];
        auto read_a = [&](const LCMA_LDS char *st, int i) { exp_fragments<T, false, 128>(st, wm * 2 + i, a); };
        auto read_b = [&](const LCMA_LDS char *st) { // (columns: two waves to a half)
            if constexpr (BCOL) {
                exp_columns_pair<T, 128>(st + HALF + (wn >> 1) * HALF, (wn & 1) * 2, b[0], b[1]);
            } else {
                exp_fragments<T, false, 256>(st + HALF, wn * 2, b[0]);
                exp_fragments<T, false, 256>(st + HALF, wn * 2 + 1, b[1]);
            }
        };
        // one step out of stage st; `of`, y2: the step two on, which goes into the stage that the step before has read.  (Reads that wait for their results: behind the loads.)
        auto step = [&](bool real, LCMA_LDS char *st, LCMA_LDS char *into, const Source &of, int y2) {
            if (real) {
                read_a(st, 0);
                if constexpr (!BCOL) read_b(st);
            }
            load(c0, c3, of, into, y2);
            if constexpr (BCOL)
                if (real) read_b(st);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0xC07F); // lgkmcnt(0)
            Turns::slot_end();
            if (real) multiply(a, b, acc[0]);
            Turns::slot_end();
            if (real) read_a(st, 1);
            load(c3, c6, of, into, y2);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0x0076); // vmcnt(6) lgkmcnt(0): the next step has landed
            Turns::slot_end();
            if (real) multiply(a, b, acc[1]);
        };
        while (true) {
            int next = job + units;
            if (next >= whole && job < whole && whole < jobs) next = whole + (int)blockIdx.x;
            nxt = source(next);
            const int ny = steps_of(cur.k), n3 = (ny + 2) / 3 * 3;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) zero(acc[i][j]);
            for (int y = 0;;) {
                const bool in = y + 3 < n3;
                const Source of = {in ? cur.a : nxt.a, in ? cur.b : nxt.b, nullptr, in ? cur.am : nxt.am, in ? cur.bn : nxt.bn, in ? cur.k : nxt.k};
                step(true, s0, s2, cur, y + 2);
                Turns::slot_end();
                step(y + 1 < ny, s1, s0, of, in ? y + 3 : 0);
                Turns::slot_end();
                step(y + 2 < ny, s2, s1, of, in ? y + 4 : 1);
                y += 3;
                if (y >= n3) break;
                Turns::slot_end();
            }
            if (!wm) Turns::slot_end(); // both groups write their halves of the tile in one slot
            if (next >= jobs) __builtin_amdgcn_s_waitcnt(0x0070); // loads past the end land before the LDS is another work-group's
            {
                const int64_t ldc_b = Turns::arguments(args).ldc_b;
                const int r0 = wm * 64, n0 = wn * 64;
                exp_store<T, 2, 2, false, 32, 16>(strips + w * STRIP, cur.c + r0 * ldc_b + n0 * T::ES, ldc_b, cur.am - r0, cur.bn - n0, acc);
            }
            if (wm) Turns::slot_end();
            if (next >= jobs) break;
            job = next;
            cur = nxt;
        }
        if (!wm) Turns::slot_end();
    }
};

} // namespace lcma
