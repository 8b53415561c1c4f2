// The 8-bit-integer product on tiles of 128 x 256, two groups of waves in turn: for fewer rows (of an expert) than a 256 x 256 tile has, and
// where there are too few of those to fill the chip or to end its last round.  Wave tiles of 64 x 64, the two groups one beside the other; a step of 128 k is
// two phases (the upper and the lower 32 rows of the wave tile) of eight matrix instructions.  What bounds it is what a CU can take in, 48 KB a step, and
// the LDS (48 KB written, 128 KB read for 1024 cycles of matrix instructions): so loads go two whole steps ahead into one of three stages (144 KB), and
// the wait for them is the count of one step's.  (Eight fragment reads in front of either phase instead of twelve and four: the next step has to have landed
// half a step earlier, 2048 x 4096 x 14336 113 -> 120 us.)
// Measured (us, bf16 results; 256 x 256 / this): 2048 x 4096 x 14336 134 / 111 (2170 TOP/s), 2048 x 4096 x 4096 40 / 35, 512 x 14336 x 4096 48 / 37, 1000 rows of 8
// experts x 4096 x 4096 42 / 35; 4096^3 58 / 70.  Work-groups walk through tiles as in csrc/lcma_i8_pingpong.hpp and the loads run on into the
// next one; so that every tile starts in the first stage its steps are rounded up to threes by steps that load zeros and multiply nothing.
#pragma once
#include "lcma_i8_pingpong.hpp"

namespace lcma {

template <class OUT> struct I8Narrow : I8Turns {
    static constexpr int TM = 128, TN = 256, A_STAGE = TM * ROW, STAGE = (TM + TN) * ROW, STRIP = 16 * 128, LDS_BYTES = 3 * STAGE + 8 * STRIP;
    static constexpr int LA = TM / 64, LB = TN / 64; // direct loads of a thread for a step
    static_assert(LDS_BYTES <= 160 * 1024, "LDS budget of one CU");

    static LCMA_DEV void multiply(const i32x4 (&a)[NK], const i32x4 (&b)[2][NK], i32x16 (&c)[2]) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            c[0] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[0][k], a[k], c[0], 0, 0, 0);
            c[1] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[1][k], a[k], c[1], 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
    }
    static LCMA_DEV void run(LCMA_LDS char *lds) { // (the argument block has to be the kernel's first argument)
        pipeline((Args)__builtin_amdgcn_kernarg_segment_ptr(), lds, lds + STAGE, lds + 2 * STAGE, lds + 3 * STAGE);
    }
    // restrict: the loads in flight towards one stage do not touch what is read from another (the compiler would otherwise wait for all of them in
    // front of every read)
    static LCMA_DEV void pipeline(Args args, LCMA_LDS char *__restrict__ s0, LCMA_LDS char *__restrict__ s1, LCMA_LDS char *__restrict__ s2,
                                  LCMA_LDS char *__restrict__ strips) {
        const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = tid & 31, lh = (tid >> 5) & 1;
        const int wm = w >> 2, wn = w & 3, g = wm; // the wave's place among 2 x 4 wave tiles, its group; waves w and w + 4 share a SIMD
        int nx, jobs;
        {
            const I8GemmParams p = arguments(args);
            const I8Rows<TM> groups(p);
            i8_zero_behind<OUT>(p, groups.behind, gridDim.x, NT);
            nx = groups.tiles;
            jobs = nx * p.nz;
        }
        const int units = gridDim.x, per = units >> 3; // rounds of one tile per work-group, as in I8PingPong
        const int unit = (int)blockIdx.x < (per << 3) ? (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
        const int whole = jobs / units * units;
        int job = unit < whole ? unit : (int)blockIdx.x;
        if (job >= jobs) return;
        const int pitch = args->pitch, ny = args->steps, n3 = (ny + 2) / 3 * 3;
        const uint32_t voff = (uint32_t)(tid >> 3) * pitch + swz(tid >> 3, tid & 7) * 16, rows = 64 * pitch;
        uint32_t fa[NK], fb[NK];
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            const int ar = wm * 64 + l32, br = wn * 64 + l32;
            fa[k] = ar * ROW + swz(ar, k * 2 + lh) * 16;
            fb[k] = A_STAGE + br * ROW + swz(br, k * 2 + lh) * 16;
        }
        I8Place at, at_next;
        Source cur = source<TM, TN>(args, nx, jobs, jobs, job, at), nxt;
        // loads FROM .. TO of a step: first those of A, then those of B
        auto load = [&](auto from, auto to, const Source &s, LCMA_LDS char *st, int y) {
            const auto ra = rsrc(s.a, s.a_bytes), rb = rsrc(s.b, s.b_bytes);
            const uint32_t off = y < ny ? (uint32_t)y * ROW : NONE;
#pragma unroll
            for (int q = from; q < to; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(q < LA ? ra : rb, (LCMA_LDS void *)(st + (q * NT + w * 64) * 16), 16, (int)voff,
                                                         (int)(off + (q < LA ? q : q - LA) * rows), 0, 0);
        };
        constexpr std::integral_constant<int, 0> c0{};
        constexpr std::integral_constant<int, 3> c3{};
        constexpr std::integral_constant<int, 6> c6{};
        load(c0, c6, cur, s0, 0);
        load(c0, c6, cur, s1, 1);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0076); // vmcnt(6)
        slot_end();
        if (g) slot_end(); // the second group runs one slot behind the first
        i32x16 acc[2][2];
        i32x4 a[NK], b[2][NK];
        // one step out of stage st; `of`, y2: the step two on, which goes into the stage that the step before has read
        auto step = [&](bool real, LCMA_LDS char *st, LCMA_LDS char *into, const Source &of, int y2) {
            if (real) {
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    a[k] = *(const LCMA_LDS i32x4 *)(st + fa[k]);
                    b[0][k] = *(const LCMA_LDS i32x4 *)(st + fb[k]);
                    b[1][k] = *(const LCMA_LDS i32x4 *)(st + fb[k] + 32 * ROW);
                }
            }
            load(c0, c3, of, into, y2);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0xC07F); // lgkmcnt(0)
            slot_end();
            if (real) multiply(a, b, acc[0]);
            slot_end();
            if (real) {
#pragma unroll
                for (int k = 0; k < NK; ++k) a[k] = *(const LCMA_LDS i32x4 *)(st + fa[k] + 32 * ROW);
            }
            load(c3, c6, of, into, y2);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0x0076); // vmcnt(6) lgkmcnt(0): the next step has landed
            slot_end();
            if (real) multiply(a, b, acc[1]);
        };
        while (true) {
            int next = job + units;
            if (next >= whole && job < whole && whole < jobs) next = whole + (int)blockIdx.x;
            nxt = source<TM, TN>(args, nx, jobs, jobs, next, at_next);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
            for (int y = 0;;) {
                const bool in = y + 3 < n3;
                const Source of = {in ? cur.a : nxt.a, in ? cur.b : nxt.b, in ? cur.a_bytes : nxt.a_bytes, in ? cur.b_bytes : nxt.b_bytes};
                step(true, s0, s2, cur, y + 2);
                slot_end();
                step(y + 1 < ny, s1, s0, of, in ? y + 3 : 0);
                slot_end();
                step(y + 2 < ny, s2, s1, of, in ? y + 4 : 1);
                y += 3;
                if (y >= n3) break;
                slot_end();
            }
            if (!g) slot_end(); // both groups write their halves of the tile in one slot
            if (next >= jobs) __builtin_amdgcn_s_waitcnt(0x0070); // loads past the end land before the LDS is another work-group's
            {
                const I8GemmParams p = arguments(args);
                i8_store_part<OUT, 2, 16>(p, strips + w * STRIP, at, wm * 64, wn * 64, acc);
            }
            if (g) slot_end();
            if (next >= jobs) break;
            job = next;
            cur = nxt;
            at = at_next;
        }
        if (!g) slot_end();
    }
};

} // namespace lcma
