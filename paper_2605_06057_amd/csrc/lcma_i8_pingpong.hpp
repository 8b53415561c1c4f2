// The 8-bit-integer product on tiles of 256 x 256, the two waves of every SIMD in turn: what csrc/lcma_pingpong.hpp does for 16-bit and FP8
// operands (phases, slots, waits and the placing of the operand halves are described there), with 32-bit integer accumulators, the tiles
// of groups of rows, and 64-bit bases.
//
// What bounds it: a step of 128 k is 2048 cycles of matrix instructions per SIMD against 192 KB of fragment reads (1536 clocks) and 64 KB of direct loads (820) of the
// LDS, and beyond about a hundred work-groups power: a step takes 0.98 us on 64 CUs and 1.4 to 1.7 on 256, where the chip runs at 1.6 GHz with the matrix pipe
// 71 % busy (8192 x 14336 x 4096; 2.2 GHz under the tiles of 128 x 256).
// Measured (us, bf16 results): 8192 x 14336 x 4096 385 to 400 (2400 to 2500 TOP/s; 520 at worst between 2 and 20 ms after a pause, while the power is being held; operands of zeros, which spare it, 287; the vendor's 32-bit product of the same codes 506), 4096^3
// 58, 16384 x 4096 x 14336 715 (2690 TOP/s), 16384 rows of 8 experts x 28672 x 4096 1600, 8192 of 8 x 4096 x 14336 449.
// Tried and not kept: the next tile's scales through LDS, with strips of 16 rows to make room (0.5 to 1 % slower).
// Every work-group walks through tiles of its own, in turn; the loads run two steps ahead, into the next tile too.  The descriptors of the
// operands are made anew for every pair of steps, from scalars: a tile's own rows, so that groups may start anywhere and matrices be of any size.
// The weights are the left operand of the matrix instruction: a lane then holds four neighbouring columns of a row, which are scaled, rounded and
// written to the wave's strip of LDS (32 rows of 128 bytes) at once, and leave it as whole lines.
#pragma once
#include "lcma_i8.hpp"

namespace lcma {

// What the kernels have in common in which work-groups walk through tiles and two groups of waves take turns.
struct I8Turns {
    static constexpr int NT = 512, ROW = 128, NK = 4;
    static LCMA_DEV constexpr int swz(int row, int c) { return c ^ ((row >> 1) & 7); } // position of 16-byte chunk c of a row in LDS

    // The end of a slot.  (Not __syncthreads(): its fences would wait for the loads in flight.  The scheduling barriers keep matrix instructions, which
    // touch no memory, in their slot.)
    static LCMA_DEV void slot_end() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    }

    // The argument block is read where it is needed: kept in scalar registers through the steps, its fields would push the offsets of the loads out
    // of them (and the compiler then loops over the lanes of each load).
    typedef const __attribute__((address_space(4))) I8GemmParams *Args;
    static LCMA_DEV I8GemmParams arguments(Args at) {
        asm volatile("" : "+s"(at));
        return I8GemmParams{at->A, at->W, at->SA, at->SW, at->bias, at->C, at->offsets, at->ldc, at->rows, at->N, at->pitch, at->experts, at->steps, at->nz, at->panel};
    }

    // Where the operands of a tile are: bases, and extents in bytes (0: no tile, all reads are past the end).
    struct Source {
        const int8_t *a, *b;
        int a_bytes, b_bytes;
    };
    static LCMA_DEV const int8_t *uniform(const int8_t *at) {
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)at >> 32));
        return (const int8_t *)((uint64_t)hi << 32 | lo);
    }
    static LCMA_DEV __amdgpu_buffer_rsrc_t rsrc(const int8_t *base, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(base), 0, bytes, 0x00020000); }
    // Jobs from `halved` on are halves of tiles along the rows, upper and lower in turn.
    template <int TM, int TN> static LCMA_DEV Source source(Args args, int nx, int jobs, int halved, int job, I8Place &at) {
        Source s = {nullptr, nullptr, 0, 0};
        at = I8Place{0, 0, 0, 0};
        if (job < jobs) {
            const I8GemmParams p = arguments(args);
            int x, z;
            i8_tile_of_job(nx, p.nz, p.panel, job < halved ? job : halved + (job - halved) / 2, x, z);
            at = I8Rows<TM>(p).place(p, x);
            at.col0 = z * TN;
            if (job >= halved) {
                const int skip = (job - halved) % 2 * (TM / 2), left = at.rows > skip ? at.rows - skip : 0;
                at.row0 += left ? skip : 0;
                at.rows = left < TM / 2 ? left : TM / 2;
            }
            const int cols = p.N - at.col0 < TN ? p.N - at.col0 : TN;
            s.a = p.A + (int64_t)at.row0 * p.pitch;
            s.a_bytes = at.rows * p.pitch;
            s.b = p.W + ((int64_t)at.expert * p.N + at.col0) * p.pitch;
            s.b_bytes = cols * p.pitch;
        }
        // (uniform anyway; said here so that the descriptors stay in scalar registers)
        s.a = uniform(s.a);
        s.b = uniform(s.b);
        s.a_bytes = __builtin_amdgcn_readfirstlane(s.a_bytes);
        s.b_bytes = __builtin_amdgcn_readfirstlane(s.b_bytes);
        return s;
    }
    static constexpr uint32_t NONE = 1u << 30; // an offset past any extent
};

template <class OUT> struct I8PingPong : I8Turns {
    static constexpr int TM = 256, TN = 256, WM = 128, WN = 64, NMI = 4, NNI = 2;
    static constexpr int HALF = 128 * ROW, STRIP = 32 * 128;
    static constexpr int LDS_BYTES = 8 * HALF + 8 * STRIP;
    static_assert(LDS_BYTES <= 160 * 1024, "LDS budget of one CU");

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
    static LCMA_DEV void read_a(const LCMA_LDS char *half, const uint32_t (&at)[NK], i32x4 (&f)[2][NK]) {
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) f[i][k] = *(const LCMA_LDS i32x4 *)(half + i * 32 * ROW + at[k]);
    }
    static LCMA_DEV void read_b(const LCMA_LDS char *half, const uint32_t (&at)[NK], i32x4 (&f)[NK]) {
#pragma unroll
        for (int k = 0; k < NK; ++k) f[k] = *(const LCMA_LDS i32x4 *)(half + at[k]);
    }
    static LCMA_DEV void multiply(const i32x4 (&a)[2][NK], const i32x4 (&b)[NK], i32x16 &c0, i32x16 &c1) {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            c0 = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[k], a[0][k], c0, 0, 0, 0);
            c1 = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[k], a[1][k], c1, 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
    }

    static LCMA_DEV void run(LCMA_LDS char *lds) { // (the argument block has to be the kernel's first argument)
        pipeline((Args)__builtin_amdgcn_kernarg_segment_ptr(), lds, lds + HALF, lds + 2 * HALF, lds + 3 * HALF, lds + 4 * HALF, lds + 5 * HALF, lds + 6 * HALF, lds + 7 * HALF,
                 lds + 8 * HALF);
    }

    static LCMA_DEV void pipeline(Args args, LCMA_LDS char *__restrict__ A00, LCMA_LDS char *__restrict__ A10, LCMA_LDS char *__restrict__ A01,
                                  LCMA_LDS char *__restrict__ A11, LCMA_LDS char *__restrict__ B00, LCMA_LDS char *__restrict__ B10,
                                  LCMA_LDS char *__restrict__ B01, LCMA_LDS char *__restrict__ B11, LCMA_LDS char *__restrict__ strips) {
        const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w >> 2, wn = w & 3, l32 = tid & 31, lh = (tid >> 5) & 1, wave_chunk = w * 64;
        int nx, jobs;
        {
            const I8GemmParams p = arguments(args);
            const I8Rows<TM> groups(p);
            i8_zero_behind<OUT>(p, groups.behind, gridDim.x, NT);
            nx = groups.tiles;
            jobs = nx * p.nz;
        }
        const int units = gridDim.x;
        // tile-products in rounds of one per work-group; inside a round an XCD (work-groups go to the eight in turn) has consecutive ones
        const int per = units >> 3;
        const int unit = (int)blockIdx.x < (per << 3) ? (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
        const int whole = jobs / units * units;
        // a last round that at most half of the work-groups have a tile in: half a tile for twice as many (1024 x 4096 x 4096 41.2 -> 36.3 us)
        const int rest = jobs - whole, halved = 2 * rest <= units ? whole : jobs;
        jobs += jobs - halved;
        int job = unit < whole ? unit : (int)blockIdx.x;
        if (job >= jobs) return;
        const int pitch = args->pitch, ny = args->steps, n2 = (ny + 1) & ~1;
        uint32_t a_voff, b_voff;
        {
            const int row = tid >> 3, c = swz(row, tid & 7) * 16;
            a_voff = (uint32_t)row * pitch + c;
            b_voff = (uint32_t)((row >> 5) * 64 + (row & 31)) * pitch + c;
        }
        const uint32_t rows = 128 * pitch, a_half = 64 * pitch, b_half = 32 * pitch;
        uint32_t a_frag[NK], b_frag[NK];
        {
            const int ar = wm * 64 + l32, br = wn * 32 + l32;
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                a_frag[k] = ar * ROW + swz(ar, k * 2 + lh) * 16;
                b_frag[k] = br * ROW + swz(br, k * 2 + lh) * 16;
            }
        }
        I8Place at, at_next;
        Source cur = source<TM, TN>(args, nx, jobs, halved, job, at), nxt;
        i32x4 fa0[2][NK], fa1[2][NK], fb0[NK], fb1[NK];
        i32x16 acc[NMI][NNI];
        {
            const auto ra = rsrc(cur.a, cur.a_bytes), rb = rsrc(cur.b, cur.b_bytes);
            auto load_step = [&](LCMA_LDS char *A0, LCMA_LDS char *A1, LCMA_LDS char *B0, LCMA_LDS char *B1, uint32_t off) {
                load_half(rb, B0, wave_chunk, b_voff, off, rows);
                load_half(ra, A0, wave_chunk, a_voff, off, rows);
                load_half(ra, A1, wave_chunk, a_voff, off + a_half, rows);
                load_half(rb, B1, wave_chunk, b_voff, off + b_half, rows);
            };
            load_step(A00, A10, B00, B10, 0);
            load_step(A01, A11, B01, B11, ny > 1 ? ROW : NONE);
        }
        memory_slot_end();
        read_b(B00, b_frag, fb0);
        memory_slot_end();
        if (wm) slot_end(); // the second group runs one slot behind the first
        while (true) {
            int next = job + units;
            if (next >= whole && job < whole && whole < jobs) next = whole + (int)blockIdx.x;
            nxt = source<TM, TN>(args, nx, jobs, halved, next, at_next);
            const bool mine = at.rows > wm * WM; // (a group without rows multiplies nothing)
#pragma unroll
            for (int mi = 0; mi < NMI; ++mi)
#pragma unroll
                for (int ni = 0; ni < NNI; ++ni)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[mi][ni][v] = 0;
            auto walk = [&](auto multiplies) {
            for (int y = 0;;) {
                const bool in = y + 2 < n2;
                const auto ra = rsrc(in ? cur.a : nxt.a, in ? cur.a_bytes : nxt.a_bytes), rb = rsrc(in ? cur.b : nxt.b, in ? cur.b_bytes : nxt.b_bytes);
                const uint32_t off = in ? (uint32_t)(y + 2) * ROW : 0;
                // one step out of stage (A0, A1, B0, B1); nextB0: half 0 of B of the next step; off: of the loads into this stage
                auto step = [&](LCMA_LDS char *A0, LCMA_LDS char *A1, LCMA_LDS char *B0, LCMA_LDS char *B1, LCMA_LDS char *nextB0, uint32_t off) {
                    if constexpr (multiplies) read_a(A0, a_frag, fa0);
                    load_half(rb, B0, wave_chunk, b_voff, off, rows);
                    memory_slot_end();
                    if constexpr (multiplies) multiply(fa0, fb0, acc[0][0], acc[1][0]);
                    slot_end();
                    if constexpr (multiplies) read_a(A1, a_frag, fa1);
                    load_half(ra, A0, wave_chunk, a_voff, off, rows);
                    memory_slot_end();
                    if constexpr (multiplies) multiply(fa1, fb0, acc[2][0], acc[3][0]);
                    slot_end();
                    if constexpr (multiplies) read_b(B1, b_frag, fb1);
                    load_half(ra, A1, wave_chunk, a_voff, off + a_half, rows);
                    memory_slot_end();
                    if constexpr (multiplies) multiply(fa1, fb1, acc[2][1], acc[3][1]);
                    slot_end();
                    read_b(nextB0, b_frag, fb0);
                    load_half(rb, B1, wave_chunk, b_voff, off + b_half, rows);
                    memory_slot_end();
                    if constexpr (multiplies) multiply(fa0, fb1, acc[0][1], acc[1][1]);
                };
                step(A00, A10, B00, B10, B01, off);
                slot_end();
                step(A01, A11, B01, B11, B00, (in ? y + 3 == ny : ny == 1) ? NONE : off + ROW); // (an odd number of steps: one of zeros behind)
                y += 2;
                if (y >= n2) break;
                slot_end();
            }
            };
            if (mine) walk(std::true_type{});
            else walk(std::false_type{});
            if (!wm) slot_end(); // both groups write their halves of the tile in one slot
            if (next >= jobs) __builtin_amdgcn_s_waitcnt(0x0070); // loads past the end land before the LDS is another work-group's
            store_tile(args, strips + w * STRIP, at, wm, wn, acc);
            if (wm) slot_end();
            if (next >= jobs) break;
            job = next;
            cur = nxt;
            at = at_next;
        }
        if (!wm) slot_end();
    }

    static LCMA_DEV void store_tile(Args args, LCMA_LDS char *strip, const I8Place &at, int wm, int wn, const i32x16 (&acc)[NMI][NNI]) {
        const I8GemmParams p = arguments(args);
        i8_store_part<OUT, NMI, 32>(p, strip, at, wm * WM, wn * WN, acc);
    }
};

} // namespace lcma
