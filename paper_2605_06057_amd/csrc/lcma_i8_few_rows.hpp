// The 8-bit-integer product on few rows: bound by reading the weights once.  As csrc/lcma_few_rows.hpp does in 16 bit, a work-group owns a tile of T x T
// of C and its waves split K between them, a line (128 k, 128 bytes of every row) to a wave in turn.  Nothing is shared between waves, so there is no barrier
// in the loop: each wave has stages of its own in LDS, sends the loads of its next lines straight into them (whole lines, eight lanes to a row, which a
// CU takes in four times as fast as the fragments' own order), waits for a line by count and reads its fragments.  At the end the waves' sums are added
// in LDS, as integers, so in any order, scaled and rounded once.  Four waves with two lines in flight each, 32 KB (tiles of 16) and 64 KB (32), so that several
// work-groups share a CU: four lines in flight or eight waves are level on 16 x 4096 x 14336, 9 and 39 % slower on 1 x 14336 x 4096, 23 and 93 % on
// 16 rows of 8 experts x 28672 x 4096.
// Measured (us): 1 x 14336 x 4096 13.3 (4.4 TB/s with the launch; the kernel alone 11.7, 5.0), 16 x 4096 x 14336 13.8, 64 x 4096 x 4096 on 32 x 32 7.1, 16 rows of
// 8 experts x 28672 x 4096 133 to 142 (5.8 TB/s; a large read 6.1).
#pragma once
#include "lcma_i8.hpp"

namespace lcma {

template <int T, int WK, class OUT> struct I8FewRows {
    static constexpr int F = T == 16 ? 16 : 32, NF = T / F, KF = 128 / (1024 / F); // 16x16x64 or 32x32x32 instructions; fragments of a line along K
    static constexpr int LOADS = T / 8, HALF = T * 128, STAGE = 2 * HALF;
    static constexpr int PITCH = T + 4, SUMS = WK * T * PITCH * 4, STAGES = WK * 2 * STAGE, LDS_BYTES = SUMS > STAGES ? SUMS : STAGES;
    static_assert(LDS_BYTES <= 160 * 1024 && 2 * LOADS * 2 <= 63, "LDS budget of one CU; counter of loads");
    using Acc = std::conditional_t<F == 16, i32x4, i32x16>;

    static LCMA_DEV void run(const I8GemmParams &p, LCMA_LDS char *lds) {
        const int lane = threadIdx.x & 63, fr = lane & (F - 1), fk = lane / F, wk = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const I8Rows<T> groups(p);
        i8_zero_behind<OUT>(p, groups.behind, gridDim.x, 64 * WK);
        const int nx = groups.tiles, jobs = nx * p.nz, per = (jobs + 7) / 8;
        const int job = (blockIdx.x & 7) * per + (blockIdx.x >> 3); // an eighth of the tiles to every XCD, row tiles that share weights next to each other
        if ((int)(blockIdx.x >> 3) >= per || job >= jobs) return;
        int x, z;
        i8_tile_of_job(nx, p.nz, p.panel, job, x, z);
        I8Place at = groups.place(p, x);
        at.col0 = z * T;
        Acc acc[NF][NF];
#pragma unroll
        for (int i = 0; i < NF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j)
#pragma unroll
                for (int v = 0; v < F * F / 64; ++v) acc[i][j][v] = 0;
        LCMA_LDS char *st = lds + wk * (2 * STAGE);
        lines_of_wave(p, at, wk, acc, st, st + STAGE);
        __syncthreads(); // no load is in flight and every wave has read its last line: the sums take the place of the stages
        LCMA_LDS int *mine = (LCMA_LDS int *)lds + wk * (T * PITCH);
#pragma unroll
        for (int i = 0; i < NF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j)
#pragma unroll
                for (int g = 0; g < F * F / 256; ++g) { // four neighbouring columns of row fr
                    const i32x4 v = {acc[i][j][g * 4], acc[i][j][g * 4 + 1], acc[i][j][g * 4 + 2], acc[i][j][g * 4 + 3]};
                    *(LCMA_LDS i32x4 *)(mine + (i * F + fr) * PITCH + j * F + g * 8 + fk * 4) = v;
                }
        __syncthreads();
        for (int t = threadIdx.x; t < T * T / 4; t += 64 * WK) {
            const int row = t / (T / 4), n = t % (T / 4) * 4, col = at.col0 + n;
            if (row >= at.rows || col >= p.N) continue;
            const LCMA_LDS int *of = (const LCMA_LDS int *)lds + row * PITCH + n;
            i32x4 sum = *(const LCMA_LDS i32x4 *)of;
#pragma unroll
            for (int k = 1; k < WK; ++k) sum += *(const LCMA_LDS i32x4 *)(of + k * T * PITCH);
            const float sa = p.SA[at.row0 + row];
            const f32x4 sw = i8_four(p.SW + (int64_t)at.expert * p.N, col, p.N);
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = (float)sum[i] * sa * sw[i];
            if (p.bias) v += i8_four(p.bias + (int64_t)at.expert * p.N, col, p.N);
            i8_store4<OUT>((char *)p.C + ((int64_t)(at.row0 + row) * p.ldc + col) * OUT::ES, v, p.N - col);
        }
    }
    // Lines `line`, line + WK, ... of a tile.  s0, s1: the stages of the wave.  restrict: the loads in flight towards one do not touch what is read
    // from another (the compiler would otherwise wait for all of them in front of every read).
    static LCMA_DEV void lines_of_wave(const I8GemmParams &p, const I8Place &tile, int line, Acc (&acc)[NF][NF], LCMA_LDS char *__restrict__ s0,
                                       LCMA_LDS char *__restrict__ s1) {
        const int lane = threadIdx.x & 63, fr = lane & (F - 1), fk = lane / F, end = p.steps;
        const int cols = p.N - tile.col0 < T ? p.N - tile.col0 : T;
        const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(p.A) + (int64_t)tile.row0 * p.pitch, 0, tile.rows * p.pitch, 0x00020000);
        const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(p.W) + ((int64_t)tile.expert * p.N + tile.col0) * p.pitch, 0, cols * p.pitch, 0x00020000);
        uint32_t off[2]; // of the even and odd loads of a line
#pragma unroll
        for (int i = 0; i < 2; ++i) off[i] = (uint32_t)(lane >> 3) * p.pitch + ((lane & 7) ^ (lane >> 4) ^ (4 * i)) * 16;
        auto load = [&](LCMA_LDS char *st, int line) { // a line past the end: zeros, from past the extents
            const int k = line < end ? line * 128 : 1 << 30;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (LCMA_LDS void *)(st + HALF + i * 1024), 16, (int)off[i & 1], k + i * 8 * p.pitch, 0, 0);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (LCMA_LDS void *)(st + i * 1024), 16, (int)off[i & 1], k + i * 8 * p.pitch, 0, 0);
        };
        uint32_t frag[KF]; // of this lane's 16 bytes in either operand's rows
#pragma unroll
        for (int k = 0; k < KF; ++k) frag[k] = fr * 128 + ((k * (64 / F) + fk) ^ (fr >> 1 & 7)) * 16;
        auto step = [&](LCMA_LDS char *st, int line) {
            i32x4 a[KF][NF], b[KF][NF];
            wait_loads<2 * LOADS>();
#pragma unroll
            for (int k = 0; k < KF; ++k)
#pragma unroll
                for (int i = 0; i < NF; ++i) {
                    a[k][i] = *(const LCMA_LDS i32x4 *)(st + frag[k] + i * F * 128);
                    b[k][i] = *(const LCMA_LDS i32x4 *)(st + HALF + frag[k] + i * F * 128);
                }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0xC07F); // lgkmcnt(0): what was read has left LDS, so its place may be loaded anew
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            load(st, line + 2 * WK);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < KF; ++k)
#pragma unroll
                for (int i = 0; i < NF; ++i)
#pragma unroll
                    for (int j = 0; j < NF; ++j) {
                        if constexpr (F == 16) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[k][j], a[k][i], acc[i][j], 0, 0, 0);
                        else acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[k][j], a[k][i], acc[i][j], 0, 0, 0);
                    }
        };
        load(s0, line);
        load(s1, line + WK);
        while (line < end) {
            step(s0, line);
            if ((line += WK) >= end) break;
            step(s1, line);
            line += WK;
        }
        wait_loads<0>();
    }
};

} // namespace lcma
