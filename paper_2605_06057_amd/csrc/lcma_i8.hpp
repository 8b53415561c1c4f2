// C = (A W^T) in 8-bit integers for gfx950: codes A (rows x K) and W (N x K, or experts x N x K), a scale for each row of A and of W:
//   C[m][n] = SA[m] SW[n] sum_k A[m][k] W[n][k] (+ bias[n])
// The sum is exact in 32-bit integers (K <= 131071), is turned into fp32 once, scaled there and rounded once to the type of C (16-bit rows that are combined into tokens
// afterwards are rounded a second time there: half the bytes of fp32 rows, which a caller can have by asking for them).  With
// offsets the rows of A are in groups, group e times the weights of expert e; rows behind the last group give zeros.
//
// Rows of codes are whole 128 bytes (zeros behind K).  All addresses of a tile are 32-bit offsets from 64-bit bases, so a matrix may be of any
// size; rows past a group and columns past N lie past the extent of the tile's descriptor and read as zero.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lcma_device.hpp"
#include "lcma_few_rows.hpp" // wait_loads
#include "lcma_experts_params.h"
#include "lcma_lanes.hpp"

namespace lcma {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// A tile of C: rows row0 .. row0 + rows - 1 of A, all of expert `expert`, columns col0 .. of C.
struct I8Place {
    int row0, rows, col0, expert;
};

// First row of group e (experts: of the rows behind the groups), inside A whatever the offsets say; tiles of TM rows that a group takes.
template <class P> LCMA_DEV int i8_row(const P &p, int e) {
    const int row = p.offsets[e];
    return row < 0 ? 0 : row > p.rows ? p.rows : row;
}
template <int TM> LCMA_DEV int i8_tiles(int begin, int end) { return end > begin ? (int)(((uint32_t)(end - begin) + (TM - 1)) / TM) : 0; } // (up to 2^31 - 1 rows)

// The tiles of TM rows of all groups, in expert order, every group in tiles of its own: how many there are, and the rows of tile x.  Every wave
// by itself, a lane per expert; the first 64 experts are kept, which are mostly all.
// P: an argument block with rows, offsets and experts.
template <int TM, class P = I8GemmParams> struct I8Rows {
    int begin, end, upto; // rows of this lane's expert, tiles up to and with it
    int tiles, behind;    // all tiles, and the first row behind the groups

    LCMA_DEV void experts_from(const P &p, int e0, int before) {
        const int e = e0 + (int)(threadIdx.x & 63);
        begin = end = 0;
        if (e < p.experts) {
            begin = i8_row(p, e);
            end = i8_row(p, e + 1);
        }
        upto = before + lanes_upto(i8_tiles<TM>(begin, end));
    }
    LCMA_DEV I8Rows(const P &p) {
        if (!p.offsets) {
            tiles = i8_tiles<TM>(0, p.rows);
            behind = p.rows;
            return;
        }
        experts_from(p, 0, 0);
        tiles = __builtin_amdgcn_readlane(upto, 63);
        behind = __builtin_amdgcn_readlane(end, (p.experts - 1) & 63);
        for (int e0 = 64; e0 < p.experts; e0 += 64) {
            I8Rows more = *this;
            more.experts_from(p, e0, tiles);
            tiles = __builtin_amdgcn_readlane(more.upto, 63);
            behind = __builtin_amdgcn_readlane(more.end, (p.experts - 1) & 63);
        }
    }
    // All tiles, and no more than ascending offsets can make: the launch's count, which fits 32 bits with the tiles along the columns.
    LCMA_DEV int within(const P &p) const {
        const int most = p.rows / TM + (p.rows < p.experts ? p.rows : p.experts);
        return tiles < most ? tiles : most;
    }
    LCMA_DEV I8Place place(const P &p, int x) const {
        if (!p.offsets) return {x * TM, p.rows - x * TM < TM ? p.rows - x * TM : TM, 0, 0};
        I8Rows at = *this;
        int e0 = 0;
        uint64_t past;
        while (!(past = __ballot(x < at.upto)) && e0 + 64 < p.experts) {
            e0 += 64;
            at.experts_from(p, e0, __builtin_amdgcn_readlane(at.upto, 63));
        }
        const int l = past ? __builtin_ctzll(past) : 63;
        const int begin = __builtin_amdgcn_readlane(at.begin, l), end = __builtin_amdgcn_readlane(at.end, l);
        const int row0 = begin + (x - (__builtin_amdgcn_readlane(at.upto, l) - i8_tiles<TM>(begin, end))) * TM;
        return {row0, end - row0 < TM ? end - row0 : TM, 0, e0 + l};
    }
};

// Tile j of nx x nz: they run down the rows inside column panels of `panel` tiles.
LCMA_DEV void i8_tile_of_job(int nx, int nz, int panel, int j, int &x, int &z) {
    const int whole = nz / panel * panel, full = whole * nx;
    const int width = j < full ? panel : nz - whole, id = j < full ? j % (panel * nx) : j - full;
    x = id / width;
    z = (j < full ? j / (panel * nx) * panel : whole) + id % width;
}

// Scales (or biases) of columns n .. n + 3, zeros from N on.
LCMA_DEV f32x4 i8_four(const float *at, int n, int N) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (n + 4 <= N) __builtin_memcpy(&v, at + n, 16);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < N) v[i] = at[n + i];
    return v;
}

// 16 bytes of a row of C, `cols` columns of which are inside it.
template <class OUT> LCMA_DEV void i8_store16(char *at, u32x4 v, int cols) {
    if (cols >= 16 / OUT::ES) __builtin_memcpy(at, &v, 16);
    else
#pragma unroll
        for (int i = 0; i < 16 / OUT::ES; ++i)
            if (i < cols) {
                if constexpr (OUT::ES == 4) ((uint32_t *)at)[i] = v[i];
                else ((uint16_t *)at)[i] = (uint16_t)(v[i / 2] >> (i & 1) * 16);
            }
}

// Rows of C behind the groups are zero: the work-groups of the launch share them.
template <class OUT, class P> LCMA_DEV void i8_zero_behind(const P &p, int behind, int groups, int threads) {
    constexpr int V = 16 / OUT::ES;
    for (uint32_t row = behind + blockIdx.x; row < (uint32_t)p.rows; row += groups) // (past 2^31 before it ends)
        for (int n = threadIdx.x * V; n < p.N; n += threads * V) i8_store16<OUT>((char *)p.C + ((int64_t)row * p.ldc + n) * OUT::ES, u32x4{0, 0, 0, 0}, p.N - n);
}

// Four neighbouring columns of a row of C, the last ones of which may be past N.
template <class OUT> LCMA_DEV void i8_store4(char *at, f32x4 v, int cols) {
    if constexpr (OUT::ES == 4) {
        if (cols >= 4) {
            __builtin_memcpy(at, &v, 16);
        } else {
            #pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < cols) ((float *)at)[i] = v[i];
        }
    } else {
        if (cols >= 4) {
            const uint32_t raw[2] = {Round<OUT>::run(v[0]) | (Round<OUT>::run(v[1]) << 16), Round<OUT>::run(v[2]) | (Round<OUT>::run(v[3]) << 16)};
            __builtin_memcpy(at, raw, 8);
        } else {
            #pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < cols) ((uint16_t *)at)[i] = (uint16_t)Round<OUT>::run(v[i]);
        }
    }
}

// A wave's part of a tile (NMI x 2 blocks of 32 x 32 from (row, col) of the tile on) scaled, rounded and stored: through a strip of LDS that is the wave's own, SR
// rows of 128 bytes, so that it leaves as whole lines, 16 bytes a lane.  FULL: all of it lies inside C.
template <class OUT, int NMI, int SR, bool FULL>
LCMA_DEV void i8_store_rows(const I8GemmParams &p, LCMA_LDS char *strip, const I8Place &at, int row, int col, const i32x16 (&acc)[NMI][2]) {
    constexpr int ES = OUT::ES, BLOCKS = ES == 2 ? 2 : 1; // 32-column blocks in a strip's 128 bytes
    // (the lane number anew, hidden: what derives from it would otherwise be kept in registers through the steps)
    int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(lane));
    const int l32 = lane & 31, lh = lane >> 5, cols = p.N - at.col0 - col, left = at.rows - row;
    if (!FULL && (cols <= 0 || left <= 0)) return;
    const int64_t channel = (int64_t)at.expert * p.N + at.col0 + col;
    auto vector = [&](const float *of) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(of + channel), 0, cols * 4, 0x00020000); };
    const auto rsw = vector(p.SW), rbias = vector(p.bias ? p.bias : p.SW);
    auto four = [&](__amdgpu_buffer_rsrc_t of, int n) { // (past the last column: zeros)
        if constexpr (FULL) {
            return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(of, lh * 16, n * 4, 0));
        } else {
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(of, lh * 16 + i * 4, n * 4, 0));
            return v;
        }
    };
    f32x4 sw[2][4];
    float sa[NMI];
#pragma unroll
    for (int mi = 0; mi < NMI; ++mi) {
        const int m = mi * 32 + l32;
        sa[mi] = p.SA[at.row0 + row + (FULL || m < left ? m : left - 1)];
    }
#pragma unroll
    for (int ni = 0; ni < 2; ++ni)
#pragma unroll
        for (int g = 0; g < 4; ++g) sw[ni][g] = four(rsw, ni * 32 + g * 8);
    const int row8 = lane >> 3, ch = lane & 7; // a store: eight rows, eight lanes along each
    char *c = (char *)p.C + ((int64_t)(at.row0 + row + row8) * p.ldc + at.col0 + col) * ES + ch * 16;
    const int64_t down = 8 * p.ldc * ES;
#pragma unroll
    for (int mi = 0; mi < NMI; ++mi) {
#pragma unroll
        for (int n0 = 0; n0 < 2; n0 += BLOCKS) {
            u32x4 out[2][4]; // (16 bit: the first two words)
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int ni = n0 + b;
                    f32x4 v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = (float)acc[mi][ni][g * 4 + i] * sa[mi] * sw[ni][g][i];
                    if (p.bias) v += four(rbias, ni * 32 + g * 8);
                    if constexpr (ES == 2) {
                        out[b][g][0] = Round<OUT>::run(v[0]) | (Round<OUT>::run(v[1]) << 16);
                        out[b][g][1] = Round<OUT>::run(v[2]) | (Round<OUT>::run(v[3]) << 16);
                    } else {
                        out[b][g] = __builtin_bit_cast(u32x4, v);
                    }
                }
#pragma unroll
            for (int h = 0; h < 32 / SR; ++h) {
                if (SR == 32 || l32 / SR == h) {
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const int byte = (b * 32 + g * 8 + lh * 4) * ES;
                            LCMA_LDS char *to = strip + l32 % SR * 128 + ((byte >> 4) ^ (l32 & 7)) * 16 + (byte & 15);
                            if constexpr (ES == 2) *(LCMA_LDS uint64_t *)to = (uint64_t)out[b][g][1] << 32 | out[b][g][0];
                            else *(LCMA_LDS u32x4 *)to = out[b][g];
                        }
                }
                lanes_meet();
#pragma unroll
                for (int it = 0; it < SR / 8; ++it) {
                    const u32x4 v = *(const LCMA_LDS u32x4 *)(strip + (it * 8 + row8) * 128 + (ch ^ row8) * 16);
                    char *to = c + (h * (SR / 8) + it) * down + n0 * 32 * ES;
                    const int n = n0 * 32 + ch * (16 / ES);
                    if constexpr (FULL) __builtin_memcpy(to, &v, 16);
                    else if (mi * 32 + h * SR + it * 8 + row8 < left && n < cols) i8_store16<OUT>(to, v, cols - n);
                }
                lanes_meet();
            }
        }
        c += 4 * down;
    }
}
template <class OUT, int NMI, int SR>
LCMA_DEV void i8_store_part(const I8GemmParams &p, LCMA_LDS char *strip, const I8Place &at, int row, int col, const i32x16 (&acc)[NMI][2]) {
    if (at.rows >= row + NMI * 32 && at.col0 + col + 64 <= p.N) i8_store_rows<OUT, NMI, SR, true>(p, strip, at, row, col, acc);
    else i8_store_rows<OUT, NMI, SR, false>(p, strip, at, row, col, acc);
}

// One tile of TM x TN per work-group of WGM x WGN waves.  A step is 128 bytes of K; S stages of LDS hold the steps in flight, the loads (straight into LDS)
// run S - 1 steps ahead and are waited for by count, and one barrier a step says that all waves' parts of it have landed and that all
// have read the stage that is loaded anew.  What the depth is for: with two stages a step takes as long as a load does, about 0.8 us,
// whatever the tile.  What bounds it is the LDS, which writes what is loaded (80 bytes a clock) and reads it again for every wave (128 bytes a clock): 1178 clocks a
// step of 128 x 128 in eight waves against 512 of matrix instructions, 691 against 256 for 64 x 128 and 461 against 128 for 64 x 64 in four, which run two to a CU.
// Measured (us, bf16 results): 333 x 4096 x 4096 on 64 x 64 15.2 (two stages 23), 128 x 14336 x 4096 on 64 x 128 19.6, 1024 x 4096 x 4096 on 128 x 128 24 (1430
// TOP/s; the same in two groups of waves that take the steps of K in turn 28), 3000 rows of 64 experts x 2816 x 2048 on 64 x 128 79 (4.9 TB/s).  Stores of
// eight bytes a lane instead of whole lines: 15.6 for the first, 26.8 for the third.
// The weights are the left operand of the matrix instruction, so a lane holds four neighbouring columns of one row of C.
template <int TM, int TN, int WGM, int WGN, int S, class OUT> struct I8Ring {
    static constexpr int NT = 64 * WGM * WGN, NMI = TM / WGM / 32, NNI = TN / WGN / 32;
    static constexpr int A_STAGE = TM * 128, STAGE = (TM + TN) * 128, LDS_BYTES = S * STAGE;
    static constexpr int QA = TM * 8 / NT, QB = TN * 8 / NT;
    static_assert(NNI != 2 || NT * 64 <= LDS_BYTES, "strips");
    static_assert(TM * 8 % NT == 0 && TN * 8 % NT == 0 && LDS_BYTES <= 160 * 1024 && (S == 3 || S == 4) && (S - 1) * (QA + QB) <= 63, "tile and wave grid");

    // 16-byte chunk c of a row sits at position c ^ (row / 2 % 8)
    static LCMA_DEV constexpr int swz(int row, int c) { return c ^ ((row >> 1) & 7); }

    static LCMA_DEV void run(const I8GemmParams &p, LCMA_LDS char *lds) {
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w / WGN, wn = w % WGN;
        const I8Rows<TM> groups(p);
        i8_zero_behind<OUT>(p, groups.behind, gridDim.x, NT);
        const int nx = groups.tiles, jobs = nx * p.nz, per = (jobs + 7) / 8;
        const int job = (blockIdx.x & 7) * per + (blockIdx.x >> 3); // an eighth of the tiles to every XCD
        if ((int)(blockIdx.x >> 3) >= per || job >= jobs) return;
        int x, z;
        i8_tile_of_job(nx, p.nz, p.panel, job, x, z);
        I8Place at = groups.place(p, x);
        at.col0 = z * TN;
        i32x16 acc[NMI][NNI];
#pragma unroll
        for (int i = 0; i < NMI; ++i)
#pragma unroll
            for (int j = 0; j < NNI; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
        multiply(p, at, w, wm, wn, acc, lds, lds + STAGE, lds + 2 * STAGE, lds + (S == 4 ? 3 * STAGE : 0));
        if constexpr (NNI == 2) {
            __syncthreads(); // no load is in flight and every wave has read its last step: the strips take the place of the stages
            i8_store_part<OUT, NMI, 32>(p, lds + w * 4096, at, wm * NMI * 32, wn * 64, acc);
            return;
        }
// (wave parts of 32 columns: the tile meets in LDS, rows of TN columns)
        constexpr int ES = OUT::ES, PITCH = TN * ES, CHUNKS = PITCH / 16;
        static_assert(NNI == 2 || TM * PITCH <= LDS_BYTES, "the tile of C fits the stages");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NMI; ++i) {
            const int row = (wm * NMI + i) * 32 + (lane & 31);
            const float sa = row < at.rows ? p.SA[at.row0 + row] : 0.f;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int n = wn * 32 + g * 8 + (lane >> 5) * 4, byte = n * ES;
                const f32x4 sw = i8_four(p.SW + (int64_t)at.expert * p.N, at.col0 + n, p.N);
                f32x4 v;
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = (float)acc[i][0][g * 4 + k] * sa * sw[k];
                if (p.bias) v += i8_four(p.bias + (int64_t)at.expert * p.N, at.col0 + n, p.N);
                LCMA_LDS char *to = lds + row * PITCH + ((byte >> 4) ^ (row & 7)) * 16 + (byte & 15);
                if constexpr (ES == 2) {
                    const uint32_t lo = Round<OUT>::run(v[0]) | (Round<OUT>::run(v[1]) << 16), hi = Round<OUT>::run(v[2]) | (Round<OUT>::run(v[3]) << 16);
                    *(LCMA_LDS uint64_t *)to = (uint64_t)hi << 32 | lo;
                } else {
                    *(LCMA_LDS f32x4 *)to = v;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TM * CHUNKS / NT; ++t) {
            const int row = (t * NT + (int)threadIdx.x) / CHUNKS, ch = threadIdx.x % CHUNKS, col = at.col0 + ch * (16 / ES);
            const u32x4 v = *(const LCMA_LDS u32x4 *)(lds + row * PITCH + (ch ^ (row & 7)) * 16);
            if (row < at.rows && col < p.N) i8_store16<OUT>((char *)p.C + ((int64_t)(at.row0 + row) * p.ldc + col) * ES, v, p.N - col);
        }
    }
    // restrict: the loads in flight towards one stage do not touch what is read from another (the compiler would otherwise wait for all of them in
    // front of every read)
    static LCMA_DEV void multiply(const I8GemmParams &p, const I8Place &at, int w, int wm, int wn, i32x16 (&acc)[NMI][NNI], LCMA_LDS char *__restrict__ s0,
                                  LCMA_LDS char *__restrict__ s1, LCMA_LDS char *__restrict__ s2, LCMA_LDS char *__restrict__ s3) {
        const int tid = threadIdx.x, lane = tid & 63, cols = p.N - at.col0 < TN ? p.N - at.col0 : TN, steps = p.steps;
        const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(p.A) + (int64_t)at.row0 * p.pitch, 0, at.rows * p.pitch, 0x00020000);
        const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(p.W) + ((int64_t)at.expert * p.N + at.col0) * p.pitch, 0, cols * p.pitch, 0x00020000);
        const uint32_t voff = (uint32_t)(tid >> 3) * p.pitch + swz(tid >> 3, tid & 7) * 16;
        auto load = [&](LCMA_LDS char *st, int y) { // a step past the end: zeros, from past the extents
            const int k = y < steps ? y * 128 : 1 << 30;
#pragma unroll
            for (int q = 0; q < QB; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (LCMA_LDS void *)(st + A_STAGE + (q * NT + w * 64) * 16), 16, (int)voff, k + q * (NT / 8) * p.pitch, 0, 0);
#pragma unroll
            for (int q = 0; q < QA; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (LCMA_LDS void *)(st + (q * NT + w * 64) * 16), 16, (int)voff, k + q * (NT / 8) * p.pitch, 0, 0);
        };
        uint32_t fa[4], fb[4]; // of this lane's 16 bytes in the first 32 rows of the wave
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int c = k * 2 + (lane >> 5), ra0 = wm * NMI * 32 + (lane & 31), rb0 = wn * NNI * 32 + (lane & 31);
            fa[k] = ra0 * 128 + swz(ra0, c) * 16;
            fb[k] = A_STAGE + rb0 * 128 + swz(rb0, c) * 16;
        }
        auto step = [&](LCMA_LDS char *st, LCMA_LDS char *before, int y) {
            wait_loads<(S - 2) * (QA + QB)>();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            load(before, y + S - 1);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                i32x4 a[NMI], b[NNI];
#pragma unroll
                for (int i = 0; i < NMI; ++i) a[i] = *(const LCMA_LDS i32x4 *)(st + fa[k] + i * 32 * 128);
#pragma unroll
                for (int j = 0; j < NNI; ++j) b[j] = *(const LCMA_LDS i32x4 *)(st + fb[k] + j * 32 * 128);
#pragma unroll
                for (int i = 0; i < NMI; ++i)
#pragma unroll
                    for (int j = 0; j < NNI; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[j], a[i], acc[i][j], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0); // (the multiplications stay in front of the next wait; what they read has left LDS)
        };
        load(s0, 0);
        load(s1, 1);
        if constexpr (S == 4) load(s2, 2);
        for (int y = 0; y < steps;) {
            step(s0, S == 4 ? s3 : s2, y);
            if (++y >= steps) break;
            step(s1, s0, y);
            if (++y >= steps) break;
            step(s2, s1, y);
            ++y;
            if constexpr (S == 4) {
                if (y >= steps) break;
                step(s3, s2, y);
                ++y;
            }
        }
        wait_loads<0>(); // the loads past the end land before the LDS is another work-group's
    }
};

} // namespace lcma
