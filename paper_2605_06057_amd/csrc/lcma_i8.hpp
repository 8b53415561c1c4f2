// C = (A W^T) in 8-bit integers for gfx950: codes A (rows x K) and W (N x K, or experts x N x K), a scale for each row of A and of W:
//   C[m][n] = SA[m] SW[n] sum_k A[m][k] W[n][k] (+ bias[n])
// The sum is exact in 32-bit integers (K <= 131071), is turned into fp32 once, scaled there and rounded once to the type of C.  With
// offsets the rows of A are in groups, group e times the weights of expert e; rows behind the last group give zeros.
//
// Rows of codes are whole 128 bytes (zeros behind K).  All addresses of a tile are 32-bit offsets from 64-bit bases, so a matrix may be of any
// size; rows past a group and columns past N lie past the extent of the tile's descriptor and read as zero.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lcma_device.hpp"
#include "lcma_experts_params.h"

namespace lcma {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// A tile of C: rows row0 .. row0 + rows - 1 of A, all of expert `expert` (experts: the rows behind the groups), columns col0 .. of C.
struct I8Place {
    int row0, rows, col0, expert;
};

// First row of group e (experts: of the rows behind the groups), inside A whatever the offsets say; tiles of TM rows that a group takes.
LCMA_DEV int i8_row(const I8GemmParams &p, int e) {
    const int row = e <= p.experts ? p.offsets[e] : p.rows;
    return row < 0 ? 0 : row > p.rows ? p.rows : row;
}
template <int TM> LCMA_DEV int i8_tiles(int begin, int end) { return end > begin ? (end - begin + TM - 1) / TM : 0; }

// Tile `x` of TM rows among those of all groups (in expert order, every group in tiles of its own, the rows behind the groups last): its
// place along the rows; false past the last one.  total: how many there are.  Every wave by itself, a lane per expert.
template <int TM> LCMA_DEV int i8_row_tiles(const I8GemmParams &p) {
    if (!p.offsets) return (p.rows + TM - 1) / TM;
    const int lane = threadIdx.x & 63;
    int total = 0;
    for (int e0 = 0; e0 <= p.experts; e0 += 64) {
        const int e = e0 + lane;
        int tiles = 0;
        if (e <= p.experts) tiles = i8_tiles<TM>(i8_row(p, e), i8_row(p, e + 1));
#pragma unroll
        for (int d = 32; d; d >>= 1) tiles += __shfl_xor(tiles, d);
        total += tiles;
    }
    return __builtin_amdgcn_readfirstlane(total);
}
template <int TM> LCMA_DEV I8Place i8_row_place(const I8GemmParams &p, int x) {
    I8Place at = {x * TM, p.rows - x * TM, 0, 0};
    if (p.offsets) {
        const int lane = threadIdx.x & 63;
        int before = 0;
        for (int e0 = 0; e0 <= p.experts; e0 += 64) {
            const int e = e0 + lane;
            int begin = 0, end = 0;
            if (e <= p.experts) {
                begin = i8_row(p, e);
                end = i8_row(p, e + 1);
            }
            const int tiles = i8_tiles<TM>(begin, end);
            int upto = tiles;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int below = __shfl_up(upto, d);
                if (lane >= d) upto += below;
            }
            upto += before;
            const uint64_t past = __ballot(x < upto);
            if (past) {
                const int l = __builtin_ctzll(past);
                const int skip = (x - (__shfl(upto, l) - __shfl(tiles, l))) * TM;
                at.expert = e0 + l;
                at.row0 = __shfl(begin, l) + skip;
                at.rows = __shfl(end, l) - at.row0;
                break;
            }
            before = __shfl(upto, 63);
        }
    }
    at.row0 = __builtin_amdgcn_readfirstlane(at.row0);
    at.rows = __builtin_amdgcn_readfirstlane(at.rows < TM ? at.rows : TM);
    at.expert = __builtin_amdgcn_readfirstlane(at.expert);
    return at;
}

// Four neighbouring columns of a row of C, the last ones of which may be past N.
template <class OUT> LCMA_DEV void i8_store4(char *at, const float (&v)[4], int cols) {
    if constexpr (OUT::ES == 4) {
        if (cols >= 4) {
            const u32x4 raw = {Round<OUT>::run(v[0]), Round<OUT>::run(v[1]), Round<OUT>::run(v[2]), Round<OUT>::run(v[3])};
            __builtin_memcpy(at, &raw, 16);
        } else {
            for (int i = 0; i < cols; ++i) ((float *)at)[i] = v[i];
        }
    } else {
        if (cols >= 4) {
            const uint32_t raw[2] = {Round<OUT>::run(v[0]) | (Round<OUT>::run(v[1]) << 16), Round<OUT>::run(v[2]) | (Round<OUT>::run(v[3]) << 16)};
            __builtin_memcpy(at, raw, 8);
        } else {
            for (int i = 0; i < cols; ++i) ((uint16_t *)at)[i] = (uint16_t)Round<OUT>::run(v[i]);
        }
    }
}

// One tile of TM x TN per work-group of WGM x WGN waves, two LDS stages of 128 bytes of K.  The weights are the left operand of the matrix
// instruction, so a lane holds four neighbouring columns of one row of C.
template <int TM, int TN, int WGM, int WGN, class OUT> struct I8Tile {
    static constexpr int NT = 64 * WGM * WGN, NMI = TM / WGM / 32, NNI = TN / WGN / 32;
    static constexpr int A_STAGE = TM * 128, STAGE = (TM + TN) * 128, LDS_BYTES = 2 * STAGE;
    static constexpr int QA = TM * 8 / NT, QB = TN * 8 / NT;
    static_assert(TM * 8 % NT == 0 && TN * 8 % NT == 0 && LDS_BYTES <= 160 * 1024, "tile and wave grid");

    // 16-byte chunk c of a row sits at position c ^ (row / 2 % 8)
    static LCMA_DEV constexpr int swz(int row, int c) { return c ^ ((row >> 1) & 7); }

    static LCMA_DEV void run(const I8GemmParams &p, LCMA_LDS char *lds) {
        const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w / WGN, wn = w % WGN;
        const int nx = i8_row_tiles<TM>(p), jobs = nx * p.nz, per = (jobs + 7) / 8;
        const int job = (blockIdx.x & 7) * per + (blockIdx.x >> 3); // an eighth of the tiles to every XCD
        if ((int)(blockIdx.x >> 3) >= per || job >= jobs) return;
        const int whole = p.nz / p.panel * p.panel, full = whole * nx, width = job < full ? p.panel : p.nz - whole, id = job < full ? job : job - full;
        const int x = job < full ? id % (p.panel * nx) / p.panel : id / width, z = job < full ? id / (p.panel * nx) * p.panel + id % p.panel : whole + id % width;
        const I8Place at = i8_row_place<TM>(p, x);
        const int col0 = z * TN, cols = p.N - col0 < TN ? p.N - col0 : TN, steps = at.expert < p.experts ? p.steps : 0;
        const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(p.A) + (int64_t)at.row0 * p.pitch, 0, at.rows * p.pitch, 0x00020000);
        const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(p.W) + ((int64_t)at.expert * p.N + col0) * p.pitch, 0, cols * p.pitch, 0x00020000);
        const uint32_t voff = (uint32_t)(tid >> 3) * p.pitch + swz(tid >> 3, tid & 7) * 16;
        i32x16 acc[NMI][NNI];
#pragma unroll
        for (int i = 0; i < NMI; ++i)
#pragma unroll
            for (int j = 0; j < NNI; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;
        auto load = [&](LCMA_LDS char *st, int y) {
#pragma unroll
            for (int q = 0; q < QA; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (LCMA_LDS void *)(st + (q * NT + w * 64) * 16), 16, (int)voff, y * 128 + q * (NT / 8) * p.pitch, 0, 0);
#pragma unroll
            for (int q = 0; q < QB; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (LCMA_LDS void *)(st + A_STAGE + (q * NT + w * 64) * 16), 16, (int)voff, y * 128 + q * (NT / 8) * p.pitch, 0, 0);
        };
        if (steps) load(lds, 0);
        for (int y = 0; y < steps; ++y) {
            __syncthreads(); // step y has landed, and all waves have read the stage of step y - 1
            LCMA_LDS char *st = lds + (y & 1) * STAGE;
            if (y + 1 < steps) load(lds + (~y & 1) * STAGE, y + 1);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                i32x4 a[NMI], b[NNI];
#pragma unroll
                for (int i = 0; i < NMI; ++i) {
                    const int row = (wm * NMI + i) * 32 + (lane & 31);
                    a[i] = *(const LCMA_LDS i32x4 *)(st + row * 128 + swz(row, k * 2 + (lane >> 5)) * 16);
                }
#pragma unroll
                for (int j = 0; j < NNI; ++j) {
                    const int row = (wn * NNI + j) * 32 + (lane & 31);
                    b[j] = *(const LCMA_LDS i32x4 *)(st + A_STAGE + row * 128 + swz(row, k * 2 + (lane >> 5)) * 16);
                }
#pragma unroll
                for (int i = 0; i < NMI; ++i)
#pragma unroll
                    for (int j = 0; j < NNI; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[j], a[i], acc[i][j], 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < NMI; ++i) {
            const int row = (wm * NMI + i) * 32 + (lane & 31);
            if (row >= at.rows) continue;
            const bool some = at.expert < p.experts; // rows behind the groups are zero
            const float sa = some ? p.SA[at.row0 + row] : 0.f;
            char *c = (char *)p.C + (int64_t)(at.row0 + row) * p.ldc * OUT::ES;
#pragma unroll
            for (int j = 0; j < NNI; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int col = col0 + (wn * NNI + j) * 32 + g * 8 + (lane >> 5) * 4, left = p.N - col;
                    float v[4];
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const int64_t n = (int64_t)at.expert * p.N + col + i4;
                        v[i4] = 0.f;
                        if (some && i4 < left) {
                            v[i4] = (float)acc[i][j][g * 4 + i4] * sa * p.SW[n];
                            if (p.bias) v[i4] += p.bias[n];
                        }
                    }
                    if (left > 0) i8_store4<OUT>(c + (int64_t)col * OUT::ES, v, left);
                }
        }
    }
};

} // namespace lcma
