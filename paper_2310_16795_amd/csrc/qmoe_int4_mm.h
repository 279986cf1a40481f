// Four-bit weights: the product for many tokens.  Each qmoe_int4_mm_*.hip compiles its share of the variants.
#pragma once

#include "qmoe_int4.h"

namespace qmoe {
namespace {

// A workgroup of four wavefronts multiplies 256 rows (gated: 128 of each projection) with 64 tokens, 128 columns a step: four tiles of 16 rows
// a wavefront, 64 matrix instructions a step.
// The activations go through LDS in two turns and are read by all four; a wavefront's weights are its alone: loaded 64 bytes a row,
// brought to their lanes by ds_bpermute and decoded (int4_weights) 32 columns at a time, right before the 16 matrix instructions that use
// them, so that decoding one tile runs beside multiplying the one before and few registers hold operands.  Two wavefronts a SIMD: the
// sums (64 registers) are scaled into the result (64) in fp32, which accumulation registers could not take part in.
// Scales and zero points of kMmAtOnce groups lie in LDS, a wavefront's own.
// 12288 x 2080 (gated, groups of 128), 4001 tokens: 271 to 281 us back to back, 730 to 760 TFLOP/s; of a launch's cycles vector instructions are issued in 63 % (decoding is 53 %
// of them, scaling 13), the matrix cores are busy in 31 and LDS in about 40, its bank conflicts among them, at two wavefronts a SIMD and with a barrier a step: three pipes that overlap in part.
// The library's bf16 product of that shape is 196 us, without the activation.  With zero points 300, groups of 64 332, groups of 32 412: the zero points' constants spill 50 to 120
// bytes a lane.
constexpr int kMmRows = 4, kMmTiles = 4, kMmAtOnce = 32;

template <bool GATED, bool ZEROS, int PER_BLOCK>
__global__ __launch_bounds__(256, 2) void k_int4_mm(const Int4Args a)
{
    constexpr int TOKENS = 16 * kMmTiles, OUT_TILES = GATED ? kMmRows / 2 : kMmRows, LD = kInt4BlockCols + 8;
    constexpr int LD_SCALE = kMmAtOnce + 8, LD_ZERO = kMmAtOnce + 8;
    __shared__ __align__(16) uint16_t s_x[2][TOKENS * LD];
    __shared__ __align__(16) uint16_t s_scale[4][16 * kMmRows * LD_SCALE];
    __shared__ __align__(16) uint8_t s_zero[4][ZEROS ? 16 * kMmRows * LD_ZERO : 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n16 = lane & 15, quarter = lane >> 4, from_lane = 4 * (4 * n16 + quarter);
    const int piece = threadIdx.x & 15, stager = threadIdx.x >> 4;  // stages 8 columns of tokens stager + 16 t
    const int row_blocks = (a.rows + 64 * OUT_TILES - 1) / (64 * OUT_TILES);
    const int n_items = (a.batch + TOKENS - 1) / TOKENS;
    const long long total = (long long)n_items * row_blocks;
    const size_t row_bytes = (size_t)64 * a.blocks;
    const Int4Matrix m{a.weights, (gp_u16)a.scale, (gp_bytes)a.zero};
    for (long long unit = blockIdx.x; unit < total; unit += gridDim.x) {
        // Workgroups go to the eight XCDs in turn: an XCD's units follow each other and go by eight tiles of tokens, so that what it holds at a
        // time shares rows and activations in its L2.
        const long long whole = total / 8 * 8, at = unit < whole ? (unit & 7) * (whole / 8) + (unit >> 3) : unit;
        const int tiles8 = n_items / 8;  // whole groups of eight tiles
        const int group = (int)(at / (8LL * row_blocks)), in = (int)(at - group * 8LL * row_blocks);
        const int wide = group < tiles8 ? 8 : n_items - 8 * tiles8;
        const int rb = in / wide, token0 = (8 * group + in % wide) * TOKENS, ntok = min(TOKENS, a.batch - token0);
        const int first = 16 * OUT_TILES * (4 * rb + wave);  // row of this wavefront
        // the matrix's row that a tile's row is
        auto row_of = [&](int r, int in_tile) {
            return (size_t)(min(first + 16 * (r % OUT_TILES) + in_tile, a.rows - 1) + (r / OUT_TILES) * a.rows);
        };
        const uint8_t *w_row[kMmRows];
#pragma unroll
        for (int r = 0; r < kMmRows; r++) w_row[r] = m.weights + row_of(r, lane >> 2) * row_bytes + 16 * (lane & 3);
        const uint16_t *x_row[kMmTiles];
#pragma unroll
        for (int t = 0; t < kMmTiles; t++) x_row[t] = a.x + (size_t)(token0 + min(16 * t + stager, ntok - 1)) * a.ld_x;
        u32x4 x_next[kMmTiles], w_next[kMmRows];
        auto load = [&](int blk) {
#pragma unroll
            for (int t = 0; t < kMmTiles; t++) x_next[t] = int4_x_load(x_row[t], kInt4BlockCols * blk + 8 * piece, a.cols);
#pragma unroll
            for (int r = 0; r < kMmRows; r++) w_next[r] = *(gp_u32x4)(w_row[r] + (size_t)64 * blk);
        };
        auto stage = [&](int blk, int buf) {
            if (kInt4BlockCols * (blk + 1) > a.cols) {
#pragma unroll
                for (int t = 0; t < kMmTiles; t++) x_next[t] = int4_x_end(x_next[t], kInt4BlockCols * blk + 8 * piece, a.cols);
            }
#pragma unroll
            for (int t = 0; t < kMmTiles; t++) {
                const int token = 16 * t + stager;
                *reinterpret_cast<u32x4 *>(&s_x[buf][token * LD + 8 * piece]) = x_next[t];
            }
        };
        // groups g0 .. g0 + kMmAtOnce - 1 of the wavefront's 64 rows: four lanes a row, eight groups a lane
        auto fill = [&](int g0) {
#pragma unroll
            for (int r = 0; r < kMmRows; r++) {
                const int in_tile = lane >> 2, at8 = 8 * (lane & 3);
                const size_t row = row_of(r, in_tile) * a.groups;
                uint16_t *to = &s_scale[wave][(16 * r + in_tile) * LD_SCALE + at8];
                uint8_t *to_zero = &s_zero[wave][ZEROS ? (16 * r + in_tile) * LD_ZERO + at8 : 0];
                if (g0 + at8 + 8 <= a.groups) {
                    uint32_t v[4], z[2] = {0x08080808u, 0x08080808u};
                    int4_load_packed<16>(v, m.scale + (row + g0 + at8));
                    if (ZEROS && m.zero) int4_load_packed<8>(z, m.zero + (row + g0 + at8));
                    *reinterpret_cast<u32x4 *>(to) = (u32x4){v[0], v[1], v[2], v[3]};
                    if constexpr (ZEROS) *reinterpret_cast<uint2 *>(to_zero) = make_uint2(z[0], z[1]);
                } else {
                    for (int i = 0; i < 8; i++) {  // 0 behind the last group: its columns are none, but what lies there could be infinite
                        const bool is = g0 + at8 + i < a.groups;
                        to[i] = is ? m.scale[row + g0 + at8 + i] : 0;
                        if constexpr (ZEROS) to_zero[i] = is && m.zero ? m.zero[row + g0 + at8 + i] : 8;
                    }
                }
            }
        };
        f32x4 acc[kMmRows][kMmTiles];
#pragma unroll
        for (int r = 0; r < kMmRows; r++)
#pragma unroll
            for (int t = 0; t < kMmTiles; t++) acc[r][t] = (f32x4){0, 0, 0, 0};
        load(0);
        __syncthreads();  // the unit before has read its last step
        stage(0, 0);
        __syncthreads();
        const int x_at = n16 * LD + 8 * quarter;
        const int span = a.blocks_per_group > 1 ? kMmAtOnce * a.blocks_per_group : kMmAtOnce / PER_BLOCK;  // blocks whose scales lie in LDS
        for (int s0 = 0; s0 < a.blocks; s0 += span) {
            const int g_from = a.blocks_per_group > 1 ? s0 / a.blocks_per_group : s0 * PER_BLOCK, s1 = min(a.blocks, s0 + span);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();  // the wavefront has read those before
            fill(g_from);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            for (int blk = s0; blk < s1; blk++) {
                const int buf = blk & 1;
                uint32_t w[kMmRows][4];
#pragma unroll
                for (int r = 0; r < kMmRows; r++)
#pragma unroll
                    for (int s = 0; s < 4; s++) w[r][s] = (uint32_t)__builtin_amdgcn_ds_bpermute(from_lane, (int)w_next[r][s]);
                load(min(blk + 1, a.blocks - 1));
                const int g_at = (a.blocks_per_group > 1 ? blk / a.blocks_per_group : blk * PER_BLOCK) - g_from;
                f32x4 sum[kMmRows][kMmTiles];
                Int4Zero zero[kMmRows];
#pragma unroll
                for (int s = 0; s < 4; s++) {
                    const int g = s * PER_BLOCK / 4;
                    __builtin_amdgcn_sched_barrier(0);  // (operands of several turns at once would not fit the registers)
                    bf16x8 xf[kMmTiles];
#pragma unroll
                    for (int t = 0; t < kMmTiles; t++) xf[t] = *reinterpret_cast<const bf16x8 *>(&s_x[buf][x_at + 16 * t * LD + 32 * s]);
                    if (s * PER_BLOCK % 4 == 0) {
#pragma unroll
                        for (int r = 0; r < kMmRows; r++) {
                            zero[r] = int4_zero(ZEROS ? s_zero[wave][(16 * r + n16) * LD_ZERO + g_at + g] : 8u);
#pragma unroll
                            for (int t = 0; t < kMmTiles; t++) sum[r][t] = (f32x4){0, 0, 0, 0};
                        }
                    }
#pragma unroll
                    for (int r = 0; r < kMmRows; r++) {
                        const bf16x8 wf = int4_weights(w[r][s], zero[r]);
#pragma unroll
                        for (int t = 0; t < kMmTiles; t++) sum[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[t], wf, sum[r][t], 0, 0, 0);
                    }
                    if ((s + 1) * PER_BLOCK % 4) continue;
#pragma unroll
                    for (int r = 0; r < kMmRows; r++) {
                        const float scale = int4_scale(s_scale[wave][(16 * r + n16) * LD_SCALE + g_at + g]);
#pragma unroll
                        for (int t = 0; t < kMmTiles; t++)
#pragma unroll
                            for (int i = 0; i < 4; i++) acc[r][t][i] = fmaf(scale, sum[r][t][i], acc[r][t][i]);
#pragma unroll
                        for (int t = 0; t < kMmTiles; t++) int4_now(acc[r][t]);
                    }
                }
                if (blk + 1 < a.blocks) stage(blk + 1, buf ^ 1);
                __syncthreads();
            }
        }
#pragma unroll
        for (int t = 0; t < kMmTiles; t++) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int in_tile = 16 * t + 4 * quarter + i;
                if (in_tile >= ntok) continue;
#pragma unroll
                for (int r = 0; r < OUT_TILES; r++) {
                    const int row = first + 16 * r + n16;
                    if (row >= a.rows) continue;
                    float v = acc[r][t][i];
                    if constexpr (GATED) v = int4_gated(v, acc[r + OUT_TILES][t][i], a.activation);
                    int4_store(a, token0 + in_tile, 1.0f, row, v);
                }
            }
        }
    }
}

template <bool GATED, bool ZEROS>
qmoe_status launch_mm(const Int4Args &a, int grid, hipStream_t s)
{
    const dim3 g(grid), b(256);
    if (a.per_block == 1) hipLaunchKernelGGL((k_int4_mm<GATED, ZEROS, 1>), g, b, 0, s, a);
    else if (a.per_block == 2) hipLaunchKernelGGL((k_int4_mm<GATED, ZEROS, 2>), g, b, 0, s, a);
    else hipLaunchKernelGGL((k_int4_mm<GATED, ZEROS, 4>), g, b, 0, s, a);
    QMOE_HIP_TRY(hipGetLastError());
    return QMOE_OK;
}

}  // namespace
}  // namespace qmoe
