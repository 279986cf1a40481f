// Four-bit weights: the product for many tokens.  Each qmoe_int4_mm_*.hip compiles its share of the variants.
#pragma once

#include "qmoe_int4.h"

namespace qmoe {
namespace {

// A workgroup of four wavefronts multiplies 64 * ROWS rows (gated: 32 * ROWS of each projection) with 16 * TILES tokens, 128 columns
// at a time.  The activations of a step go through LDS, which all four read; the weights of a row are one
// wavefront's alone and go from memory into its registers, 16 bytes a lane, and there become the operands of the matrix
// instruction (int4_plus16): decoded once for all the tokens of the tile.
// With PER_BLOCK groups of 128 / PER_BLOCK columns, a group's sum starts at -(16 + z) * sum of x (the sums of x are formed by
// those who stage it) and is scaled into the result in fp32.
constexpr int kMmWaves = 4;
constexpr int kXRow = kInt4BlockCols + 8;  // bf16 values from a token's row in LDS to the next: 16 lanes' 16-byte reads meet no bank twice

template <int ROWS, int TILES, bool GATED, bool ZEROS, int PER_BLOCK>
__global__ __launch_bounds__(64 * kMmWaves, TILES == 8 ? 1 : 2) void k_int4_mm(const Int4Args a)
{
    constexpr int TOKENS = 16 * TILES, OUT_TILES = GATED ? ROWS / 2 : ROWS;
    __shared__ __align__(16) uint16_t s_x[2][TOKENS * kXRow];
    __shared__ __align__(16) float s_sum[2][PER_BLOCK][TOKENS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n16 = lane & 15, quarter = lane >> 4;
    const int piece = threadIdx.x & 15, stager = threadIdx.x >> 4;  // stages 8 columns of tokens stager + 16 i
    const int row_blocks = (a.rows + 16 * OUT_TILES * kMmWaves - 1) / (16 * OUT_TILES * kMmWaves);
    const int n_items = a.items ? min(*a.n_items_dev, a.max_items) : (a.batch + TOKENS - 1) / TOKENS;
    const long long total = (long long)n_items * row_blocks;
    const size_t row_bytes = (size_t)64 * a.blocks;
    for (long long unit = blockIdx.x; unit < total; unit += gridDim.x) {
        const int item = (int)(unit / row_blocks), rb = (int)(unit - (long long)item * row_blocks);
        int expert = 0, slot0 = item * TOKENS, ntok = min(TOKENS, a.batch - slot0);
        if (a.items) {
            const Item it = a.items[item];
            expert = it.expert, slot0 = it.slot0, ntok = min(it.ntok, TOKENS);
        }
        const int tiles = (ntok + 15) / 16;
        const Int4Matrix m = int4_matrix(a, expert);
        const int tile0 = (rb * kMmWaves + wave) * OUT_TILES;
        const uint8_t *w_row[ROWS];
        size_t meta[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; r++) {
            const int row = min(16 * (tile0 + r % OUT_TILES) + n16, a.rows - 1) + (r / OUT_TILES) * a.rows;
            w_row[r] = m.weights + (size_t)row * row_bytes + 16 * quarter;
            meta[r] = (size_t)row * a.groups;
        }
        const uint16_t *x_row[TILES];
#pragma unroll
        for (int t = 0; t < TILES; t++) {
            const int slot = slot0 + min(16 * t + stager, ntok - 1);
            x_row[t] = a.x + (size_t)(a.perm && !a.x_by_slot ? a.perm[slot] : slot) * a.ld_x;
        }
        u32x4 x_next[TILES], w_next[ROWS];
        uint16_t scale_next[ROWS][PER_BLOCK];
        uint8_t zero_next[ROWS][PER_BLOCK];
        auto load_x = [&](int blk) {
#pragma unroll
            for (int t = 0; t < TILES; t++)
                if (t < tiles) x_next[t] = int4_x(x_row[t], kInt4BlockCols * blk + 8 * piece, a.cols, kInt4BlockCols * (blk + 1) <= a.cols);
        };
        auto load_w = [&](int blk) {
#pragma unroll
            for (int r = 0; r < ROWS; r++) {
                w_next[r] = *(gp_u32x4)(w_row[r] + (size_t)64 * blk);
#pragma unroll
                for (int g = 0; g < PER_BLOCK; g++) {
                    const int of = PER_BLOCK > 1 ? blk * PER_BLOCK + g : (int)((uint32_t)blk / (uint32_t)a.blocks_per_group);
                    const size_t at = meta[r] + min(of, a.groups - 1);
                    scale_next[r][g] = m.scale[at];
                    if constexpr (ZEROS) zero_next[r][g] = m.zero ? m.zero[at] : 8;
                }
            }
        };
        auto stage_x = [&](int buf) {
#pragma unroll
            for (int t = 0; t < TILES; t++) {
                if (t >= tiles) break;
                const int token = 16 * t + stager;
                *reinterpret_cast<u32x4 *>(&s_x[buf][token * kXRow + 8 * piece]) = x_next[t];
                const float s = int4_group_sum<PER_BLOCK>(x_next[t]);
                if ((piece + 1) % (16 / PER_BLOCK) == 0) s_sum[buf][piece / (16 / PER_BLOCK)][token] = ZEROS ? s : -24.0f * s;
            }
        };
        f32x4 acc[ROWS][TILES];
#pragma unroll
        for (int r = 0; r < ROWS; r++)
#pragma unroll
            for (int t = 0; t < TILES; t++) acc[r][t] = (f32x4){0, 0, 0, 0};
        load_x(0);
        load_w(0);
        __syncthreads();  // the unit before has read its last step
        stage_x(0);
        __syncthreads();
        for (int blk = 0; blk < a.blocks; blk++) {
            const int buf = blk & 1;
            bf16x8 wf[ROWS][4];
            float scale[ROWS][PER_BLOCK], zero[ROWS][PER_BLOCK];
#pragma unroll
            for (int r = 0; r < ROWS; r++) {
#pragma unroll
                for (int s = 0; s < 4; s++) wf[r][s] = int4_plus16(w_next[r][s]);
#pragma unroll
                for (int g = 0; g < PER_BLOCK; g++) {
                    scale[r][g] = half_bits_to_float(scale_next[r][g]);
                    if constexpr (ZEROS) zero[r][g] = -16.0f - (float)zero_next[r][g];
                }
            }
            if (blk + 1 < a.blocks) {
                load_x(blk + 1);
                load_w(blk + 1);
            }
#pragma unroll
            for (int t = 0; t < TILES; t++) {
                if (t >= tiles) break;
#pragma unroll
                for (int g = 0; g < PER_BLOCK; g++) {
                    const f32x4 xs = *reinterpret_cast<const f32x4 *>(&s_sum[buf][g][16 * t + 4 * quarter]);
                    f32x4 sum[ROWS];
#pragma unroll
                    for (int r = 0; r < ROWS; r++) sum[r] = ZEROS ? xs * zero[r][g] : xs;
#pragma unroll
                    for (int s = g * 4 / PER_BLOCK; s < (g + 1) * 4 / PER_BLOCK; s++) {
                        const bf16x8 xf = *reinterpret_cast<const bf16x8 *>(&s_x[buf][(16 * t + n16) * kXRow + 32 * s + 8 * quarter]);
#pragma unroll
                        for (int r = 0; r < ROWS; r++) sum[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf, wf[r][s], sum[r], 0, 0, 0);
                    }
#pragma unroll
                    for (int r = 0; r < ROWS; r++)
#pragma unroll
                        for (int i = 0; i < 4; i++) acc[r][t][i] = fmaf(scale[r][g], sum[r][i], acc[r][t][i]);
                }
            }
            if (blk + 1 < a.blocks) stage_x(buf ^ 1);
            __syncthreads();
        }
#pragma unroll
        for (int t = 0; t < TILES; t++) {
            if (t >= tiles) break;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int in_tile = 16 * t + 4 * quarter + i;
                if (in_tile >= ntok) continue;
                const int token = a.perm ? a.perm[slot0 + in_tile] : slot0 + in_tile;
                const float gate = a.gate ? a.gate[token] : 1.0f;
#pragma unroll
                for (int r = 0; r < OUT_TILES; r++) {
                    const int row = 16 * (tile0 + r) + n16;
                    if (row >= a.rows) continue;
                    float v = acc[r][t][i];
                    if constexpr (GATED) v = int4_gated(v, acc[r + OUT_TILES][t][i], a.activation);
                    int4_store(a, a.out_by_slot ? slot0 + in_tile : token, gate, row, v);
                }
            }
        }
    }
}

template <int ROWS, int TILES, bool GATED, bool ZEROS>
qmoe_status launch_shape(const Int4Args &a, long long items, int cus, hipStream_t s)
{
    const int block_rows = 16 * (GATED ? ROWS / 2 : ROWS) * kMmWaves;
    const int grid = (int)std::min<long long>(items * ((a.rows + block_rows - 1) / block_rows), 16LL * cus);
    const dim3 g(grid), b(64 * kMmWaves);
    if (a.per_block == 1) hipLaunchKernelGGL((k_int4_mm<ROWS, TILES, GATED, ZEROS, 1>), g, b, 0, s, a);
    else if (a.per_block == 2) hipLaunchKernelGGL((k_int4_mm<ROWS, TILES, GATED, ZEROS, 2>), g, b, 0, s, a);
    else hipLaunchKernelGGL((k_int4_mm<ROWS, TILES, GATED, ZEROS, 4>), g, b, 0, s, a);
    QMOE_HIP_TRY(hipGetLastError());
    return QMOE_OK;
}

template <bool GATED, bool ZEROS>
qmoe_status launch_mm(const Int4Args &a, int cus, hipStream_t s)
{
    if (a.items) return launch_shape<2, 4, GATED, ZEROS>(a, a.max_items, cus, s);
    const long long tiles128 = (a.batch + 127) / 128, blocks = (a.rows + (GATED ? 127 : 255)) / (GATED ? 128 : 256);
    if (tiles128 * blocks >= cus) return launch_shape<4, 8, GATED, ZEROS>(a, tiles128, cus, s);
    const long long tiles64 = (a.batch + 63) / 64;
    if (tiles64 * blocks >= cus) return launch_shape<4, 4, GATED, ZEROS>(a, tiles64, cus, s);
    return launch_shape<2, 4, GATED, ZEROS>(a, tiles64, cus, s);
}

}  // namespace
}  // namespace qmoe
