// Four-bit weights: the product for few tokens, and the C entry points.
#include "qmoe_int4.h"

namespace qmoe {
namespace {

constexpr int kInt4MaxSplit = 8;

// Sixteen rows of a matrix (gated: and the sixteen of the other projection) times up to 16 * TILES tokens.
//
// v_mfma_f32_16x16x32_bf16 takes 16 tokens as its first operand and 16 rows as its second, so a result lane holds one
// row and four tokens and needs one scale.  A lane's 16 bytes of a row are its operands for four steps of 32 columns; weights go
// straight from memory into them, each read once per tile of tokens, and become 16 + q with two instructions a pair.
// What the zero points (and the 16) take off is (16 + z) * sum of x over the group: a second MFMA with ones gives those
// sums in the place where they are needed; the matrix cores have the time, since reading the weights is what bounds the kernel.
// `split` wavefronts share the rows along the columns, so that a single matrix fills the GPU, and join through LDS
// in a fixed order.
template <int TILES, bool GATED>
__global__ __launch_bounds__(512) void k_int4_rows(const Int4Args a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr int SIDES = GATED ? 2 : 1;
    constexpr int AHEAD = TILES == 1 ? 4 : 2;  // blocks whose weights are asked for together
    f32x4 *joined = reinterpret_cast<f32x4 *>(smem);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int part = wave % a.split, in_group = wave / a.split, side_by_side = (int)(blockDim.x >> 6) / a.split;
    const int n16 = lane & 15, quarter = lane >> 4;
    const int row_tiles = (a.rows + 15) / 16, units_per_item = (row_tiles + side_by_side - 1) / side_by_side;
    const int n_items = a.items ? min(*a.n_items_dev, a.max_items) : (a.batch + 16 * TILES - 1) / (16 * TILES);
    const long long total = (long long)n_items * units_per_item;
    const int b0 = (int)((long long)a.blocks * part / a.split), b1 = (int)((long long)a.blocks * (part + 1) / a.split);
    const size_t row_bytes = (size_t)64 * a.blocks;
    const bf16x8 ones = __builtin_bit_cast(bf16x8, (u32x4){0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
    for (long long unit = blockIdx.x; unit < total; unit += gridDim.x) {
        const int item = (int)(unit / units_per_item), tile = (int)(unit - (long long)item * units_per_item) * side_by_side + in_group;
        int expert = 0, slot0 = item * 16 * TILES, ntok = min(16 * TILES, a.batch - slot0);
        if (a.items) {
            const Item it = a.items[item];
            expert = it.expert, slot0 = it.slot0, ntok = min(it.ntok, 16 * TILES);
        }
        const Int4Matrix m = int4_matrix(a, expert);
        const uint8_t *w_row[SIDES];
        size_t meta[SIDES];
#pragma unroll
        for (int g = 0; g < SIDES; g++) {
            const int r = min(16 * tile + n16, a.rows - 1) + g * a.rows;
            w_row[g] = m.weights + (size_t)r * row_bytes + 16 * quarter;
            meta[g] = (size_t)r * a.groups;
        }
        const uint16_t *x_row[TILES];
#pragma unroll
        for (int t = 0; t < TILES; t++) {
            const int slot = slot0 + min(16 * t + n16, ntok - 1);
            x_row[t] = a.x + (size_t)(a.perm && !a.x_by_slot ? a.perm[slot] : slot) * a.ld_x;
        }
        f32x4 acc[SIDES][TILES], sum[SIDES][TILES], ones_sum[TILES];
#pragma unroll
        for (int t = 0; t < TILES; t++) {
            ones_sum[t] = (f32x4){0, 0, 0, 0};
#pragma unroll
            for (int g = 0; g < SIDES; g++) acc[g][t] = sum[g][t] = (f32x4){0, 0, 0, 0};
        }
        for (int b = b0; b < b1; b += AHEAD) {
            u32x4 w[AHEAD][SIDES];
            float scale[AHEAD][SIDES][4], zero[AHEAD][SIDES][4];
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                const int blk = min(b + u, b1 - 1);
#pragma unroll
                for (int g = 0; g < SIDES; g++) w[u][g] = *(gp_u32x4)(w_row[g] + (size_t)64 * blk);
            }
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                const int blk = min(b + u, b1 - 1);
#pragma unroll
                for (int g = 0; g < SIDES; g++)
#pragma unroll
                    for (int s = 0; s < 4; s++) {
                        // the group that ends with step s, if one does
                        if (((s + 1) * a.per_block) & 3) continue;
                        const int of = a.blocks_per_group > 1 ? blk / a.blocks_per_group
                                                              : blk * a.per_block + ((s + 1) * a.per_block) / 4 - 1;
                        const size_t at = meta[g] + min(of, a.groups - 1);
                        scale[u][g][s] = half_bits_to_float(m.scale[at]);
                        zero[u][g][s] = m.zero ? 16.0f + (float)m.zero[at] : 24.0f;
                    }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                if (b + u >= b1) break;
                const int c = kInt4BlockCols * (b + u) + 8 * quarter;
#pragma unroll
                for (int s = 0; s < 4; s++) {
                    bf16x8 wf[SIDES];
#pragma unroll
                    for (int g = 0; g < SIDES; g++) wf[g] = int4_plus16(w[u][g][s]);
#pragma unroll
                    for (int t = 0; t < TILES; t++) {
                        const bf16x8 xf = __builtin_bit_cast(bf16x8, int4_x(x_row[t], c + 32 * s, a.cols));
                        ones_sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf, ones, ones_sum[t], 0, 0, 0);
#pragma unroll
                        for (int g = 0; g < SIDES; g++)
                            sum[g][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf, wf[g], sum[g][t], 0, 0, 0);
                    }
                    if (((s + 1) * a.per_block) & 3) continue;
#pragma unroll
                    for (int t = 0; t < TILES; t++) {
#pragma unroll
                        for (int g = 0; g < SIDES; g++) {
#pragma unroll
                            for (int i = 0; i < 4; i++)
                                acc[g][t][i] = fmaf(scale[u][g][s], fmaf(-zero[u][g][s], ones_sum[t][i], sum[g][t][i]), acc[g][t][i]);
                            sum[g][t] = (f32x4){0, 0, 0, 0};
                        }
                        ones_sum[t] = (f32x4){0, 0, 0, 0};
                    }
                }
            }
        }
        if (a.split > 1) {
            f32x4 *mine = joined + (size_t)(in_group * a.split) * SIDES * TILES * 64;
#pragma unroll
            for (int g = 0; g < SIDES; g++)
#pragma unroll
                for (int t = 0; t < TILES; t++) mine[((part * SIDES + g) * TILES + t) * 64 + lane] = acc[g][t];
            __syncthreads();
        }
        const int r = 16 * tile + n16;
#pragma unroll
        for (int t = 0; t < TILES; t++) {
            if (t % a.split != part) continue;  // a tile of tokens is joined by one of the wavefronts
            if (16 * t >= ntok) break;
            if (a.split > 1) {
                const f32x4 *mine = joined + (size_t)(in_group * a.split) * SIDES * TILES * 64;
#pragma unroll
                for (int g = 0; g < SIDES; g++) {
                    f32x4 v = mine[(g * TILES + t) * 64 + lane];
                    for (int p = 1; p < a.split; p++) v += mine[((p * SIDES + g) * TILES + t) * 64 + lane];
                    acc[g][t] = v;
                }
            }
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int in_tile = 16 * t + 4 * quarter + i;
                if (in_tile >= ntok || r >= a.rows) continue;
                const int token = a.perm ? a.perm[slot0 + in_tile] : slot0 + in_tile;
                float v = acc[0][t][i];
                if constexpr (GATED) v = int4_gated(v, acc[1][t][i], a.activation);
                int4_store(a, a.out_by_slot ? slot0 + in_tile : token, a.gate ? a.gate[token] : 1.0f, r, v);
            }
        }
        if (a.split > 1) __syncthreads();  // before the next unit's sums overwrite these
    }
}

bool group_ok(int group) { return group == 32 || group == 64 || (group > 0 && group % kInt4BlockCols == 0); }

// rows: results a token
void fill_shape(Int4Args *a, int rows, int cols, int group)
{
    a->rows = rows;
    a->cols = cols;
    a->blocks = (cols + kInt4BlockCols - 1) / kInt4BlockCols;
    a->groups = (int)(((long long)cols + group - 1) / group);
    a->per_block = group < kInt4BlockCols ? kInt4BlockCols / group : 1;
    a->blocks_per_group = group < kInt4BlockCols ? 1 : group / kInt4BlockCols;
}

template <int TILES>
qmoe_status launch_tiles(const Int4Args &a, int grid, int threads, hipStream_t s)
{
    const size_t smem = a.split > 1 ? (size_t)(threads / 64) * (int4_is_gated(a.activation) ? 2 : 1) * TILES * 64 * sizeof(f32x4) : 0;
    if (int4_is_gated(a.activation)) {
        const qmoe_status st = allow_lds(k_int4_rows<TILES, true>, smem);
        if (st != QMOE_OK) return st;
        hipLaunchKernelGGL((k_int4_rows<TILES, true>), dim3(grid), dim3(threads), smem, s, a);
    } else {
        const qmoe_status st = allow_lds(k_int4_rows<TILES, false>, smem);
        if (st != QMOE_OK) return st;
        hipLaunchKernelGGL((k_int4_rows<TILES, false>), dim3(grid), dim3(threads), smem, s, a);
    }
    QMOE_HIP_TRY(hipGetLastError());
    return QMOE_OK;
}

// tiles: tiles of 16 tokens of an item; items: how many the call has, about
qmoe_status launch_rows_kernel(Int4Args a, int tiles, long long items, int cus, hipStream_t s)
{
    const long long units = items * ((a.rows + 15) / 16);
    a.split = 1;
    while (a.split < kInt4MaxSplit && units * a.split < 8LL * cus && 2 * a.split <= a.blocks) a.split *= 2;
    const int threads = 64 * (a.split < 4 ? 4 : a.split);
    const int side_by_side = threads / 64 / a.split;
    const long long groups = items * (((a.rows + 15) / 16 + side_by_side - 1) / side_by_side);
    const int grid = (int)std::min<long long>(groups, 64LL * cus);
    if (tiles <= 1) return launch_tiles<1>(a, grid, threads, s);
    if (tiles <= 2) return launch_tiles<2>(a, grid, threads, s);
    return launch_tiles<4>(a, grid, threads, s);
}

// zeros: a matrix has zero points (descriptors in device memory: may have)
qmoe_status launch_mm_kernel(const Int4Args &a, bool zeros, int cus, hipStream_t s)
{
    if (int4_is_gated(a.activation)) return zeros ? launch_int4_mm_gated_zeros(a, cus, s) : launch_int4_mm_gated(a, cus, s);
    return zeros ? launch_int4_mm_zeros(a, cus, s) : launch_int4_mm_plain(a, cus, s);
}

}  // namespace
}  // namespace qmoe

using namespace qmoe;

extern "C" {

qmoe_status qmoe_int4_matvec(const qmoe_int4_matrix *W, const uint16_t *x_bf16, size_t ld_x, int batch, int activation, void *y,
                             int y_type, size_t ld_y, void *stream)
{
    if (!W || !W->weights || !W->scale_f16 || !x_bf16 || !y || W->rows < 1 || W->cols < 1 || batch < 1 || !group_ok(W->group) ||
        W->reserved || reinterpret_cast<uintptr_t>(W->weights) % 16 || (y_type != QMOE_F32 && y_type != QMOE_BF16) ||
        activation < QMOE_ACT_NONE || activation > QMOE_ACT_GELU_GATED || (int4_is_gated(activation) && W->rows % 2))
        return QMOE_E_INVALID_ARG;
    const int rows = int4_is_gated(activation) ? W->rows / 2 : W->rows;
    if (ld_x < (size_t)W->cols || ld_y < (size_t)rows) return QMOE_E_INVALID_ARG;
    if (W->rows > kMaxInt4Rows || W->cols > kMaxInt4Cols || batch > kMaxTokens) return QMOE_E_LIMIT;
    DeviceInfo di;
    const qmoe_status st = gpu_info(&di);
    if (st != QMOE_OK) return st;
    Int4Args a{};
    a.weights = W->weights;
    a.scale = W->scale_f16;
    a.zero = W->zero;
    a.batch = batch;
    a.x = x_bf16;
    a.ld_x = ld_x;
    a.out = y;
    a.ld_out = ld_y;
    a.out_f32 = y_type == QMOE_F32;
    a.activation = activation;
    fill_shape(&a, rows, W->cols, W->group);
    if (batch > 64) return launch_mm_kernel(a, a.zero != nullptr, di.cus, static_cast<hipStream_t>(stream));
    const int tiles = (batch + 15) / 16, at_once = tiles <= 2 ? tiles : 4;
    return launch_rows_kernel(a, tiles, (tiles + at_once - 1) / at_once, di.cus, static_cast<hipStream_t>(stream));
}

qmoe_status qmoe_int4_layer_forward(const qmoe_int4_matrix *wi, const qmoe_int4_matrix *wo, int group, int activation, int n_experts,
                                    int d_model, int d_ff, const uint16_t *x_bf16, const int32_t *expert_idx, const float *gate,
                                    int n_tokens, void *y, int y_type, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!wi || !wo || !x_bf16 || !expert_idx || !y || !group_ok(group) || (activation != QMOE_ACT_RELU && !int4_is_gated(activation)) ||
        (y_type != QMOE_F32 && y_type != QMOE_BF16) || d_model % 8 || d_ff % 8 || reinterpret_cast<uintptr_t>(x_bf16) % 16 ||
        reinterpret_cast<uintptr_t>(y) % 4)
        return QMOE_E_INVALID_ARG;
    qmoe_status st = layer_workspace_ok(n_tokens, n_experts, d_model, d_ff, workspace, workspace_bytes);
    if (st != QMOE_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    DeviceInfo di;
    if ((st = gpu_info(&di)) != QMOE_OK) return st;
    GroupedTokens g;
    if ((st = group_by_expert(expert_idx, n_tokens, n_experts, d_model, d_ff, workspace, static_cast<float *>(y),
                              y_type == QMOE_F32 ? d_model : d_model / 2, s, &g)) != QMOE_OK)
        return st;
    Int4Args a{};
    a.mats = wi;
    a.items = g.items;
    a.n_items_dev = g.n_items;
    a.max_items = g.max_items;
    a.n_experts = n_experts;
    a.perm = g.perm;
    a.x = x_bf16;
    a.ld_x = d_model;
    a.out = g.hidden;
    a.ld_out = d_ff;
    a.out_by_slot = 1;
    a.activation = activation;
    fill_shape(&a, d_ff, d_model, group);
    const int items = std::min(n_tokens, n_experts + n_tokens / kMmTokens);
    const bool mm = n_tokens >= 4 * n_experts && n_tokens > 64;
    if ((st = mm ? launch_mm_kernel(a, true, di.cus, s) : launch_rows_kernel(a, 4, items, di.cus, s)) != QMOE_OK) return st;
    a.mats = wo;
    a.x = g.hidden;
    a.ld_x = d_ff;
    a.x_by_slot = 1;
    a.out = y;
    a.ld_out = d_model;
    a.out_by_slot = 0;
    a.out_f32 = y_type == QMOE_F32;
    a.gate = gate;
    a.activation = QMOE_ACT_NONE;
    fill_shape(&a, d_model, d_ff, group);
    return mm ? launch_mm_kernel(a, true, di.cus, s) : launch_rows_kernel(a, 4, items, di.cus, s);
}

}  // extern "C"
