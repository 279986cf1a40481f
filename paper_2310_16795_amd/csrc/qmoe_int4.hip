// Four-bit weights: the product for few tokens, and the C entry points.
#include "qmoe_int4.h"

namespace qmoe {
namespace {

constexpr int kInt4MaxSplit = 8;
constexpr size_t kInt4XBytes = 32 * 1024;  // of activations in a workgroup's LDS: 64 tokens' 256 columns and more
constexpr int kInt4FewTokens = 16;  // of an expert: a tile of k_int4_rows
constexpr int kInt4AllFew = 64;     // layer calls of up to so many tokens leave all of them to it

// Two tiles of sixteen rows of a matrix (gated: of the gate and the same ones of the other projection) times up to 16 * TILES tokens.
//
// v_mfma_f32_16x16x32_bf16 takes 16 tokens as its first operand and 16 rows as its second, so a result lane holds one
// row and four tokens and needs one scale.  16 bytes of a row are a lane's operands for four steps of 32 columns and become 16 + q with two
// instructions a pair.  What the zero points (and the 16) take off is (16 + z) * sum of x over the group, where a group's sum starts;
// the sums of x are formed by those who bring x into LDS.
// Four neighbouring lanes load the 64 bytes that a row has in a block (one access of the cache; a load in the operands' order, a row a
// lane, is four), and ds_bpermute brings them to their lanes.  Scales come for four steps at a time, a step's to a quarter of the
// wavefront each.  The activations of the tokens lie in LDS, a piece of the columns at a time if they must, for all wavefronts
// of the workgroup and `reps` tiles of each.
// `split` wavefronts share the rows along the columns, so that a single matrix fills the GPU, and join through LDS
// in a fixed order.
template <int TILES, int PER_BLOCK>
__global__ __launch_bounds__(64 * kInt4MaxSplit, TILES == 1 ? 4 : 2) void k_int4_rows(const Int4Args a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr int AHEAD = 2, GROUPS = AHEAD * PER_BLOCK;  // blocks of a step, and the groups in them
    constexpr int WORDS = (GROUPS + 1) / 2, ZERO_WORDS = (GROUPS + 3) / 4;
    uint16_t *s_x = reinterpret_cast<uint16_t *>(smem);
    float *s_sum = reinterpret_cast<float *>(smem + a.x_bytes);  // [group of the piece of columns][16 * TILES tokens]
    f32x4 *joined = reinterpret_cast<f32x4 *>(smem + a.x_bytes + a.sum_bytes);
    const bool gated = a.activation == QMOE_ACT_SILU_GATED || a.activation == QMOE_ACT_GELU_GATED;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int part = wave % a.split, in_group = wave / a.split, side_by_side = (int)(blockDim.x >> 6) / a.split;
    const int n16 = lane & 15, quarter = lane >> 4;
    const int from_lane = 4 * (4 * n16 + quarter);  // whose load holds this lane's operands, in bytes
    const int unit_rows = gated ? 16 : 32;
    const int row_tiles = (a.rows + unit_rows - 1) / unit_rows, unit_tiles = side_by_side * a.reps;
    const int units_per_item = (row_tiles + unit_tiles - 1) / unit_tiles;
    const int n_items = a.items ? min(*a.n_items_dev, a.max_items) : (a.batch + 16 * TILES - 1) / (16 * TILES);
    const long long total = (long long)n_items * units_per_item;
    const size_t row_bytes = (size_t)64 * a.blocks;
    for (long long unit = blockIdx.x; unit < total; unit += gridDim.x) {
        const int item = (int)(unit / units_per_item), first_tile = (int)(unit - (long long)item * units_per_item) * unit_tiles;
        int expert = 0, slot0 = item * 16 * TILES, ntok = min(16 * TILES, a.batch - slot0);
        if (a.items) {
            const Item it = a.items[item];
            expert = it.expert, slot0 = it.slot0, ntok = min(it.ntok, 16 * TILES);
        }
        const Int4Matrix m = int4_matrix(a, expert);
        const int fit = (int)min((a.x_bytes / 2 / (uint32_t)ntok - 8) / kInt4BlockCols, a.sum_bytes / (4 * 16 * TILES * PER_BLOCK));
        const int chunk = min(a.blocks, fit), ld_s = chunk * kInt4BlockCols + 8;
        for (int rep = 0; rep < a.reps; rep++) {
            if (first_tile + rep * side_by_side >= row_tiles) break;  // (for the whole workgroup)
            const int tile = first_tile + rep * side_by_side + in_group;
            const uint8_t *w_row[2];
            size_t meta[2];
#pragma unroll
            for (int g = 0; g < 2; g++) {
                const int base = gated ? 16 * tile : 32 * tile + 16 * g, behind = gated ? g * a.rows : 0;
                w_row[g] = m.weights + (size_t)(min(base + (lane >> 2), a.rows - 1) + behind) * row_bytes + 16 * (lane & 3);
                meta[g] = (size_t)(min(base + n16, a.rows - 1) + behind) * a.groups;
            }
            f32x4 acc[2][TILES], sum[2][TILES];
#pragma unroll
            for (int t = 0; t < TILES; t++)
#pragma unroll
                for (int g = 0; g < 2; g++) acc[g][t] = (f32x4){0, 0, 0, 0};
            for (int c0 = 0; c0 < a.blocks; c0 += chunk) {
                const int n_blocks = min(chunk, a.blocks - c0);
                const int b0 = c0 + n_blocks * part / a.split, b1 = c0 + n_blocks * (part + 1) / a.split;
                u32x4 w_next[AHEAD][2];
                auto load_w = [&](int b) {
#pragma unroll
                    for (int u = 0; u < AHEAD; u++)
#pragma unroll
                        for (int g = 0; g < 2; g++) w_next[u][g] = *(gp_u32x4)(w_row[g] + (size_t)64 * max(0, min(b + u, b1 - 1)));
                };
                load_w(b0);
                if (rep == 0 || chunk < a.blocks) {
                    __syncthreads();  // what lay there before has been read
                    const int pieces = n_blocks * (kInt4BlockCols / 8);
                    for (int i = threadIdx.x; i < ntok * pieces; i += blockDim.x) {
                        const int token = i / pieces, c = 8 * (i - token * pieces), slot = slot0 + token;
                        const uint16_t *x = a.x + (size_t)(a.perm && !a.x_by_slot ? a.perm[slot] : slot) * a.ld_x;
                        const u32x4 v = int4_x(x, kInt4BlockCols * c0 + c, a.cols);
                        *reinterpret_cast<u32x4 *>(&s_x[token * ld_s + c]) = v;
                        const float all = int4_group_sum<PER_BLOCK>(v);  // (16 lanes hold a block of a token)
                        if ((lane + 1) % (16 / PER_BLOCK) == 0) s_sum[(c / (kInt4BlockCols / PER_BLOCK)) * (16 * TILES) + token] = all;
                    }
                    __syncthreads();
                }
                uint32_t scales[2][WORDS], zeros[2][ZERO_WORDS];  // quarter i: of the i-th step from the last multiple of four on
                for (int b = b0, it = 0; b < b1; b += AHEAD, it = (it + 1) & 3) {
                    if (it == 0) {
                        const int mine = b + AHEAD * quarter, g0 = PER_BLOCK * mine;
                        if (a.blocks_per_group == 1 && g0 + GROUPS <= a.groups) {
#pragma unroll
                            for (int g = 0; g < 2; g++) {
                                __builtin_memcpy(scales[g], m.scale + meta[g] + g0, 2 * GROUPS);
                                if (m.zero) __builtin_memcpy(zeros[g], m.zero + meta[g] + g0, GROUPS);
                            }
                        } else {
#pragma unroll
                            for (int g = 0; g < 2; g++) {
#pragma unroll
                                for (int i = 0; i < WORDS; i++) scales[g][i] = 0;
#pragma unroll
                                for (int i = 0; i < ZERO_WORDS; i++) zeros[g][i] = 0;
#pragma unroll
                                for (int i = 0; i < GROUPS; i++) {
                                    const int of = a.blocks_per_group > 1 ? (mine + i) / a.blocks_per_group : g0 + i;
                                    const size_t at = meta[g] + min(of, a.groups - 1);
                                    scales[g][i / 2] |= (uint32_t)m.scale[at] << (16 * (i % 2));
                                    if (m.zero) zeros[g][i / 4] |= (uint32_t)m.zero[at] << (8 * (i % 4));
                                }
                            }
                        }
                    }
                    u32x4 w[AHEAD][2];
#pragma unroll
                    for (int u = 0; u < AHEAD; u++)
#pragma unroll
                        for (int g = 0; g < 2; g++)
#pragma unroll
                            for (int s = 0; s < 4; s++) w[u][g][s] = (uint32_t)__builtin_amdgcn_ds_bpermute(from_lane, (int)w_next[u][g][s]);
                    load_w(b + AHEAD);
                    uint32_t scale_of[2][WORDS], zero_of[2][ZERO_WORDS];
                    const int from_step = 4 * (n16 + 16 * it);
#pragma unroll
                    for (int g = 0; g < 2; g++) {
#pragma unroll
                        for (int i = 0; i < WORDS; i++) scale_of[g][i] = (uint32_t)__builtin_amdgcn_ds_bpermute(from_step, (int)scales[g][i]);
                        if (m.zero) {
#pragma unroll
                            for (int i = 0; i < ZERO_WORDS; i++) zero_of[g][i] = (uint32_t)__builtin_amdgcn_ds_bpermute(from_step, (int)zeros[g][i]);
                        }
                    }
#pragma unroll
                    for (int u = 0; u < AHEAD; u++) {
                        if (b + u >= b1) break;
                        const uint16_t *x_at = s_x + kInt4BlockCols * (b + u - c0) + 8 * quarter;
                        const float *sum_at = s_sum + PER_BLOCK * (b + u - c0) * (16 * TILES) + 4 * quarter;
#pragma unroll
                        for (int s = 0; s < 4; s++) {
                            const int in_block = s * PER_BLOCK / 4, i = u * PER_BLOCK + in_block;
                            if (s * PER_BLOCK % 4 == 0) {
#pragma unroll
                                for (int g = 0; g < 2; g++) {
                                    const float zero = m.zero ? -16.0f - (float)((zero_of[g][i / 4] >> (8 * (i % 4))) & 255u) : -24.0f;
#pragma unroll
                                    for (int t = 0; t < TILES; t++)
                                        sum[g][t] = zero * *reinterpret_cast<const f32x4 *>(sum_at + in_block * 16 * TILES + 16 * t);
                                }
                            }
                            const bf16x8 w0 = int4_plus16(w[u][0][s]), w1 = int4_plus16(w[u][1][s]);
#pragma unroll
                            for (int t = 0; t < TILES; t++) {
                                const bf16x8 xf = *reinterpret_cast<const bf16x8 *>(x_at + min(16 * t + n16, ntok - 1) * ld_s + 32 * s);
                                sum[0][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf, w0, sum[0][t], 0, 0, 0);
                                sum[1][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf, w1, sum[1][t], 0, 0, 0);
                            }
                            if ((s + 1) * PER_BLOCK % 4) continue;
#pragma unroll
                            for (int g = 0; g < 2; g++) {
                                const float scale = half_bits_to_float((uint16_t)(scale_of[g][i / 2] >> (16 * (i % 2))));
#pragma unroll
                                for (int t = 0; t < TILES; t++)
#pragma unroll
                                    for (int k = 0; k < 4; k++) acc[g][t][k] = fmaf(scale, sum[g][t][k], acc[g][t][k]);
                            }
                        }
                    }
                }
            }
            f32x4 *mine = joined + (size_t)(in_group * a.split) * 2 * TILES * 64;
            if (a.split > 1) {
#pragma unroll
                for (int g = 0; g < 2; g++)
#pragma unroll
                    for (int t = 0; t < TILES; t++) mine[((part * 2 + g) * TILES + t) * 64 + lane] = acc[g][t];
                __syncthreads();
            }
#pragma unroll
            for (int t = 0; t < TILES; t++) {
                if (t % a.split != part) continue;  // a tile of tokens is joined by one of the wavefronts
                if (16 * t >= ntok) break;
                if (a.split > 1) {
#pragma unroll
                    for (int g = 0; g < 2; g++) {
                        f32x4 v = mine[(g * TILES + t) * 64 + lane];
                        for (int p = 1; p < a.split; p++) v += mine[((p * 2 + g) * TILES + t) * 64 + lane];
                        acc[g][t] = v;
                    }
                }
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const int in_tile = 16 * t + 4 * quarter + k;
                    if (in_tile >= ntok) continue;
                    const int token = a.perm ? a.perm[slot0 + in_tile] : slot0 + in_tile;
                    const size_t out_row = a.out_by_slot ? slot0 + in_tile : token;
                    const float gate = a.gate ? a.gate[token] : 1.0f;
                    const int r = unit_rows * tile + n16;
                    if (gated) {
                        if (r < a.rows) int4_store(a, out_row, gate, r, int4_gated(acc[0][t][k], acc[1][t][k], a.activation));
                    } else {
                        if (r < a.rows) int4_store(a, out_row, gate, r, acc[0][t][k]);
                        if (r + 16 < a.rows) int4_store(a, out_row, gate, r + 16, acc[1][t][k]);
                    }
                }
            }
            if (a.split > 1) __syncthreads();  // before the next tile's sums overwrite these
        }
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

template <int TILES, int PER_BLOCK>
qmoe_status launch_rows_variant(const Int4Args &a, int grid, int threads, hipStream_t s)
{
    const size_t smem = a.x_bytes + a.sum_bytes + (a.split > 1 ? (size_t)(threads / 64) * 2 * TILES * 64 * sizeof(f32x4) : 0);
    const qmoe_status st = allow_lds(k_int4_rows<TILES, PER_BLOCK>, smem);
    if (st != QMOE_OK) return st;
    hipLaunchKernelGGL((k_int4_rows<TILES, PER_BLOCK>), dim3(grid), dim3(threads), smem, s, a);
    QMOE_HIP_TRY(hipGetLastError());
    return QMOE_OK;
}

// tiles: tiles of 16 tokens of an item; items: how many the call has, about
qmoe_status launch_rows_kernel(Int4Args a, int tiles, long long items, int cus, hipStream_t s)
{
    const int unit_rows = int4_is_gated(a.activation) ? 16 : 32, row_tiles = (a.rows + unit_rows - 1) / unit_rows;
    const long long units = items * row_tiles;
    a.split = 1;
    while (a.split < kInt4MaxSplit && units * a.split < 8LL * cus && 2 * a.split <= a.blocks) a.split *= 2;
    const int threads = 64 * (a.split < 4 ? 4 : a.split);
    const int side_by_side = threads / 64 / a.split;
    // several tiles a wavefront where that leaves enough workgroups: the activations are staged once for them
    a.reps = (int)std::min<long long>(2, std::max<long long>(1, items * row_tiles / (16LL * cus * side_by_side)));
    const long long groups = items * ((row_tiles + side_by_side * a.reps - 1) / (side_by_side * a.reps));
    const int tokens = 16 * (tiles <= 1 ? 1 : tiles <= 2 ? 2 : 4);
    a.x_bytes = (uint32_t)std::min<size_t>(kInt4XBytes, (size_t)tokens * 2 * (a.blocks * kInt4BlockCols + 8));
    const int grid = (int)std::min<long long>(groups, 64LL * cus);
    a.sum_bytes = (uint32_t)std::min<size_t>(kInt4XBytes / 4, (size_t)tokens * 4 * a.blocks * a.per_block);
    const int variant = (tiles <= 1 ? 0 : tiles <= 2 ? 3 : 6) + (a.per_block == 1 ? 0 : a.per_block == 2 ? 1 : 2);
    switch (variant) {
    case 0: return launch_rows_variant<1, 1>(a, grid, threads, s);
    case 1: return launch_rows_variant<1, 2>(a, grid, threads, s);
    case 2: return launch_rows_variant<1, 4>(a, grid, threads, s);
    case 3: return launch_rows_variant<2, 1>(a, grid, threads, s);
    case 4: return launch_rows_variant<2, 2>(a, grid, threads, s);
    case 5: return launch_rows_variant<2, 4>(a, grid, threads, s);
    case 6: return launch_rows_variant<4, 1>(a, grid, threads, s);
    case 7: return launch_rows_variant<4, 2>(a, grid, threads, s);
    default: return launch_rows_variant<4, 4>(a, grid, threads, s);
    }
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
    const bool crowded = n_tokens > kInt4AllFew;
    GroupedTokens g;
    if ((st = group_by_expert(expert_idx, n_tokens, n_experts, d_model, d_ff, kInt4FewTokens,
                              crowded ? kInt4FewTokens + 1 : 0x7FFFFFFF, workspace, static_cast<float *>(y),
                              y_type == QMOE_F32 ? d_model : d_model / 2, s, &g)) != QMOE_OK)
        return st;
    Int4Args a{};
    a.mats = wi;
    a.n_experts = n_experts;
    a.perm = g.perm;
    a.x = x_bf16;
    a.ld_x = d_model;
    a.out = g.hidden;
    a.ld_out = d_ff;
    a.out_by_slot = 1;
    a.activation = activation;
    fill_shape(&a, d_ff, d_model, group);
    auto product = [&]() {
        a.items = g.few;
        a.n_items_dev = g.n_few;
        a.max_items = std::min(n_tokens, n_experts + n_tokens / kInt4FewTokens);
        qmoe_status r = launch_rows_kernel(a, 1, a.max_items, di.cus, s);
        if (r != QMOE_OK || !crowded) return r;
        a.items = g.many;
        a.n_items_dev = g.n_many;
        a.max_items = n_tokens / kInt4FewTokens;  // (each has more than that, or stands beside a whole tile)
        return launch_mm_kernel(a, true, di.cus, s);
    };
    if ((st = product()) != QMOE_OK) return st;
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
    return product();
}

}  // extern "C"
